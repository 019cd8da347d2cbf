// 8-bit activation checkpoints (include/lossy_local.h): ll_act_pack and
// ll_act_unpack.
#include <hip/hip_runtime.h>

#include "local.h"
#include "local_device.h"

namespace lossy {

namespace {

// Exponent k of a group's scale from the bits of its largest finite |x|:
// 448 = 1.75 * 2^8, so a = f * 2^e (1 <= f < 2) needs k = e - 8, or e - 7
// where f > 1.75.
__device__ __forceinline__ int group_exp(uint32_t a) {
    const int e = (int)(a >> 23) - 127;
    const int k = e - 8 + ((a & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return k < kActMinExp ? kActMinExp : k;
}

__device__ __forceinline__ float exp2_int(int k) { return __uint_as_float((uint32_t)(k + 127) << 23); }

__device__ __forceinline__ bool finite_bits(uint32_t a) { return (a & 0x7F800000u) != 0x7F800000u; }

// Largest magnitude that a group of exponent k stores: 448, but 240 where 256
// times the scale is 2^128, which no type of the restored values holds.
__device__ __forceinline__ float code_limit(int k) { return k == 120 ? 240.0f : 448.0f; }

// Largest of x over the aligned 4 (LANES = 4) or 8 lanes of a group, by
// data-parallel moves inside the row of 16 lanes.
template <int LANES>
__device__ __forceinline__ uint32_t group_max(uint32_t x) {
    auto with = [&](int moved) { x = max(x, (uint32_t)moved); };
    with(__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, true));   // lane ^ 1
    with(__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, true));   // lane ^ 2
    if (LANES == 8) with(__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xF, 0xF, true));  // 7 - lane
    return x;
}

// A lane takes one unit (16 bytes of x); the 4 or 8 lanes of a group agree on
// its scale.  One pass: x read once, codes and scales written once.  All
// lanes of a group stay in the loop together (units past the row's end carry
// zeros), which the group's maximum needs.
template <class X>
__global__ __launch_bounds__(kBlock) void k_act_pack(PackParams p, int lanes) {
    typedef typename X::T XT;
    constexpr int U = 16 / (int)sizeof(XT), kLanes = kActGroup / U;
    const int rows = kBlock / lanes, lane = threadIdx.x % lanes;
    const int64_t total = (int64_t)p.n * p.t;
    const int64_t units = (p.h + kActGroup - 1) / kActGroup * kLanes;
    for (int64_t tk = (int64_t)blockIdx.x * rows + threadIdx.x / lanes; tk < total;
         tk += (int64_t)gridDim.x * rows) {
        if (!in_batch(p.lengths, (uint32_t)tk, p.t)) continue;
        const XT* x = static_cast<const XT*>(p.x.p) + tk * p.x.ld;
        uint8_t* q = p.c.q + tk * p.c.ld_q;
        uint8_t* s = p.c.s + tk * p.c.ld_s;
        for (int64_t u = lane; u < units; u += lanes) {
            const int64_t c0 = u * U;
            const int64_t have = p.h - c0;
            float v[U];
            load_unit<XT, U, true>(x + c0, have, v);
            uint32_t top = 0, all = 0;
#pragma unroll
            for (int c = 0; c < U; ++c) {
                const uint32_t a = __float_as_uint(v[c]) & 0x7FFFFFFFu;
                top = max(top, finite_bits(a) ? a : 0u);
                all = max(all, a);
            }
            const int k = group_exp(group_max<kLanes>(top));
            if (u % kLanes == 0) s[u / kLanes] = (uint8_t)(k + 127);
            const float inv = exp2_int(-k), limit = code_limit(k);
            uint32_t code[U / 4];
#pragma unroll
            for (int w = 0; w < U / 4; ++w) {
                float z[4];
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    z[c] = __builtin_amdgcn_fmed3f(v[4 * w + c] * inv, -limit, limit);
                int r = __builtin_amdgcn_cvt_pk_fp8_f32(z[0], z[1], 0, false);
                code[w] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(z[2], z[3], r, true);
            }
            if (!finite_bits(all)) {  // rare: what is not finite becomes NaN
#pragma unroll
                for (int c = 0; c < U; ++c) {
                    const uint32_t byte = 0xFFu << (8 * (c % 4));
                    if (!finite_bits(__float_as_uint(v[c]) & 0x7FFFFFFFu))
                        code[c / 4] = (code[c / 4] & ~byte) | (0x7F7F7F7Fu & byte);
                }
            }
            if (have >= U) {
                typename RawOf<U>::T raw;
                __builtin_memcpy(&raw, code, U);
                store_raw<U, 1, true>(q + c0, raw);
            } else {
#pragma unroll
                for (int c = 0; c < U; ++c)
                    if (c < have) q[c0 + c] = (uint8_t)(code[c / 4] >> (8 * (c % 4)));
            }
        }
    }
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

template <class O>
__global__ __launch_bounds__(kBlock) void k_act_unpack(PackParams p, int lanes) {
    typedef typename O::T OT;
    constexpr int U = 16 / (int)sizeof(OT);
    const int rows = kBlock / lanes, lane = threadIdx.x % lanes;
    const int64_t total = (int64_t)p.n * p.t;
    const int64_t units = (p.h + U - 1) / U;
    for (int64_t tk = (int64_t)blockIdx.x * rows + threadIdx.x / lanes; tk < total;
         tk += (int64_t)gridDim.x * rows) {
        if (!in_batch(p.lengths, (uint32_t)tk, p.t)) continue;
        OT* out = static_cast<OT*>(p.x.p) + tk * p.x.ld;
        const uint8_t* q = p.c.q + tk * p.c.ld_q;
        const uint8_t* s = p.c.s + tk * p.c.ld_s;
#pragma unroll 2
        for (int64_t u = lane; u < units; u += lanes) {
            const int64_t c0 = u * U;
            const int64_t have = p.h - c0;
            uint32_t code[U / 4] = {};
            if (have >= U) {
                auto raw = load_raw<U, 1, true>(q + c0);
                __builtin_memcpy(code, &raw, U);
            } else {
#pragma unroll
                for (int c = 0; c < U; ++c)
                    if (c < have) code[c / 4] |= (uint32_t)q[c0 + c] << (8 * (c % 4));
            }
            const float scale = __uint_as_float((uint32_t)s[c0 / kActGroup] << 23);
            float v[U];
#pragma unroll
            for (int w = 0; w < U / 4; ++w) {
                const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)code[w], false);
                const f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8((int)code[w], true);
                v[4 * w] = a.x * scale;
                v[4 * w + 1] = a.y * scale;
                v[4 * w + 2] = b.x * scale;
                v[4 * w + 3] = b.y * scale;
            }
            store_unit<OT, U, true>(out + c0, have, v);
        }
    }
}

}  // namespace

hipError_t launch_act_pack(const PackParams& p, hipStream_t s) {
    const int64_t rows = (int64_t)p.n * p.t;
    const int u = p.x.bf16 ? 8 : 4;
    const int lanes = lanes_per_row(rows, (p.h + u - 1) / u);
    const dim3 grid(grid_for((rows * lanes + kBlock - 1) / kBlock));
    if (p.x.bf16) hipLaunchKernelGGL((k_act_pack<El16>), grid, dim3(kBlock), 0, s, p, lanes);
    else hipLaunchKernelGGL((k_act_pack<El32>), grid, dim3(kBlock), 0, s, p, lanes);
    return hipGetLastError();
}

hipError_t launch_act_unpack(const PackParams& p, hipStream_t s) {
    const int64_t rows = (int64_t)p.n * p.t;
    const int u = p.x.bf16 ? 8 : 4;
    const int lanes = lanes_per_row(rows, (p.h + u - 1) / u);
    const dim3 grid(grid_for((rows * lanes + kBlock - 1) / kBlock));
    if (p.x.bf16) hipLaunchKernelGGL((k_act_unpack<El16>), grid, dim3(kBlock), 0, s, p, lanes);
    else hipLaunchKernelGGL((k_act_unpack<El32>), grid, dim3(kBlock), 0, s, p, lanes);
    return hipGetLastError();
}

}  // namespace lossy
