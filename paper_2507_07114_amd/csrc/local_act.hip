// 8-bit activation checkpoints (include/lossy_local.h): ll_act_pack and
// ll_act_unpack.  Bound by HBM: 8 x 4096 x 11008 bf16 columns move 1093 MB each
// way, at 6.1 TB/s over the two in a long run of calls (5.1 in some of the first
// twenty after a pause).
#include <hip/hip_runtime.h>

#include "local.h"
#include "local_device.h"

namespace lossy {

namespace {

// Units of a lane, loaded together.  Inputs through the caches (what a layer just
// wrote may be there), outputs past them.  8 x 4096 x 11008 bf16, us (pack /
// unpack): 1 unit 239 / 174, 2 188 / 171, 4 186 / 183; outputs through the caches
// cost 2 and 4% more.  Of 11007 columns: 196 / 188.
constexpr int kPer = 2;
constexpr bool kStreamIn = false, kStreamOut = true;
typedef float f32x2 __attribute__((ext_vector_type(2)));

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

// Token rows and units of a lane, and whether they lie inside their batch.  The
// lengths of all of them are loaded together.
template <int PER>
__device__ __forceinline__ void flat_units(const PackParams& p, const FlatRows& f, uint32_t base,
                                           int64_t (&tk)[PER], uint32_t (&unit)[PER],
                                           bool (&in)[PER]) {
#pragma unroll
    for (int a = 0; a < PER; ++a) {
        const uint32_t w = base + a * kBlock, row = flat_row(f, w);
        unit[a] = w - row * f.units;
        tk[a] = (int64_t)blockIdx.y * f.rows + row;
        in[a] = row < f.rows && tk[a] < f.total;
    }
    if (p.lengths) {
        int32_t length[PER];
        uint32_t j[PER];
#pragma unroll
        for (int a = 0; a < PER; ++a) {
            const uint32_t at = in[a] ? (uint32_t)tk[a] : 0, i = at / (uint32_t)p.t;
            j[a] = at - i * (uint32_t)p.t;
            length[a] = p.lengths[i];
        }
#pragma unroll
        for (int a = 0; a < PER; ++a) in[a] = in[a] && (int64_t)j[a] < length[a];
    }
}

// The first `have` columns of a short unit, held as the last of U (NARROW: as the
// first), in front and zeros behind.
template <int U, bool NARROW>
__device__ __forceinline__ void own_first(int have, float (&v)[U]) {
    if (!NARROW) {
#pragma unroll
        for (int b = 1; b < U; b *= 2)
            if ((U - have) & b)
#pragma unroll
                for (int c = 0; c < U; ++c) v[c] = c + b < U ? v[c + b] : 0.0f;
    }
#pragma unroll
    for (int c = 0; c < U; ++c) v[c] = c < have ? v[c] : 0.0f;
}

// A lane takes units of 16 bytes of x; the 4 or 8 lanes of a group agree on its
// scale.  One pass: x read once, codes and scales written once.  Rows count
// whole groups of lanes (units past the row's end carry zeros), so that a group's
// lanes are always together.
template <class X, bool NARROW>
__device__ __forceinline__ void pack_units(const PackParams& p, const FlatRows& f) {
    typedef typename X::T XT;
    constexpr int U = 16 / (int)sizeof(XT), kLanes = kActGroup / U;
    const uint32_t base = blockIdx.x * (uint32_t)(kBlock * kPer) + threadIdx.x;
    Packed<XT, U> x[kPer];
    int64_t have[kPer], tk[kPer];
    uint32_t unit[kPer];
    bool in[kPer];
    flat_units<kPer>(p, f, base, tk, unit, in);
#pragma unroll
    for (int a = 0; a < kPer; ++a) {
        const int64_t c0 = (int64_t)unit[a] * U;
        have[a] = in[a] ? (p.h > c0 ? p.h - c0 : 0) : -1;
        x[a] = {};
        if (have[a] > 0)  // a short unit as the end of the row's last U columns
            x[a] = Columns<U>{c0, p.h}.template load<XT, kStreamIn, NARROW>(
                static_cast<const XT*>(p.x.p) + tk[a] * p.x.ld);
    }
#pragma unroll
    for (int a = 0; a < kPer; ++a) {
        if (have[a] < 0) continue;
        float v[U];
        widen(x[a], v);
        if (have[a] < U) own_first<U, NARROW>((int)have[a], v);
        uint8_t* q = p.c.q + tk[a] * p.c.ld_q + (int64_t)unit[a] * U;
        uint32_t top = 0, all = 0;
#pragma unroll
        for (int c = 0; c < U; ++c) {
            const uint32_t x = __float_as_uint(v[c]) & 0x7FFFFFFFu;
            top = max(top, finite_bits(x) ? x : 0u);
            all = max(all, x);
        }
        const int k = group_exp(group_max<kLanes>(top));
        if (unit[a] % kLanes == 0)
            p.c.s[tk[a] * p.c.ld_s + unit[a] / kLanes] = (uint8_t)(k + 127);
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
        if (have[a] >= U) {
            typename RawOf<U>::T raw;
            __builtin_memcpy(&raw, code, U);
            store_raw<U, 1, kStreamOut>(q, raw);
        } else {
#pragma unroll
            for (int c = 0; c < U; ++c)
                if (c < have[a]) q[c] = (uint8_t)(code[c / 4] >> (8 * (c % 4)));
        }
    }
}

template <class X>
__global__ __launch_bounds__(kBlock) void k_act_pack(PackParams p, FlatRows f) {
    if (p.h < 16 / (int)sizeof(typename X::T)) pack_units<X, true>(p, f);
    else pack_units<X, false>(p, f);
}

template <class O, bool NARROW>
__device__ __forceinline__ void unpack_units(const PackParams& p, const FlatRows& f) {
    typedef typename O::T OT;
    constexpr int U = 16 / (int)sizeof(OT);
    const uint32_t base = blockIdx.x * (uint32_t)(kBlock * kPer) + threadIdx.x;
    Packed<uint8_t, U> code[kPer] = {};
    uint8_t s[kPer] = {};
    int64_t tk[kPer];
    uint32_t unit[kPer];
    bool in[kPer];
    flat_units<kPer>(p, f, base, tk, unit, in);
#pragma unroll
    for (int a = 0; a < kPer; ++a) {
        const int64_t c0 = (int64_t)unit[a] * U;
        if (in[a]) {
            s[a] = p.c.s[tk[a] * p.c.ld_s + c0 / kActGroup];
            code[a] = Columns<U>{c0, p.h}.template load<uint8_t, kStreamIn, NARROW>(
                p.c.q + tk[a] * p.c.ld_q);
        }
    }
#pragma unroll
    for (int a = 0; a < kPer; ++a) {
        if (!in[a]) continue;
        const int64_t c0 = (int64_t)unit[a] * U, have = p.h - c0;
        const float scale = __uint_as_float((uint32_t)s[a] << 23);
        float v[U];
#pragma unroll
        for (int w = 0; w < U / 4; ++w) {
            const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)code[a].w[w], false);
            const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)code[a].w[w], true);
            v[4 * w] = lo.x * scale;
            v[4 * w + 1] = lo.y * scale;
            v[4 * w + 2] = hi.x * scale;
            v[4 * w + 3] = hi.y * scale;
        }
        if (have < U) own_first<U, NARROW>((int)have, v);
        store_unit<OT, U, kStreamOut>(static_cast<OT*>(p.x.p) + tk[a] * p.x.ld + c0, have, v);
    }
}

template <class O>
__global__ __launch_bounds__(kBlock) void k_act_unpack(PackParams p, FlatRows f) {
    if (p.h < 16 / (int)sizeof(typename O::T)) unpack_units<O, true>(p, f);
    else unpack_units<O, false>(p, f);
}

}  // namespace

hipError_t launch_act_pack(const PackParams& p, hipStream_t s) {
    const int lanes = kActGroup / (p.x.bf16 ? 8 : 4);
    FlatRows f;
    dim3 grid;
    if (!flat_rows((int64_t)p.n * p.t, (p.h + kActGroup - 1) / kActGroup * lanes, kPer, &f, &grid))
        return hipErrorInvalidConfiguration;
    if (p.x.bf16) hipLaunchKernelGGL((k_act_pack<El16>), grid, dim3(kBlock), 0, s, p, f);
    else hipLaunchKernelGGL((k_act_pack<El32>), grid, dim3(kBlock), 0, s, p, f);
    return hipGetLastError();
}

hipError_t launch_act_unpack(const PackParams& p, hipStream_t s) {
    const int u = p.x.bf16 ? 8 : 4;
    FlatRows f;
    dim3 grid;
    if (!flat_rows((int64_t)p.n * p.t, (p.h + u - 1) / u, kPer, &f, &grid))
        return hipErrorInvalidConfiguration;
    if (p.x.bf16) hipLaunchKernelGGL((k_act_unpack<El16>), grid, dim3(kBlock), 0, s, p, f);
    else hipLaunchKernelGGL((k_act_unpack<El32>), grid, dim3(kBlock), 0, s, p, f);
    return hipGetLastError();
}

}  // namespace lossy
