// Local-gradient operators (include/lossy_local.h): embedding lookup and
// gradient, 8-bit activation checkpoints, weight gradient from a checkpoint.
#include <hip/hip_runtime.h>

#include "local.h"

namespace lossy {

namespace {

constexpr int kBlock = 256;

// Element types of rows and activations.
struct El32 {
    typedef float T;
};
struct El16 {
    typedef __bf16 T;
};

template <class T>
__device__ __forceinline__ float widen(T x) {
    return (float)x;
}

template <class T>
__device__ __forceinline__ T narrow(float x) {
    return (T)x;  // round to nearest even
}

// Tokens of worker i's batch.
__device__ __forceinline__ int64_t batch_len(const int32_t* lengths, int i, int64_t t) {
    if (!lengths) return t;
    const int64_t m = lengths[i];
    return m < 0 ? 0 : (m > t ? t : m);
}

// Table row of token j of worker i, or -1 where the table does not hold it.
__device__ __forceinline__ int64_t table_row(const TokenView& tok, int i, int64_t j) {
    const int64_t at = (int64_t)i * tok.ld + j;
    const int64_t id = tok.wide ? static_cast<const int64_t*>(tok.ids)[at]
                                : (int64_t) static_cast<const int32_t*>(tok.ids)[at];
    // held ids are first .. first + v - 1; the unsigned difference wraps where
    // id < first, and where id - first would overflow
    const uint64_t row = (uint64_t)id - (uint64_t)tok.first;
    return row < (uint64_t)tok.v ? (int64_t)row : -1;
}

unsigned grid_for(int64_t blocks) {
    const int64_t cap = 1 << 20;
    return (unsigned)(blocks < 1 ? 1 : (blocks > cap ? cap : blocks));
}

// ---- embedding lookup --------------------------------------------------

template <class R, class O>
__global__ __launch_bounds__(kBlock) void k_embed(EmbedParams p) {
    typedef typename R::T RT;
    typedef typename O::T OT;
    for (int64_t tk = blockIdx.x; tk < (int64_t)p.n * p.t; tk += gridDim.x) {
        const int i = (int)(tk / p.t);
        const int64_t j = tk - i * p.t;
        if (j >= batch_len(p.lengths, i, p.t)) continue;
        const int64_t row = table_row(p.tok, i, j);
        const RT* src = static_cast<const RT*>(p.table.p) + i * p.table.ld + p.table.offset +
                        (row < 0 ? 0 : row) * p.h;
        OT* dst = static_cast<OT*>(p.out.p) + tk * p.out.ld;
        for (int64_t c = threadIdx.x; c < p.h; c += kBlock)
            dst[c] = narrow<OT>(row < 0 ? 0.0f : p.scale * widen(src[c]));
    }
}

// ---- embedding gradient --------------------------------------------------

// One workgroup per table row; it looks through the worker's tokens in order.
template <class Y, class G>
__global__ __launch_bounds__(kBlock) void k_embed_grad(EmbedGradParams p) {
    typedef typename Y::T YT;
    typedef typename G::T GT;
    const int64_t v = p.tok.v;
    for (int64_t w = blockIdx.x; w < (int64_t)p.n * v; w += gridDim.x) {
        const int i = (int)(w / v);
        const int64_t row = w - i * v;
        const int64_t m = batch_len(p.lengths, i, p.t);
        GT* dst = static_cast<GT*>(p.grads.p) + i * p.grads.ld + p.grads.offset + row * p.h;
        for (int64_t c = threadIdx.x; c < p.h; c += kBlock) {
            float sum = 0.0f;
            bool any = false;
            for (int64_t j = 0; j < m; ++j) {
                if (table_row(p.tok, i, j) != row) continue;
                any = true;
                sum += widen(static_cast<const YT*>(p.dy.p)[(i * p.t + j) * p.dy.ld + c]);
            }
            if (p.accumulate) {
                if (any) dst[c] = narrow<GT>(__builtin_fmaf(p.scale, sum, widen(dst[c])));
            } else {
                dst[c] = narrow<GT>(any ? p.scale * sum : 0.0f);
            }
        }
    }
}

// ---- 8-bit checkpoints -----------------------------------------------------

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

// e4m3 code of x * 2^-k (|x| <= 448 * 2^k), or of NaN where x is not finite.
__device__ __forceinline__ uint32_t e4m3_code(float x, float inv, float limit) {
    const float z = __builtin_amdgcn_fmed3f(x * inv, -limit, limit);
    const uint32_t c = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(z, 0.0f, 0, false) & 0xFFu;
    return finite_bits(__float_as_uint(x)) ? c : 0x7Fu;
}

template <class X>
__global__ __launch_bounds__(kBlock) void k_act_pack(PackParams p) {
    typedef typename X::T XT;
    const int64_t groups = (p.h + kActGroup - 1) / kActGroup;
    const int64_t total = (int64_t)p.n * p.t * groups;
    for (int64_t w = (int64_t)blockIdx.x * kBlock + threadIdx.x; w < total;
         w += (int64_t)gridDim.x * kBlock) {
        const int64_t tk = w / groups;
        const int64_t g = w - tk * groups;
        const int i = (int)(tk / p.t);
        if (tk - i * p.t >= batch_len(p.lengths, i, p.t)) continue;
        const int64_t c0 = g * kActGroup;
        const int64_t c1 = c0 + kActGroup < p.h ? c0 + kActGroup : p.h;
        const XT* x = static_cast<const XT*>(p.x.p) + tk * p.x.ld;
        uint32_t top = 0;
        for (int64_t c = c0; c < c1; ++c) {
            const uint32_t a = __float_as_uint(widen(x[c])) & 0x7FFFFFFFu;
            if (finite_bits(a) && a > top) top = a;
        }
        const int k = group_exp(top);
        p.c.s[tk * p.c.ld_s + g] = (uint8_t)(k + 127);
        const float inv = exp2_int(-k), limit = code_limit(k);
        for (int64_t c = c0; c < c1; ++c)
            p.c.q[tk * p.c.ld_q + c] = (uint8_t)e4m3_code(widen(x[c]), inv, limit);
    }
}

__device__ __forceinline__ float e4m3_value(uint32_t code, uint32_t s) {
    return __builtin_amdgcn_cvt_f32_fp8((int)code, 0) * __uint_as_float(s << 23);
}

template <class O>
__global__ __launch_bounds__(kBlock) void k_act_unpack(PackParams p) {
    typedef typename O::T OT;
    const int64_t total = (int64_t)p.n * p.t * p.h;
    for (int64_t w = (int64_t)blockIdx.x * kBlock + threadIdx.x; w < total;
         w += (int64_t)gridDim.x * kBlock) {
        const int64_t tk = w / p.h;
        const int64_t c = w - tk * p.h;
        const int i = (int)(tk / p.t);
        if (tk - i * p.t >= batch_len(p.lengths, i, p.t)) continue;
        static_cast<OT*>(p.x.p)[tk * p.x.ld + c] = narrow<OT>(e4m3_value(
            p.c.q[tk * p.c.ld_q + c], p.c.s[tk * p.c.ld_s + c / kActGroup]));
    }
}

// ---- weight gradient ----------------------------------------------------------

constexpr int kWT = 32;  // tile edge and tokens a turn

template <class Y, class G>
__global__ __launch_bounds__(kBlock) void k_act_wgrad(WgradParams p) {
    typedef typename Y::T YT;
    typedef typename G::T GT;
    __shared__ float ys[kWT][kWT], xs[kWT][kWT];
    const int64_t to = (p.o + kWT - 1) / kWT, th = (p.h + kWT - 1) / kWT;
    for (int64_t w = blockIdx.x; w < p.n * to * th; w += gridDim.x) {
        const int i = (int)(w / (to * th));
        const int64_t o0 = (w / th % to) * kWT, h0 = (w % th) * kWT;
        const int64_t m = batch_len(p.lengths, i, p.t);
        const int tx = threadIdx.x % kWT, ty = threadIdx.x / kWT;  // 32 x 8
        float acc[4] = {};
        for (int64_t j0 = 0; j0 < m; j0 += kWT) {
            for (int a = ty; a < kWT; a += 8) {
                const int64_t j = j0 + a, tk = i * p.t + j;
                const bool in = j < m;
                ys[a][tx] = in && o0 + tx < p.o
                                ? widen(static_cast<const YT*>(p.dy.p)[tk * p.dy.ld + o0 + tx])
                                : 0.0f;
                xs[a][tx] = in && h0 + tx < p.h
                                ? e4m3_value(p.x.q[tk * p.x.ld_q + h0 + tx],
                                             p.x.s[tk * p.x.ld_s + (h0 + tx) / kActGroup])
                                : 0.0f;
            }
            __syncthreads();
            for (int a = 0; a < kWT; ++a)
                for (int b = 0; b < 4; ++b)
                    acc[b] = __builtin_fmaf(ys[a][ty + 8 * b], xs[a][tx], acc[b]);
            __syncthreads();
        }
        GT* dst = static_cast<GT*>(p.grads.p) + i * p.grads.ld + p.grads.offset;
        for (int b = 0; b < 4; ++b) {
            const int64_t r = o0 + ty + 8 * b, c = h0 + tx;
            if (r >= p.o || c >= p.h) continue;
            GT* d = dst + r * p.h + c;
            *d = narrow<GT>(p.accumulate ? __builtin_fmaf(p.scale, acc[b], widen(*d))
                                         : p.scale * acc[b]);
        }
    }
}

}  // namespace

// Launch K<A, B> for the element types given as truth values (bf16?).
#define LOSSY_LAUNCH2(K, a, b, grid, s, p)                                                  \
    do {                                                                                    \
        if ((a) && (b)) hipLaunchKernelGGL((K<El16, El16>), grid, dim3(kBlock), 0, s, p);   \
        else if (a) hipLaunchKernelGGL((K<El16, El32>), grid, dim3(kBlock), 0, s, p);       \
        else if (b) hipLaunchKernelGGL((K<El32, El16>), grid, dim3(kBlock), 0, s, p);       \
        else hipLaunchKernelGGL((K<El32, El32>), grid, dim3(kBlock), 0, s, p);              \
    } while (0)

hipError_t launch_embed(const EmbedParams& p, hipStream_t s) {
    const dim3 grid(grid_for((int64_t)p.n * p.t));
    LOSSY_LAUNCH2(k_embed, p.table.bf16, p.out.bf16, grid, s, p);
    return hipGetLastError();
}

size_t embed_grad_workspace(int64_t, int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_embed_grad(const EmbedGradParams& p, void*, hipStream_t s) {
    const dim3 grid(grid_for((int64_t)p.n * p.tok.v));
    LOSSY_LAUNCH2(k_embed_grad, p.dy.bf16, p.grads.bf16, grid, s, p);
    return hipGetLastError();
}

hipError_t launch_act_pack(const PackParams& p, hipStream_t s) {
    const int64_t groups = (p.h + kActGroup - 1) / kActGroup;
    const dim3 grid(grid_for(((int64_t)p.n * p.t * groups + kBlock - 1) / kBlock));
    if (p.x.bf16) hipLaunchKernelGGL((k_act_pack<El16>), grid, dim3(kBlock), 0, s, p);
    else hipLaunchKernelGGL((k_act_pack<El32>), grid, dim3(kBlock), 0, s, p);
    return hipGetLastError();
}

hipError_t launch_act_unpack(const PackParams& p, hipStream_t s) {
    const dim3 grid(grid_for(((int64_t)p.n * p.t * p.h + kBlock - 1) / kBlock));
    if (p.x.bf16) hipLaunchKernelGGL((k_act_unpack<El16>), grid, dim3(kBlock), 0, s, p);
    else hipLaunchKernelGGL((k_act_unpack<El32>), grid, dim3(kBlock), 0, s, p);
    return hipGetLastError();
}

size_t act_wgrad_workspace(int64_t, int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_act_wgrad(const WgradParams& p, void*, hipStream_t s) {
    const dim3 grid(grid_for(p.n * ((p.o + kWT - 1) / kWT) * ((p.h + kWT - 1) / kWT)));
    LOSSY_LAUNCH2(k_act_wgrad, p.dy.bf16, p.grads.bf16, grid, s, p);
    return hipGetLastError();
}

}  // namespace lossy
