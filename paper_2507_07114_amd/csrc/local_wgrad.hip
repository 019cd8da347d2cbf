// Weight gradient of a linear layer from an 8-bit checkpoint of its input
// (include/lossy_local.h): ll_act_wgrad.
#include <hip/hip_runtime.h>

#include "local.h"
#include "local_device.h"

namespace lossy {

namespace {

__device__ __forceinline__ float e4m3_value(uint32_t code, uint32_t s) {
    return __builtin_amdgcn_cvt_f32_fp8((int)code, 0) * __uint_as_float(s << 23);
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

size_t act_wgrad_workspace(int64_t, int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_act_wgrad(const WgradParams& p, void*, hipStream_t s) {
    const dim3 grid(grid_for(p.n * ((p.o + kWT - 1) / kWT) * ((p.h + kWT - 1) / kWT)));
    LOSSY_LAUNCH2(k_act_wgrad, p.dy.bf16, p.grads.bf16, grid, dim3(kBlock), s, p);
    return hipGetLastError();
}

}  // namespace lossy
