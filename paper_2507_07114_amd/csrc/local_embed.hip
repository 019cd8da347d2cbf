// Embedding lookup and gradient (include/lossy_local.h): ll_embed and
// ll_embed_grad.
#include <hip/hip_runtime.h>

#include "local.h"
#include "local_device.h"

namespace lossy {

namespace {

// ---- lookup: rows read at random, written in order -------------------------
//
// 128 lanes walk a row (fewer a short one, so that a workgroup takes more
// rows).  Table rows are read through the caches, which hold the frequent ones,
// and written past them.  8 workers' 8192 tokens of 4096 bf16 columns, us: this
// 147 to 150; 64 lanes 155; 256 lanes 150; four units of a lane in flight 154;
// rows dealt out flat, as in local_act.hip, 163; written through the caches 180.
// The distinct rows and the output are 752 MB (5.0 TB/s of them), the rows
// read with repetitions 1062 MB.

template <class R, class O>
__global__ __launch_bounds__(kBlock) void k_embed(EmbedParams p, int lanes) {
    typedef typename R::T RT;
    typedef typename O::T OT;
    constexpr int U = unit_of<R, O>();
    const int rows = kBlock / lanes, lane = threadIdx.x % lanes;
    const int64_t total = (int64_t)p.n * p.t;
    const int64_t units = (p.h + U - 1) / U;
    for (int64_t tk = (int64_t)blockIdx.x * rows + threadIdx.x / lanes; tk < total;
         tk += (int64_t)gridDim.x * rows) {
        const int i = (int)((uint32_t)tk / (uint32_t)p.t);
        const int64_t j = tk - (int64_t)i * p.t;
        if (p.lengths && j >= p.lengths[i]) continue;
        const int64_t row = table_row(p.tok, i, j);
        const RT* src = static_cast<const RT*>(p.table.p) + i * p.table.ld + p.table.offset +
                        (row < 0 ? 0 : row) * p.h;
        OT* dst = static_cast<OT*>(p.out.p) + tk * p.out.ld;
#pragma unroll 1
        for (int64_t u = lane; u < units; u += lanes) {
            const int64_t have = p.h - u * U;
            float v[U] = {};
            if (row >= 0) {
                load_unit<RT, U, false>(src + u * U, have, v);
#pragma unroll
                for (int c = 0; c < U; ++c) v[c] *= p.scale;
            }
            store_unit<OT, U, true>(dst + u * U, have, v);
        }
    }
}

// ---- gradient ----------------------------------------------------------------
//
// 1. k_token_sort groups every worker's token places by table row, in order
//    of the places inside a row.  The rows are dealt to 2^b slices by their low
//    bits (frequent ids lie side by side and would fill one slice), and a
//    workgroup sorts one slice by itself: it reads all the worker's tokens,
//    counts those of lower slices (its place in the output) and sorts its
//    own by counting.  No workgroup waits for another and one launch does.
// 2. k_embed_grad gives a wavefront a chunk of consecutive sorted tokens and a
//    strip of columns, whatever rows they belong to, so a row that takes half
//    of all tokens is summed by many wavefronts.  A row whose tokens lie in
//    one chunk is stored; the others leave fp32 partial sums.  More
//    wavefronts of the launch store zeros in the rows that have no token.
// 3. k_embed_grad_join adds the partial sums of rows that cross chunks, in
//    order.

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / kWave;
constexpr int kMaxBins = 512;  // table rows a slice can hold: 32 KiB of counts
constexpr int kMinSlices = 64;

struct Sorted {
    int32_t* row;    // [n][t] table rows, grouped
    int32_t* place;  // [n][t] token places, ascending inside a row
    int32_t* count;  // [n][v] tokens of each table row
    int32_t* held;   // [n] sorted tokens of a worker
    int log_slices;
};

struct GradPlan {
    Sorted s;
    float* part;    // [n][chunks][2][h] partial sums
    int chunk;      // sorted tokens of a wavefront
    int64_t chunks, strips;
    int64_t chunk_waves, zero_waves;
};

constexpr int kZeroRows = 4;  // table rows of a wavefront that stores zeros

__global__ __launch_bounds__(kSortThreads) void k_token_sort(int64_t t, const int32_t* lengths,
                                                            TokenView tok, Sorted o) {
    __shared__ int hist[kSortWaves][kMaxBins];
    __shared__ int wave_less[kSortWaves], wave_sum[kMaxBins / kWave];
    const int slices = 1 << o.log_slices;
    const int i = (int)(blockIdx.x >> o.log_slices), slice = (int)(blockIdx.x & (slices - 1));
    const int w = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int64_t m = batch_len(lengths, i, t);
    // rows slice, slice + slices, ... below v
    const int bins = slice < tok.v ? (int)((tok.v - 1 - slice) >> o.log_slices) + 1 : 0;
    for (int b = threadIdx.x; b < kSortWaves * kMaxBins; b += kSortThreads)
        (&hist[0][0])[b] = 0;
    __syncthreads();

    // each wavefront owns a run of places, 64 at a time
    const int64_t run = (m + kSortThreads - 1) / kSortThreads * kWave;
    const int64_t j0 = w * run, j1 = j0 + run < m ? j0 + run : m;
    int less = 0;
    for (int64_t j = j0; j < j1; j += kWave) {
        const int64_t row = j + lane < j1 ? table_row(tok, i, j + lane) : -1;
        const int at = (int)(row & (slices - 1));
        less += __popcll(__ballot(row >= 0 && at < slice));
        if (row >= 0 && at == slice) atomicAdd(&hist[w][row >> o.log_slices], 1);
    }
    if (lane == 0) wave_less[w] = less;
    __syncthreads();

    // counts to first places: over the bins, then over the wavefronts of a bin
    int total = 0;
    if (threadIdx.x < kMaxBins)
        for (int a = 0; a < kSortWaves; ++a) total += hist[a][threadIdx.x];
    int upto = total;  // inclusive sum inside the wavefront's bins
    for (int d = 1; d < kWave; d *= 2) {
        const int x = __shfl_up(upto, d);
        if (lane >= d) upto += x;
    }
    if (threadIdx.x < kMaxBins && lane == kWave - 1) wave_sum[w] = upto;
    __syncthreads();
    int base = 0;
    for (int a = 0; a < kSortWaves; ++a) base += wave_less[a];
    int own = 0;
    for (int a = 0; a < kMaxBins / kWave; ++a) own += wave_sum[a];
    if (threadIdx.x < kMaxBins) {
        for (int a = 0; a < w; ++a) base += wave_sum[a];
        base += upto - total;
        if ((int)threadIdx.x < bins)
            o.count[(int64_t)i * tok.v + ((int64_t)threadIdx.x << o.log_slices) + slice] = total;
        int next = base;
        for (int a = 0; a < kSortWaves; ++a) {
            const int x = hist[a][threadIdx.x];
            hist[a][threadIdx.x] = next;
            next += x;
        }
        if (slice == slices - 1 && threadIdx.x == kMaxBins - 1) o.held[i] = next;
    }
    __syncthreads();
    if (own == 0) return;

    for (int64_t j = j0; j < j1; j += kWave) {
        const int64_t row = j + lane < j1 ? table_row(tok, i, j + lane) : -1;
        const bool mine = row >= 0 && (int)(row & (slices - 1)) == slice;
        const int bin = mine ? (int)(row >> o.log_slices) : -1;
        uint64_t left = __ballot(mine);
        while (left) {  // a turn for each different row among the 64 tokens
            const int lead = __ffsll((unsigned long long)left) - 1;
            const int b = __builtin_amdgcn_readlane(bin, lead);
            const uint64_t peers = __ballot(bin == b);
            const int first = hist[w][b];
            if (bin == b) {
                const int at = first + __popcll(peers & ((1ull << lane) - 1));
                o.row[i * t + at] = (int32_t)row;
                o.place[i * t + at] = (int32_t)(j + lane);
            }
            // the wavefront's own counts: no other touches them, and its LDS
            // accesses complete in order, so the compiler's order is all that
            // has to be fixed
            if (lane == lead) hist[w][b] = first + __popcll(peers);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            left &= ~peers;
        }
    }
}

// One wavefront of step 2.  U columns a lane; rows and places of the chunk lie
// one to a lane.
template <class Y, class G>
__device__ __forceinline__ void sum_chunk(const EmbedGradParams& p, const GradPlan& g, int i,
                                          int64_t chunk, int64_t strip, int lane) {
    typedef typename Y::T YT;
    typedef typename G::T GT;
    constexpr int U = 16 / (int)sizeof(YT);
    constexpr int kAhead = 8;  // tokens whose loads are in flight
    const int held = g.s.held[i];
    const int64_t k0 = chunk * g.chunk;
    if (k0 >= held) return;
    const int len = (int)(held - k0 < g.chunk ? held - k0 : g.chunk);
    const int32_t* rows = g.s.row + i * p.t;
    const int my_row = lane < len ? rows[k0 + lane] : -1;
    const int my_place = lane < len ? g.s.place[i * p.t + k0 + lane] : 0;
    const int before = k0 > 0 ? rows[k0 - 1] : -1;
    const int after = k0 + len < held ? rows[k0 + len] : -1;
    const int64_t c0 = (strip * kWave + lane) * U;
    const int64_t have = p.h - c0;
    const YT* dy = static_cast<const YT*>(p.dy.p) + i * p.t * p.dy.ld + c0;
    GT* grads = static_cast<GT*>(p.grads.p) + i * p.grads.ld + p.grads.offset + c0;
    float* part = g.part + (i * g.chunks + chunk) * 2 * p.h + c0;

    float sum[U] = {};
    int cur = __builtin_amdgcn_readlane(my_row, 0);
    bool open = cur == before;  // the row began in an earlier chunk
    for (int k = 0; k < len; k += kAhead) {
        float y[kAhead][U];
#pragma unroll
        for (int a = 0; a < kAhead; ++a)
            if (k + a < len && have > 0)
                load_unit<YT, U, true>(
                    dy + (int64_t)__builtin_amdgcn_readlane(my_place, k + a) * p.dy.ld, have,
                    y[a]);
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            if (k + a >= len) break;
#pragma unroll
            for (int c = 0; c < U; ++c) sum[c] += y[a][c];
            const int next = k + a + 1 < len ? __builtin_amdgcn_readlane(my_row, k + a + 1) : after;
            if (next == cur && k + a + 1 < len) continue;
            if (have > 0) {
                if (open || next == cur) {  // crosses into this chunk, or out of it
                    store_unit<float, U, false>(part + (open ? 0 : p.h), have, sum);
                } else {
                    GT* d = grads + (int64_t)cur * p.h;
                    float out[U];
                    if (p.accumulate) load_unit<GT, U, false>(d, have, out);
#pragma unroll
                    for (int c = 0; c < U; ++c)
                        out[c] = p.accumulate ? __builtin_fmaf(p.scale, sum[c], out[c])
                                              : p.scale * sum[c];
                    store_unit<GT, U, true>(d, have, out);
                }
            }
#pragma unroll
            for (int c = 0; c < U; ++c) sum[c] = 0.0f;
            cur = next;
            open = false;
        }
    }
}

template <class G>
__device__ __forceinline__ void zero_rows(const EmbedGradParams& p, const GradPlan& g, int64_t w,
                                          int lane) {
    typedef typename G::T GT;
    constexpr int U = 16 / (int)sizeof(GT);
    const int64_t v = p.tok.v, groups = (v + kZeroRows - 1) / kZeroRows;
    const int i = (int)(w / groups);
    const int64_t r0 = (w - i * groups) * kZeroRows;
    const int64_t r1 = r0 + kZeroRows < v ? r0 + kZeroRows : v;
    GT* grads = static_cast<GT*>(p.grads.p) + i * p.grads.ld + p.grads.offset;
    const float zero[U] = {};
    for (int64_t r = r0; r < r1; ++r) {
        if (g.s.count[i * v + r]) continue;
        for (int64_t c = lane * U; c < p.h; c += kWave * U)
            store_unit<GT, U, true>(grads + r * p.h + c, p.h - c, zero);
    }
}

template <class Y, class G>
__global__ __launch_bounds__(kBlock) void k_embed_grad(EmbedGradParams p, GradPlan g) {
    const int64_t w = (int64_t)blockIdx.x * (kBlock / kWave) + threadIdx.x / kWave;
    const int lane = threadIdx.x % kWave;
    if (w < g.chunk_waves) {
        const int64_t per = g.chunks * g.strips;
        const int i = (int)(w / per);
        const int64_t c = (w - i * per) / g.strips;
        sum_chunk<Y, G>(p, g, i, c, w - i * per - c * g.strips, lane);
    } else if (w - g.chunk_waves < g.zero_waves) {
        zero_rows<G>(p, g, w - g.chunk_waves, lane);
    }
}

// Step 3: the wavefront of the chunk in which a crossing row begins adds the
// row's partial sums up.
template <class G>
__global__ __launch_bounds__(kBlock) void k_embed_grad_join(EmbedGradParams p, GradPlan g) {
    typedef typename G::T GT;
    constexpr int U = 4;
    const int64_t strips = (p.h + kWave * U - 1) / (kWave * U);
    const int64_t w = (int64_t)blockIdx.x * (kBlock / kWave) + threadIdx.x / kWave;
    const int64_t per = g.chunks * strips;
    if (w >= p.n * per) return;
    const int i = (int)(w / per);
    const int64_t chunk = (w - i * per) / strips, strip = w - i * per - chunk * strips;
    const int64_t c0 = (strip * kWave + threadIdx.x % kWave) * U;
    const int64_t have = p.h - c0;
    const int held = g.s.held[i];
    const int32_t* rows = g.s.row + i * p.t;
    const int64_t k0 = chunk * g.chunk, k1 = k0 + g.chunk;
    if (k1 >= held || have <= 0) return;
    const int row = rows[k1 - 1];
    if (rows[k1] != row) return;                  // does not cross
    if (k0 > 0 && rows[k0 - 1] == row) return;  // began earlier
    const float* part = g.part + (i * g.chunks + chunk) * 2 * p.h + c0;
    float sum[U];
    load_unit<float, U, false>(part + p.h, have, sum);
    int64_t c = chunk + 1;
    for (;; ++c) {
        float x[U];
        load_unit<float, U, false>(part + (c - chunk) * 2 * p.h, have, x);
#pragma unroll
        for (int a = 0; a < U; ++a) sum[a] += x[a];
        const int64_t end = (c + 1) * g.chunk;
        if (end >= held || rows[end] != row) break;
    }
    GT* d = static_cast<GT*>(p.grads.p) + i * p.grads.ld + p.grads.offset + (int64_t)row * p.h + c0;
    float out[U];
    if (p.accumulate) load_unit<GT, U, false>(d, have, out);
#pragma unroll
    for (int a = 0; a < U; ++a)
        out[a] = p.accumulate ? __builtin_fmaf(p.scale, sum[a], out[a]) : p.scale * sum[a];
    store_unit<GT, U, true>(d, have, out);
}

size_t round16(size_t x) { return (x + 15) & ~(size_t)15; }

// Sorted tokens of a wavefront: 64, fewer where that leaves fewer than 2048
// wavefronts over tokens and columns.
int chunk_of(int64_t n, int64_t t, int64_t h) {
    int c = kWave;
    while (c > 8 && n * ((t + c - 1) / c) * ((h + 511) / 512) < 2048) c /= 2;
    return c;
}

// Plan and workspace of a call; returns the bytes.
size_t grad_plan(int64_t n, int64_t t, int64_t h, int64_t v, uint8_t* ws, GradPlan* g) {
    g->s.log_slices = 0;
    while ((1ll << g->s.log_slices) < kMinSlices ||
           (v - 1) >> g->s.log_slices >= kMaxBins)
        ++g->s.log_slices;
    g->chunk = chunk_of(n, t, h);
    g->chunks = (t + g->chunk - 1) / g->chunk;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        uint8_t* p = ws + at;
        at += round16(bytes);
        return p;
    };
    g->s.row = reinterpret_cast<int32_t*>(take((size_t)n * t * 4));
    g->s.place = reinterpret_cast<int32_t*>(take((size_t)n * t * 4));
    g->s.count = reinterpret_cast<int32_t*>(take((size_t)n * v * 4));
    g->s.held = reinterpret_cast<int32_t*>(take((size_t)n * 4));
    g->part = reinterpret_cast<float*>(take((size_t)n * g->chunks * 2 * h * 4));
    return at;
}

}  // namespace

hipError_t launch_embed(const EmbedParams& p, hipStream_t s) {
    const int64_t rows = (int64_t)p.n * p.t;
    const int u = p.table.bf16 || p.out.bf16 ? 8 : 4;
    const int lanes = lanes_per_row((p.h + u - 1) / u);
    const dim3 grid(grid_for((rows * lanes + kBlock - 1) / kBlock));
    LOSSY_LAUNCH2(k_embed, p.table.bf16, p.out.bf16, grid, dim3(kBlock), s, p, lanes);
    return hipGetLastError();
}

size_t embed_grad_workspace(int64_t n, int64_t t, int64_t h, int64_t v) {
    GradPlan g;
    return grad_plan(n, t, h, v, nullptr, &g);
}

hipError_t launch_embed_grad(const EmbedGradParams& p, void* ws, hipStream_t s) {
    GradPlan g;
    grad_plan(p.n, p.t, p.h, p.tok.v, static_cast<uint8_t*>(ws), &g);
    const int u = p.dy.bf16 ? 8 : 4;
    g.strips = (p.h + kWave * u - 1) / (kWave * u);
    g.chunk_waves = p.n * g.chunks * g.strips;
    g.zero_waves = p.accumulate ? 0 : p.n * ((p.tok.v + kZeroRows - 1) / kZeroRows);
    const int64_t sorts = (int64_t)p.n << g.s.log_slices;
    const int64_t blocks = (g.chunk_waves + g.zero_waves + 3) / 4;
    const int64_t joins = (p.n * g.chunks * ((p.h + 255) / 256) + 3) / 4;
    // threads of a launch fit 32 bits
    if (sorts > 0xFFFFFFFFll / kSortThreads || blocks > 0xFFFFFFFFll / kBlock ||
        joins > 0xFFFFFFFFll / kBlock)
        return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL(k_token_sort, dim3((unsigned)sorts), dim3(kSortThreads), 0, s, p.t,
                       p.lengths, p.tok, g.s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || blocks == 0) return e;
    LOSSY_LAUNCH2(k_embed_grad, p.dy.bf16, p.grads.bf16, dim3((unsigned)blocks), dim3(kBlock), s,
                  p, g);
    e = hipGetLastError();
    if (e != hipSuccess || g.chunks < 2) return e;
    if (p.grads.bf16)
        hipLaunchKernelGGL((k_embed_grad_join<El16>), dim3((unsigned)joins), dim3(kBlock), 0, s, p, g);
    else
        hipLaunchKernelGGL((k_embed_grad_join<El32>), dim3((unsigned)joins), dim3(kBlock), 0, s, p, g);
    return hipGetLastError();
}

}  // namespace lossy
