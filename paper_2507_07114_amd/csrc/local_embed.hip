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
// 144 a call among others (147 when the following were timed, 153 under a trace); 64
// lanes 155; 256 lanes 150; four units of a lane in flight 154; rows dealt out
// flat, as in local_act.hip, 163; written through the caches 180.
// The distinct rows and the output are 752 MB (5.3 TB/s of them); each die's L2
// fetches rows for itself, 339 MB instead of 215.
// A unit is 16 bytes of the output, one store: 4 x 8192 x 4096 from bf16 to fp32
// rows take 103, with units of 16 bytes of the table 216.

template <class R, class O, bool NARROW>
__device__ __forceinline__ void embed_rows(const EmbedParams& p, int lanes) {
    typedef typename R::T RT;
    typedef typename O::T OT;
    constexpr int U = 16 / (int)sizeof(OT);
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
            const Columns<U> cols{u * U, p.h};
            float v[U] = {};
            if (row >= 0) {
                widen(cols.template load<RT, false, NARROW>(src), v);
#pragma unroll
                for (int c = 0; c < U; ++c) v[c] *= p.scale;
            }
            // two lanes give the columns that both hold the same values
            if (NARROW) cols.template store<OT, true>(dst, v);
            else store_whole<OT, U, true>(dst + cols.at(), v);
        }
    }
}

template <class R, class O>
__global__ __launch_bounds__(kBlock) void k_embed(EmbedParams p, int lanes) {
    if (p.h < 16 / (int)sizeof(typename O::T)) embed_rows<R, O, true>(p, lanes);
    else embed_rows<R, O, false>(p, lanes);
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
//    workgroups of the launch store zeros in the rows that have no token.
// 3. k_embed_grad_join adds the partial sums of rows that cross chunks, in
//    order.
// Bound by HBM where the table is large: 8 workers' 8192 tokens, 25,695 x 4096
// bf16, take 12 + 369 to 416 + 10 us, the main launch at 5.4 to 6.0 TB/s (mostly
// zeros; 394 a call in a long run of them).

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / kWave;
constexpr int kMaxBins = 512;  // table rows a slice can hold: 32 KiB of counts
// 64 slices, more where that leaves compute units without one: the whole
// gradient of 65536 tokens of 32000 x 512, one worker, 71 us with 64, 65 with 256; 32166
// of 295 x 2624 fp32 89.4, 87.5; 1024 of 1867 x 1280 15.4, 15.6.
constexpr int kMinSlices = 64, kFillSlices = 256;

struct Sorted {
    int32_t* row;    // [n][t] table rows, grouped
    int32_t* place;  // [n][t] token places, ascending inside a row
    int32_t* count;  // [n][slices][bins] tokens of each table row, slice by slice
    int32_t* held;   // [n] sorted tokens of a worker
    int log_slices;
    int64_t bins;  // most rows of a slice

    // Where row r of worker i is counted.  Slices lie apart: their workgroups
    // run on several dies, whose caches would share every line of counts in
    // the order of the rows.
    __device__ __forceinline__ int64_t at(int i, int64_t r) const {
        const int64_t slice = r & ((1 << log_slices) - 1);
        return ((((int64_t)i << log_slices) + slice) * bins) + (r >> log_slices);
    }
};

// Table rows dealt out to workgroups: kRowUnits units, of a few whole rows or a
// piece of a wide one.  16 workers' 4096 tokens, 32000 x 1024 fp32 rows, us: 512
// units 352 (6.3 TB/s), 256 510, 1024 416.
constexpr uint32_t kRowUnits = 512;

struct RowBlocks {
    int rows;               // table rows of a workgroup, at most 64
    int64_t groups, spans;  // groups of rows of a worker, workgroups of a group
    FlatRows units;         // units of a table row
};

struct GradPlan {
    Sorted s;
    float* part;    // [n][chunks][2][h] partial sums
    int chunk;      // sorted tokens of a wavefront
    int64_t chunks, strips, chunk_blocks;
    RowBlocks rows;
};

__global__ __launch_bounds__(kSortThreads) void k_token_sort(int64_t t, const int32_t* lengths,
                                                            TokenView tok, Sorted o) {
    __shared__ int hist[kSortWaves][kMaxBins];
    __shared__ int wave_less[kSortWaves], wave_sum[kMaxBins / kWave];
    const int slices = 1 << o.log_slices;
    const int i = (int)(blockIdx.x >> o.log_slices);
    const uint32_t slice = blockIdx.x & (slices - 1);
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int64_t m = batch_len(lengths, i, t);
    // rows slice, slice + slices, ... below v
    const int bins = slice < tok.v ? (int)((tok.v - 1 - (int64_t)slice) >> o.log_slices) + 1 : 0;
    for (int b = threadIdx.x; b < kSortWaves * kMaxBins; b += kSortThreads)
        (&hist[0][0])[b] = 0;
    __syncthreads();

    // each wavefront owns a run of places; kAhead tokens of a lane are loaded
    // together (and again in the second pass: the cache has them)
    constexpr int kAhead = 8;
    const int64_t run = (m + kSortThreads - 1) / kSortThreads * kWave;
    const int64_t j0 = w * run, j1 = j0 + run < m ? j0 + run : m;
    uint32_t row[kAhead];
    auto load = [&](int64_t j) {  // all loads before the first use
        int64_t id[kAhead];
        const int64_t first = (int64_t)i * tok.ld, last = j1 - 1;
        if (tok.wide) {
            const int64_t* ids = static_cast<const int64_t*>(tok.ids) + first;
#pragma unroll
            for (int a = 0; a < kAhead; ++a) {
                const int64_t at = j + a * kWave + lane;
                id[a] = ids[at < last ? at : last];
            }
        } else {
            const int32_t* ids = static_cast<const int32_t*>(tok.ids) + first;
#pragma unroll
            for (int a = 0; a < kAhead; ++a) {
                const int64_t at = j + a * kWave + lane;
                id[a] = ids[at < last ? at : last];
            }
        }
#pragma unroll
        for (int a = 0; a < kAhead; ++a)
            row[a] = j + a * kWave + lane < j1 ? (uint32_t)table_row(tok, id[a]) : ~0u;
    };
    // the slice of a row that is held; more than any where it is not
    const uint32_t low = (slices - 1) | 0x80000000u;
    int less = 0;
    for (int64_t j = j0; j < j1; j += kAhead * kWave) {
        load(j);
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            less += __popcll(__ballot((row[a] & low) < slice));
            if ((row[a] & low) == slice) atomicAdd(&hist[w][row[a] >> o.log_slices], 1);
        }
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
            o.count[o.at(i, slice) + threadIdx.x] = total;
        int next = base;
        for (int a = 0; a < kSortWaves; ++a) {
            const int x = hist[a][threadIdx.x];
            hist[a][threadIdx.x] = next;
            next += x;
        }
        if ((int)slice == slices - 1 && threadIdx.x == kMaxBins - 1) o.held[i] = next;
    }
    __syncthreads();
    if (own == 0) return;

    for (int64_t j = j0; j < j1; j += kAhead * kWave) {
        if (run > kAhead * kWave) load(j);  // else the registers still hold them
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            const bool mine = (row[a] & low) == slice;
            const int bin = mine ? (int)(row[a] >> o.log_slices) : -1;
            uint64_t left = __ballot(mine);
            while (left) {  // a turn for each different row among the 64 tokens
                const int lead = __ffsll((unsigned long long)left) - 1;
                const int b = __builtin_amdgcn_readlane(bin, lead);
                const uint64_t peers = __ballot(bin == b);
                const int first = hist[w][b];
                if (bin == b) {
                    const int at = first + __popcll(peers & ((1ull << lane) - 1));
                    o.row[i * t + at] = (int32_t)row[a];
                    o.place[i * t + at] = (int32_t)(j + a * kWave + lane);
                }
                // the wavefront's own counts: no other touches them, and its
                // LDS accesses complete in order, so the compiler's order is
                // all that has to be fixed
                if (lane == lead) hist[w][b] = first + __popcll(peers);
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                left &= ~peers;
            }
        }
    }
}

// Up to so many tokens a worker the gradient takes one launch, one token to a
// thread: workgroups of 256 threads, or 512 where there are more tokens.  us
// against the three launches: 8 workers' 256 tokens of 25,695 x 4096 bf16 250 /
// 299 (263 by 512 threads), 4 workers' 256 of 50 x 512 10 / 16; 8 workers' 512 of
// 25,695 x 4096 281 / 304, one worker's 512 of 32000 x 4096 48 / 56, 500 of 261 x
// 184 9 / 15, 4 workers' 512 of 50 x 512 16.4 / 17.4.  1024 tokens by 1024 threads:
// 4 workers' of 50 x 512 30 / 17, 8 workers' of 25,695 x 4096 324 / 312, one
// worker's of 1867 x 1280 11 / 17.
constexpr int kFewTokens = 512;

// One wavefront of step 2.  U columns a lane; rows and places of the chunk lie
// one to a lane.
template <class Y, class G, bool NARROW>
__device__ __forceinline__ void sum_chunk(const EmbedGradParams& p, const GradPlan& g, int i,
                                          int64_t chunk, int64_t strip, int lane) {
    typedef typename Y::T YT;
    typedef typename G::T GT;
    constexpr int U = 16 / (int)sizeof(YT);
    constexpr int kAhead = 8;  // tokens whose loads are in flight
    // all of these loads at once; what lies behind the held tokens is not used
    const int32_t* rows = g.s.row + i * p.t;
    const int64_t k0 = chunk * g.chunk, k1 = k0 + g.chunk, last = p.t - 1;
    const int64_t mine = k0 + lane < last ? k0 + lane : last;
    const int held = g.s.held[i];
    int my_row = rows[mine];
    const int my_place = g.s.place[i * p.t + mine];
    int before = rows[k0 > 0 ? k0 - 1 : 0], after = rows[k1 < last ? k1 : last];
    if (k0 >= held) return;
    const int len = (int)(held - k0 < g.chunk ? held - k0 : g.chunk);
    before = k0 > 0 ? before : -1;
    after = k1 < held ? after : -1;
    const Columns<U> cols{(strip * kWave + lane) * U, p.h};
    const YT* dy = static_cast<const YT*>(p.dy.p) + i * p.t * p.dy.ld;
    GT* grads = static_cast<GT*>(p.grads.p) + i * p.grads.ld + p.grads.offset;
    float* part = g.part + (i * g.chunks + chunk) * 2 * p.h;

    float sum[U] = {};
    int cur = __builtin_amdgcn_readlane(my_row, 0);
    bool open = cur == before;  // the row began in an earlier chunk
    for (int k = 0; k < len; k += kAhead) {
        Packed<YT, U> y[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {  // past the end the last one again
            const int at = k + a < len ? k + a : len - 1;
            y[a] = cols.template load<YT, true, NARROW>(
                dy + (int64_t)__builtin_amdgcn_readlane(my_place, at) * p.dy.ld);
        }
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            if (k + a >= len) break;
            float x[U];
            widen(y[a], x);
#pragma unroll
            for (int c = 0; c < U; ++c) sum[c] += x[c];
            const int next = k + a + 1 < len ? __builtin_amdgcn_readlane(my_row, k + a + 1) : after;
            if (next == cur && k + a + 1 < len) continue;
            if (open || next == cur) {  // crosses into this chunk, or out of it
                cols.template store<float, false>(part + (open ? 0 : p.h), sum);
            } else {
                GT* d = grads + (int64_t)cur * p.h;
                float out[U];
                if (p.accumulate) widen(cols.template load<GT, false, NARROW>(d), out);
#pragma unroll
                for (int c = 0; c < U; ++c)
                    out[c] = p.accumulate ? __builtin_fmaf(p.scale, sum[c], out[c])
                                          : p.scale * sum[c];
                // two accesses to a unit (bf16 dy, fp32 grads) meet in the cache
                cols.template store<GT, U * sizeof(GT) <= 16>(d, out);
            }
#pragma unroll
            for (int c = 0; c < U; ++c) sum[c] = 0.0f;
            cur = next;
            open = false;
        }
    }
}

// Zeros for a workgroup's table rows that no token names.  Every lane has its
// units' counts first, so that nothing stands between the stores.
template <class Y, class G>
__device__ __forceinline__ void zero_rows(const EmbedGradParams& p, const GradPlan& g, int64_t b) {
    typedef typename G::T GT;
    constexpr int U = 16 / (int)sizeof(GT), kTurns = kRowUnits / kBlock;
    const int64_t span = b % g.rows.spans, group = b / g.rows.spans;
    const int i = (int)(group / g.rows.groups);
    const int64_t r0 = (group - i * g.rows.groups) * g.rows.rows;
    const int rows = (int)(p.tok.v - r0 < g.rows.rows ? p.tok.v - r0 : g.rows.rows);
    const uint32_t all = rows * g.rows.units.units;
    const uint32_t u0 = (uint32_t)span * kRowUnits + threadIdx.x;
    int count[kTurns];
#pragma unroll
    for (int a = 0; a < kTurns; ++a) {
        const uint32_t u = u0 + a * kBlock;
        count[a] = g.s.count[g.s.at(i, r0 + flat_row(g.rows.units, u < all ? u : all - 1))];
    }
    GT* grads = static_cast<GT*>(p.grads.p) + i * p.grads.ld + p.grads.offset + r0 * p.h;
    const float zero[U] = {};
#pragma unroll
    for (int a = 0; a < kTurns; ++a) {
        const uint32_t u = u0 + a * kBlock;
        if (count[a] || u >= all) continue;
        const uint32_t r = flat_row(g.rows.units, u);
        const Columns<U> cols{(int64_t)(u - r * g.rows.units.units) * U, p.h};
        if (p.h < U) cols.template store<GT, true>(grads + r * p.h, zero);
        else store_whole<GT, U, true>(grads + r * p.h + cols.at(), zero);
    }
}

// 5 wavefronts to a SIMD, of 8 tokens in flight: 16 workers' 4096 tokens, 32000 x
// 1024, bf16 into fp32, 352 us (6: 377, 4 of 8 tokens 372, 8 of 4 tokens 399);
// the zeros go fastest with few writers.
template <class Y, class G>
__global__ __launch_bounds__(kBlock, 5) void k_embed_grad(EmbedGradParams p, GradPlan g) {
    if (blockIdx.x >= g.chunk_blocks) {
        zero_rows<Y, G>(p, g, blockIdx.x - g.chunk_blocks);
        return;
    }
    const int64_t w = (int64_t)blockIdx.x * (kBlock / kWave) + threadIdx.x / kWave;
    const int64_t per = g.chunks * g.strips;
    if (w >= p.n * per) return;
    const int i = (int)(w / per);
    const int64_t c = (w - i * per) / g.strips;
    if (p.h < 16 / (int)sizeof(typename Y::T))
        sum_chunk<Y, G, true>(p, g, i, c, w - i * per - c * g.strips, threadIdx.x % kWave);
    else
        sum_chunk<Y, G, false>(p, g, i, c, w - i * per - c * g.strips, threadIdx.x % kWave);
}

// Step 3: the wavefront of the chunk in which a crossing row begins adds the
// row's partial sums up.
template <class G, bool NARROW>
__device__ __forceinline__ void join_rows(const EmbedGradParams& p, const GradPlan& g) {
    typedef typename G::T GT;
    constexpr int U = 4;
    const int64_t strips = (p.h + kWave * U - 1) / (kWave * U);
    const int64_t w = (int64_t)blockIdx.x * (kBlock / kWave) + threadIdx.x / kWave;
    const int64_t per = g.chunks * strips;
    if (w >= p.n * per) return;
    const int i = (int)(w / per);
    const int64_t chunk = (w - i * per) / strips, strip = w - i * per - chunk * strips;
    const int lane = threadIdx.x % kWave;
    const Columns<U> cols{(strip * kWave + lane) * U, p.h};
    const int32_t* rows = g.s.row + i * p.t;
    const int64_t k0 = chunk * g.chunk, k1 = k0 + g.chunk, last = p.t - 1;
    const int held = g.s.held[i];
    const int mine = rows[k0 + lane < last ? k0 + lane : last];
    const int before = rows[k0 > 0 ? k0 - 1 : 0], after = rows[k1 < last ? k1 : last];
    const int row = __builtin_amdgcn_readlane(mine, g.chunk - 1);
    if (k1 >= held || after != row) return;  // does not cross
    if (k0 > 0 && before == row) return;     // began earlier
    // the further chunks that hold the rest of its tokens
    const int here = __popcll(__ballot(lane < g.chunk && mine == row));
    const int more = (g.s.count[g.s.at(i, row)] - here + g.chunk - 1) / g.chunk;
    const float* part = g.part + (i * g.chunks + chunk) * 2 * p.h;
    float sum[U];
    widen(cols.template load<float, false, NARROW>(part + p.h), sum);
    constexpr int kAhead = 8;  // partial sums whose loads are in flight
    for (int a0 = 1; a0 <= more; a0 += kAhead) {
        Packed<float, U> x[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {  // past the end the last one again
            const int at = a0 + a <= more ? a0 + a : more;
            x[a] = cols.template load<float, false, NARROW>(part + (int64_t)at * 2 * p.h);
        }
#pragma unroll
        for (int a = 0; a < kAhead; ++a)
            if (a0 + a <= more)
#pragma unroll
                for (int k = 0; k < U; ++k) sum[k] += __uint_as_float(x[a].w[k]);
    }
    GT* d = static_cast<GT*>(p.grads.p) + i * p.grads.ld + p.grads.offset + (int64_t)row * p.h;
    float out[U];
    if (p.accumulate) widen(cols.template load<GT, false, NARROW>(d), out);
#pragma unroll
    for (int a = 0; a < U; ++a)
        out[a] = p.accumulate ? __builtin_fmaf(p.scale, sum[a], out[a]) : p.scale * sum[a];
    cols.template store<GT, true>(d, out);
}

template <class G>
__global__ __launch_bounds__(kBlock) void k_embed_grad_join(EmbedGradParams p, GradPlan g) {
    if (p.h < 4) join_rows<G, true>(p, g);
    else join_rows<G, false>(p, g);
}

// Few tokens: one launch.  A workgroup of BLOCK threads takes table rows of 2
// units a thread (or a piece of a wide row), looks all the worker's tokens
// through, groups the places of those of its rows by row, in order, and each
// lane adds up its unit's.  Accumulating, it takes the row of one token, unless
// an earlier token names it (4 workers' 256 tokens of 32000 x 4096: 14 us with
// fp32 rows, 88 by table rows).
constexpr int kFewUnits = 2;

template <class Y, class G, int BLOCK, bool NARROW>
__device__ __forceinline__ void few_rows(const EmbedGradParams& p, const RowBlocks& g) {
    typedef typename Y::T YT;
    typedef typename G::T GT;
    constexpr int U = 16 / (int)sizeof(GT);
    constexpr int kWaves = BLOCK / kWave;
    constexpr int kAhead = 4;  // tokens whose loads are in flight
    __shared__ uint16_t place[BLOCK];
    __shared__ int count[kWaves][kWave];  // a wavefront's tokens of each row
    __shared__ int start[kWave + 1];      // a row's tokens are place[start ...]
    __shared__ bool found[kWaves];
    const int64_t span = blockIdx.x % g.spans, group = blockIdx.x / g.spans;
    const int i = (int)(group / g.groups);
    const int m = (int)batch_len(p.lengths, i, p.t), j = threadIdx.x;
    const int place0 = (int)(group - i * g.groups);  // accumulating, the token's
    const int64_t r0 = !p.accumulate ? (group - i * g.groups) * g.rows
                       : place0 < m  ? table_row(p.tok, i, place0)
                                     : -1;
    if (r0 < 0) return;
    const int rows = (int)(p.tok.v - r0 < g.rows ? p.tok.v - r0 : g.rows);
    const int lane = threadIdx.x % kWave, w = threadIdx.x / kWave;

    // the tokens of these rows, by row and place
    const int64_t at_row = j < m ? table_row(p.tok, i, j) - r0 : -1;
    const bool mine = at_row >= 0 && at_row < rows;
    const int row = mine ? (int)at_row : 0;
    uint64_t peers = __ballot(mine);
    if (lane == 0) found[w] = peers != 0;
    count[w][lane] = 0;
    __syncthreads();
    bool any = false;
#pragma unroll
    for (int a = 0; a < kWaves; ++a) any |= found[a];
    if (any) {  // most workgroups of a large table have none
        // the wavefront's tokens of the same row
#pragma unroll
        for (int b = 1; b < kWave; b *= 2) {
            const uint64_t set = __ballot(row & b);
            peers &= row & b ? set : ~set;
        }
        const int before = __popcll(peers & ((1ull << lane) - 1));
        if (mine && before == 0) count[w][row] = __popcll(peers);
        __syncthreads();
        if (w == 0) {
            int upto = 0;
#pragma unroll
            for (int a = 0; a < kWaves; ++a) upto += count[a][lane];
#pragma unroll
            for (int d = 1; d < kWave; d *= 2) {
                const int x = __shfl_up(upto, d);
                if (lane >= d) upto += x;
            }
            if (lane == 0) start[0] = 0;
            start[lane + 1] = upto;
        }
        __syncthreads();
        if (mine) {
            int at = start[row] + before;
#pragma unroll
            for (int a = 0; a < kWaves; ++a)
                if (a < w) at += count[a][row];
            place[at] = (uint16_t)j;
        }
        __syncthreads();
    }
    if (p.accumulate && place[0] < place0) return;

    const YT* dy = static_cast<const YT*>(p.dy.p) + (int64_t)i * p.t * p.dy.ld;
    GT* grads = static_cast<GT*>(p.grads.p) + i * p.grads.ld + p.grads.offset + r0 * p.h;
    const uint32_t all = rows * g.units.units;
    const uint32_t u0 = (uint32_t)span * (BLOCK * kFewUnits);
    const uint32_t u1 = u0 + BLOCK * kFewUnits < all ? u0 + BLOCK * kFewUnits : all;
    if (!any) {
        const float zero[U] = {};
        for (uint32_t u = u0 + threadIdx.x; u < u1; u += BLOCK) {
            const uint32_t r = flat_row(g.units, u);
            const Columns<U> cols{(int64_t)(u - r * g.units.units) * U, p.h};
            if (NARROW) cols.template store<GT, true>(grads + r * p.h, zero);
            else store_whole<GT, U, true>(grads + r * p.h + cols.at(), zero);
        }
        return;
    }
    for (uint32_t u = u0 + threadIdx.x; u < u1; u += BLOCK) {
        const int r = (int)flat_row(g.units, u);
        const Columns<U> cols{(int64_t)(u - r * g.units.units) * U, p.h};
        float sum[U] = {};
        const int k0 = start[r], k1 = start[r + 1];
        for (int k = k0; k < k1; k += kAhead) {
            Packed<YT, U> y[kAhead];
#pragma unroll
            for (int a = 0; a < kAhead; ++a)  // past the end the last one again
                y[a] = cols.template load<YT, false, NARROW>(
                    dy + place[k + a < k1 ? k + a : k1 - 1] * p.dy.ld);
#pragma unroll
            for (int a = 0; a < kAhead; ++a) {
                float x[U];
                widen(y[a], x);
#pragma unroll
                for (int c = 0; c < U; ++c) sum[c] = k + a < k1 ? sum[c] + x[c] : sum[c];
            }
        }
        GT* d = grads + r * p.h;
        if (p.accumulate) {
            float old[U];
            widen(cols.template load<GT, false, NARROW>(d), old);
#pragma unroll
            for (int c = 0; c < U; ++c) sum[c] = __builtin_fmaf(p.scale, sum[c], old[c]);
        } else {
            // an empty row is 0, not -0
#pragma unroll
            for (int c = 0; c < U; ++c) sum[c] = k0 < k1 ? p.scale * sum[c] : 0.0f;
        }
        cols.template store<GT, true>(d, sum);
    }
}

template <class Y, class G>
__global__ __launch_bounds__(256) void k_embed_grad_few_256(EmbedGradParams p, RowBlocks g) {
    if (p.h < 16 / (int)sizeof(typename G::T)) few_rows<Y, G, 256, true>(p, g);
    else few_rows<Y, G, 256, false>(p, g);
}

template <class Y, class G>
__global__ __launch_bounds__(512) void k_embed_grad_few_512(EmbedGradParams p, RowBlocks g) {
    if (p.h < 16 / (int)sizeof(typename G::T)) few_rows<Y, G, 512, true>(p, g);
    else few_rows<Y, G, 512, false>(p, g);
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
    while ((1ll << g->s.log_slices) < kMinSlices || n << g->s.log_slices < kFillSlices ||
           (v - 1) >> g->s.log_slices >= kMaxBins)
        ++g->s.log_slices;
    g->s.bins = ((v - 1) >> g->s.log_slices) + 1;
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
    g->s.count = reinterpret_cast<int32_t*>(take(((size_t)n << g->s.log_slices) * g->s.bins * 4));
    g->s.held = reinterpret_cast<int32_t*>(take((size_t)n * 4));
    g->part = reinterpret_cast<float*>(take((size_t)n * g->chunks * 2 * h * 4));
    return at;
}

// `span` units to a workgroup, fewer rows where that leaves fewer workgroups
// than two to a compute unit; one row where few tokens are accumulated.
bool row_blocks(const EmbedGradParams& p, int64_t span, RowBlocks* g) {
    const int64_t row = p.grads.bf16 ? (p.h + 7) / 8 : (p.h + 3) / 4;
    const int64_t fit = span / row, few = p.n * p.tok.v / 512, rows = fit < few ? fit : few;
    g->rows = p.accumulate ? 1 : (int)(rows < 1 ? 1 : (rows > kWave ? kWave : rows));
    g->groups = p.accumulate ? p.t : (p.tok.v + g->rows - 1) / g->rows;
    g->spans = (g->rows * row + span - 1) / span;
    dim3 unused;
    return flat_rows(g->rows, row, 1, &g->units, &unused);
}

hipError_t launch_embed_grad_few(const EmbedGradParams& p, hipStream_t s) {
    const int threads = p.t <= 256 ? 256 : 512;
    RowBlocks g;
    if (!row_blocks(p, threads * kFewUnits, &g)) return hipErrorInvalidConfiguration;
    const int64_t blocks = p.n * g.groups * g.spans;
    if (blocks == 0) return hipSuccess;
    if (blocks > 0xFFFFFFFFll / threads) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)blocks);
    if (threads == 256) {
        // LDS that nothing uses: 6 workgroups to a compute unit.  4 workers' 256 tokens
        // of 32000 x 4096, us: bf16 155, fp32 319; with 8 workgroups 173, 336; with 5
        // 173, 340.
        LOSSY_LAUNCH2_LDS(k_embed_grad_few_256, p.dy.bf16, p.grads.bf16, grid, dim3(256), 24000,
                          s, p, g);
    } else {
        LOSSY_LAUNCH2(k_embed_grad_few_512, p.dy.bf16, p.grads.bf16, grid, dim3(512), s, p, g);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_embed(const EmbedParams& p, hipStream_t s) {
    const int64_t rows = (int64_t)p.n * p.t;
    const int u = p.out.bf16 ? 8 : 4;
    const int lanes = lanes_per_row((p.h + u - 1) / u);
    const dim3 grid(grid_for((rows * lanes + kBlock - 1) / kBlock));
    LOSSY_LAUNCH2(k_embed, p.table.bf16, p.out.bf16, grid, dim3(kBlock), s, p, lanes);
    return hipGetLastError();
}

size_t embed_grad_workspace(int64_t n, int64_t t, int64_t h, int64_t v) {
    if (t <= kFewTokens) return 0;
    GradPlan g;
    return grad_plan(n, t, h, v, nullptr, &g);
}

hipError_t launch_embed_grad(const EmbedGradParams& p, void* ws, hipStream_t s) {
    if (p.t <= kFewTokens) return launch_embed_grad_few(p, s);
    GradPlan g;
    grad_plan(p.n, p.t, p.h, p.tok.v, static_cast<uint8_t*>(ws), &g);
    const int u = p.dy.bf16 ? 8 : 4;
    g.strips = (p.h + kWave * u - 1) / (kWave * u);
    g.chunk_blocks = (p.n * g.chunks * g.strips + 3) / 4;
    int64_t blocks = g.chunk_blocks;
    if (!p.accumulate) {
        if (!row_blocks(p, kRowUnits, &g.rows)) return hipErrorInvalidConfiguration;
        blocks += p.n * g.rows.groups * g.rows.spans;
    }
    const int64_t sorts = (int64_t)p.n << g.s.log_slices;
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
