// Weight gradient of a linear layer from an 8-bit checkpoint of its input
// (include/lossy_local.h): ll_act_wgrad.
//
// D[o][h] = sum_t dy[t][o] x^[t][h] on the bf16 matrix units.  x^ = code * 2^k
// is exact in bf16 (4 significant bits), so bf16 dy needs one product per
// element; fp32 dy is a sum of three bf16 terms, three products over the same
// codes.  Both factors lie token by token, the matrix units want each lane's
// tokens side by side: LDS holds the tiles as they come and the transposing
// LDS read turns them.
//
// 4096 tokens, 4096 x 4096, bf16: 113 to 117 us, 1175 to 1216 TFLOP/s (152 us with 4
// wavefronts a tile, 137 with 8 that meet twice a step, 125 once in two steps, 114
// with reads, stores and loads dealt out between the products and rows stored
// whole).  2 x 8192 tokens, 11008 x 4096, in a long run of calls: 1200 to 1250 us,
// 1181 to 1230 TFLOP/s; up to 1670 us in the first ten calls after a pause.  The
// matrix units are busy in 65% of the cycles and LDS in 42%, at a clock that this
// load holds at 1.6 to 1.8 GHz.
#include <hip/hip_runtime.h>

#include "local.h"
#include "local_device.h"
#include "wgrad_plan.h"

namespace lossy {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) i16x4 LdsQuad;

// A tile row (one token, T columns of bf16) is T / 16 units of 32 bytes; unit u
// of row k lies at u ^ 2 (k % 4).  The transposing read of 16 lanes takes 32
// bytes from 4 consecutive rows; with the exchange these and the neighbouring
// 16 lanes' fall on different banks.
__device__ __forceinline__ int unit_at(int k, int unit) { return unit ^ (2 * (k & 3)); }

// Two fp32 values' bf16 term PART side by side: the leading 8 significant bits,
// the next 8 and the rest, each cut off, so that every difference is exact.  An
// infinite value has only the first; a NaN is one in the others.
template <int PART>
__device__ __forceinline__ uint32_t f32_terms(uint32_t lo, uint32_t hi) {
    auto rest = [](uint32_t u) {  // what the first PART terms leave
        float x = __uint_as_float(u);
        const float r = x - __uint_as_float(u & 0xFFFF0000u);
        x = __builtin_isinf(x) ? 0.0f : r;
        if (PART == 2) x -= __uint_as_float(__float_as_uint(x) & 0xFFFF0000u);
        return __float_as_uint(x);
    };
    if (PART > 0) {
        lo = rest(lo);
        hi = rest(hi);
    }
    return __builtin_amdgcn_perm(hi, lo, 0x07060302);  // the upper halves
}

// 8 columns of dy of one token, and one column.
template <class Y>
struct Chunk8;
template <>
struct Chunk8<El16> {
    u32x4 a;
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, uint32_t at) {
        a = __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, 0);
    }
    template <int PART>
    __device__ __forceinline__ u32x4 terms() const {
        return a;
    }
    static __device__ __forceinline__ uint32_t load1(__amdgpu_buffer_rsrc_t r, uint32_t at) {
        return __builtin_amdgcn_raw_buffer_load_b16(r, at, 0, 0);
    }
    template <int PART>
    static __device__ __forceinline__ uint32_t term1(uint32_t x) {
        return x;
    }
};
template <>
struct Chunk8<El32> {
    u32x4 a, b;
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, uint32_t at) {
        a = __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, 0);
        b = __builtin_amdgcn_raw_buffer_load_b128(r, at + 16, 0, 0);
    }
    template <int PART>
    __device__ __forceinline__ u32x4 terms() const {
        return u32x4{f32_terms<PART>(a.x, a.y), f32_terms<PART>(a.z, a.w),
                     f32_terms<PART>(b.x, b.y), f32_terms<PART>(b.z, b.w)};
    }
    static __device__ __forceinline__ uint32_t load1(__amdgpu_buffer_rsrc_t r, uint32_t at) {
        return __builtin_amdgcn_raw_buffer_load_b32(r, at, 0, 0);
    }
    template <int PART>
    static __device__ __forceinline__ uint32_t term1(uint32_t x) {
        return f32_terms<PART>(x, 0);
    }
};

// bf16 values of 8 codes under one scale.
__device__ __forceinline__ u32x4 restore8(u32x2 code, uint32_t s) {
    const float scale = __uint_as_float(s << 23);
    auto two = [&](uint32_t w, bool hi) {
        const bf16x2 v = hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, scale, true)
                            : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, scale, false);
        uint32_t r;
        __builtin_memcpy(&r, &v, 4);
        return r;
    };
    return u32x4{two(code.x, false), two(code.x, true), two(code.y, false), two(code.y, true)};
}

// Staging registers of one step of one thread: 8 columns of kPass token rows,
// and an element of the columns past the last whole 8.
template <class Y, int TO, int TH, int THREADS>
struct Staged {
    static constexpr int kPassY = kStepT * TO / 8 / THREADS;
    static constexpr int kPassX = kStepT * TH / 8 / THREADS;
    Chunk8<Y> y[kPassY];
    u32x2 x[kPassX];
    uint32_t s[kPassX];
    uint32_t ytail, xtail, stail;
};

// The next `rows` (0 to 32) token rows at p, `row` bytes each of which the first
// `width` are the tile's: loads past them give zeros and touch no memory.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t step_rows(const uint8_t* p, int rows, int row,
                                                            int width) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), (short)0,
                                             rows > 0 ? (rows - 1) * row + width : 0, kBufferRaw);
}
// An offset past every row, also with a row's offset added: 32 rows are below
// 2^31 bytes (checked at the entry point).
constexpr uint32_t kNowhere = 0x80000000u;

struct Tile {
    int i;           // worker
    int64_t o0, h0;  // corner
};

// Consecutive workgroups go to the 8 dies in turn; each die takes a contiguous
// run of tiles.
__device__ __forceinline__ int64_t spread(int64_t b, int64_t total) {
    const int64_t die = b % 8, each = total / 8, more = total % 8;
    return die * each + (die < more ? die : more) + b / 8;
}

// Tiles run through a worker's matrix in bands 4 tiles high, column by column:
// the 32 tiles that a die works on are 4 x 8, whose dy and codes its L2 holds.
template <int TO, int TH>
__device__ __forceinline__ Tile tile_at(const WgradPlan& g, int64_t lin) {
    const int64_t per = g.tiles_o * g.tiles_h;
    const int64_t i = lin / per, tile = lin - i * per;
    const int64_t band = tile / (4 * g.tiles_h), in = tile - band * 4 * g.tiles_h;
    const int64_t height = g.tiles_o - band * 4 < 4 ? g.tiles_o - band * 4 : 4;
    return Tile{(int)i, (band * 4 + in % height) * TO, in / height * TH};
}

// Row o, columns h .. h + U of a worker's gradient take U sums.
template <class G, int U>
__device__ __forceinline__ void put_sums(const WgradParams& p, int i, int64_t o, int64_t h,
                                         float (&v)[U]) {
    typedef typename G::T GT;
    GT* d = static_cast<GT*>(p.grads.p) + i * p.grads.ld + p.grads.offset + o * p.h + h;
    const int64_t have = p.h - h;
    float old[U];
    if (p.accumulate) load_unit<GT, U, false>(d, have, old);
#pragma unroll
    for (int k = 0; k < U; ++k)
        v[k] = p.accumulate ? __builtin_fmaf(p.scale, v[k], old[k]) : p.scale * v[k];
    store_unit<GT, U, true>(d, have, v);
}

// Bytes of LDS of an EDGE x EDGE tile: four steps of bf16 dy and codes, or two of
// the three terms of fp32 dy and the codes.
template <int EDGE>
constexpr int lds_bytes() {
    return 2 * 4 * kStepT * 2 * EDGE;
}

// LDS of a light workgroup: two steps of bf16 dy and codes take 32 KiB, the rows at
// the end a little more.  Four such workgroups fit a compute unit.
constexpr int kLightLds = 4 * 32 * 68 * 4;

// A workgroup of WO x WH wavefronts owns a TO x TH tile of D over a run of
// tokens.  TAILS: the tile's width or height is not a multiple of 8.  LIGHT: for few
// tokens, where a tile is over before loads dealt out between products pay.
template <class Y, class G, int TO, int TH, int WO, int WH, bool TAILS, bool LIGHT>
__device__ __forceinline__ void wgrad_tile(const WgradParams& p, const WgradPlan& g, Tile tile,
                                           int64_t ticket, int run, bool apart, uint8_t* lds) {
    typedef typename Y::T YT;
    constexpr int kThreads = WO * WH * kWave;
    constexpr int NI = TO / WO / 32, MI = TH / WH / 32;  // 32 x 32 products of a wavefront
    constexpr int kTerms = sizeof(YT) == 4 ? 3 : 1;
    constexpr int kRowY = TO * 2, kRowX = TH * 2;  // bytes of a tile row
    constexpr int kStageY = kStepT * kRowY, kStageX = kStepT * kRowX;
    constexpr int kAllY = kTerms * kStageY, kStage = kAllY + kStageX;
    // half of the LDS, a power of two: two stages of bf16 dy (LIGHT: one), one of
    // fp32 dy
    constexpr int kFlip = kTerms == 1 && !LIGHT ? 2 * kStage : kStage;
    constexpr int kLds = LIGHT ? kLightLds : lds_bytes<TO>();
    static_assert(TO == TH && 2 * kFlip <= kLds, "LDS");
    typedef Staged<Y, TO, TH, kThreads> Stage;
    const int i = tile.i;
    const int64_t o0 = tile.o0, h0 = tile.h0;
    const int64_t m = batch_len(p.lengths, i, p.t);
    const int64_t t0 = run * g.run_t;
    const int64_t t1 = apart && t0 + g.run_t < m ? t0 + g.run_t : m;
    const uint32_t left = t1 > t0 ? (uint32_t)(t1 - t0) : 0;  // tokens, below 2^31

    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    // staging: thread -> token row and 8 columns; the columns past the last
    // whole 8 of the tile's width go one to a thread
    const int ywidth = (int)(p.o - o0 < TO ? p.o - o0 : TO);
    const int xwidth = (int)(p.h - h0 < TH ? p.h - h0 : TH);
    const int yld = (int)p.dy.ld * (int)sizeof(YT), xld = (int)p.x.ld_q, sld = (int)p.x.ld_s;
    const uint8_t* ynext = reinterpret_cast<const uint8_t*>(
        static_cast<const YT*>(p.dy.p) + (i * p.t + t0) * p.dy.ld + o0);
    const uint8_t* xnext = p.x.q + (i * p.t + t0) * p.x.ld_q + h0;
    const uint8_t* snext = p.x.s + (i * p.t + t0) * p.x.ld_s + h0 / kActGroup;
    int rows_left = (int)left;  // from the next step's first token on
    const int yrow = tid / (TO / 8), ycol = tid % (TO / 8) * 8;
    const int xrow = tid / (TH / 8), xcol = tid % (TH / 8) * 8;
    const uint32_t yat = ycol + 8 <= ywidth ? yrow * (uint32_t)yld + ycol * (int)sizeof(YT) : kNowhere;
    const uint32_t xat = xcol + 8 <= xwidth ? xrow * (uint32_t)xld + xcol : kNowhere;
    const uint32_t sat = xcol + 8 <= xwidth ? xrow * (uint32_t)sld + xcol / kActGroup : kNowhere;
    const bool ysplit = TAILS && ywidth % 8 != 0, xsplit = TAILS && xwidth % 8 != 0;
    const int trow = tid / 8 % kStepT, ytcol = ywidth / 8 * 8 + tid % 8, xtcol = xwidth / 8 * 8 + tid % 8;
    const uint32_t ytat = ytcol < ywidth ? trow * (uint32_t)yld + ytcol * (int)sizeof(YT) : kNowhere;
    const uint32_t xtat = xtcol < xwidth ? trow * (uint32_t)xld + xtcol : kNowhere;
    const uint32_t stat = xtcol < xwidth ? trow * (uint32_t)sld + xtcol / kActGroup : kNowhere;
    const bool ywhole = !(ysplit && ycol == ywidth / 8 * 8);
    const bool xwhole = !(xsplit && xcol == xwidth / 8 * 8);

    // Loads of the next step's tiles, one piece a call (y rows, then x rows); past
    // the run's end they give zeros.
    __amdgpu_buffer_rsrc_t yr, xr, sr;
    auto open_stage = [&] {
        const int rows = rows_left < kStepT ? rows_left : kStepT;
        yr = step_rows(ynext, rows, yld, ywidth * (int)sizeof(YT));
        xr = step_rows(xnext, rows, xld, xwidth);
        sr = step_rows(snext, rows, sld, (xwidth + kActGroup - 1) / kActGroup);
        ynext += (int64_t)kStepT * yld;
        xnext += (int64_t)kStepT * xld;
        snext += (int64_t)kStepT * sld;
        rows_left -= kStepT;
    };
    constexpr int kPieces = Stage::kPassY + Stage::kPassX;
    auto load_piece = [&](Stage& r, int piece) {
        if (piece < Stage::kPassY) {
            r.y[piece].load(yr, yat + (uint32_t)(piece * (kStepT / Stage::kPassY)) * (uint32_t)yld);
        } else {
            const int a = piece - Stage::kPassY;
            const uint32_t row = a * (kStepT / Stage::kPassX);
            r.x[a] = __builtin_amdgcn_raw_buffer_load_b64(xr, xat + row * (uint32_t)xld, 0, 0);
            r.s[a] = __builtin_amdgcn_raw_buffer_load_b8(sr, sat + row * (uint32_t)sld, 0, 0);
        }
        if (piece == kPieces - 1) {
            if (ysplit) r.ytail = Chunk8<Y>::load1(yr, ytat);
            if (xsplit) {
                r.xtail = __builtin_amdgcn_raw_buffer_load_b8(xr, xtat, 0, 0);
                r.stail = __builtin_amdgcn_raw_buffer_load_b8(sr, stat, 0, 0);
            }
        }
    };
    auto load_stage = [&](Stage& r) {
        open_stage();
#pragma unroll
        for (int a = 0; a < kPieces; ++a) load_piece(r, a);
    };
    // LDS places of what a thread stages, in one half of the LDS; the other's
    // differ in one bit
    auto place = [](int k, int col, int row_bytes) {
        return k * row_bytes + unit_at(k, col / 16) * 32 + col % 16 * 2;
    };
    int yput[Stage::kPassY], xput[Stage::kPassX];
#pragma unroll
    for (int a = 0; a < Stage::kPassY; ++a)
        yput[a] = place(yrow + a * (kStepT / Stage::kPassY), ycol, kRowY);
#pragma unroll
    for (int a = 0; a < Stage::kPassX; ++a)
        xput[a] = kAllY + place(xrow + a * (kStepT / Stage::kPassX), xcol, kRowX);
    const int ytput = place(trow, ytcol, kRowY), xtput = kAllY + place(trow, xtcol, kRowX);
    // store a piece into the half that `flip` says (0 or kFlip), stage `stage` of it
    auto store_piece = [&](const Stage& r, int flip, int stage, int piece) {
        uint8_t* to = lds + stage * kStage;
        if (piece < Stage::kPassY) {
            if (!TAILS || ywhole) {
                u32x4* y = reinterpret_cast<u32x4*>(to + (yput[piece] ^ flip));
                y[0] = r.y[piece].template terms<0>();
                if (kTerms == 3) {
                    y[kStageY / 16] = r.y[piece].template terms<1>();
                    y[2 * kStageY / 16] = r.y[piece].template terms<2>();
                }
            }
        } else {
            const int a = piece - Stage::kPassY;
            if (!TAILS || xwhole)
                *reinterpret_cast<u32x4*>(to + (xput[a] ^ flip)) = restore8(r.x[a], r.s[a]);
        }
        if (piece == kPieces - 1) {
            if (ysplit) {
                uint16_t* y = reinterpret_cast<uint16_t*>(to + (ytput ^ flip));
                y[0] = (uint16_t)Chunk8<Y>::template term1<0>(r.ytail);
                if (kTerms == 3) {
                    y[kStageY / 2] = (uint16_t)Chunk8<Y>::template term1<1>(r.ytail);
                    y[2 * kStageY / 2] = (uint16_t)Chunk8<Y>::template term1<2>(r.ytail);
                }
            }
            if (xsplit)
                *reinterpret_cast<uint16_t*>(to + (xtput ^ flip)) =
                    (uint16_t)restore8(u32x2{r.xtail, 0}, r.stail).x;
        }
    };
    auto store_stage = [&](const Stage& r, int flip, int stage) {
#pragma unroll
        for (int a = 0; a < kPieces; ++a) store_piece(r, flip, stage, a);
    };
    auto barrier = [] {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
    };

    // fragments: lane -> column l % 32 of a 32-column block, 8 tokens.  16
    // lanes read 4 token rows x 16 columns, 8 bytes each, and get a column each.
    const int wo = wave / WH * (TO / WO), wh = wave % WH * (TH / WH);
    const int frow = (lane / 32) * 8 + lane % 16 / 4;  // and + 4 for the second read
    int yaddr[NI], xaddr[MI];
#pragma unroll
    for (int a = 0; a < NI; ++a)
        yaddr[a] = frow * kRowY + unit_at(frow, (wo + a * 32) / 16 + lane / 16 % 2) * 32 +
                   lane % 4 * 8;
#pragma unroll
    for (int a = 0; a < MI; ++a)
        xaddr[a] = kAllY + frow * kRowX +
                   unit_at(frow, (wh + a * 32) / 16 + lane / 16 % 2) * 32 + lane % 4 * 8;
    auto fragment = [&](int at, int row_bytes) {
        uint8_t* q = lds + at;
        const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsQuad*)q);
        const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsQuad*)(q + 4 * row_bytes));
        bf16x8 f;
        __builtin_memcpy(&f, &lo, 8);
        __builtin_memcpy(reinterpret_cast<char*>(&f) + 8, &hi, 8);
        return f;
    };
    auto read_y = [&](int flip, int stage, int half, int term, int b) {
        return fragment((yaddr[b] ^ flip) + stage * kStage + term * kStageY + half * 16 * kRowY,
                        kRowY);
    };
    auto read_x = [&](int flip, int stage, int half, int b) {
        return fragment((xaddr[b] ^ flip) + stage * kStage + half * 16 * kRowX, kRowX);
    };
    f32x16 acc[MI][NI] = {};
    constexpr int kProducts = MI * NI;
    // The products of half a step's tokens (of one term).  A wavefront issues an
    // instruction every 4 cycles and a product takes 32, so after each product
    // comes a share of the `reads` next fragments and the `moves` pieces to be
    // stored or loaded.
    auto half = [&](const bf16x8 (&x)[MI], const bf16x8 (&y)[NI], int reads, auto read, int moves,
                    auto move) {
#pragma unroll
        for (int k = 0; k < kProducts; ++k) {
            acc[k / NI][k % NI] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                x[k / NI], y[k % NI], acc[k / NI][k % NI], 0, 0, 0);
#pragma unroll
            for (int b = k * reads / kProducts; b < (k + 1) * reads / kProducts; ++b) read(b);
#pragma unroll
            for (int a = k * moves / kProducts; a < (k + 1) * moves / kProducts; ++a) move(a);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    if constexpr (LIGHT) {
        // A step's tile goes into one half of the LDS while the other may still be
        // read; the workgroups beside this one fill the waits.
        Stage r;
        load_stage(r);
        int flip = 0;
        auto nothing = [](int) {};
        for (uint32_t k = 0; k < left; k += kStepT) {
            store_stage(r, flip, 0);
            load_stage(r);
            barrier();
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                bf16x8 x[MI], y[NI];
#pragma unroll
                for (int b = 0; b < MI; ++b) x[b] = read_x(flip, 0, part, b);
#pragma unroll
                for (int b = 0; b < NI; ++b) y[b] = read_y(flip, 0, part, 0, b);
                half(x, y, 0, nothing, 0, nothing);
            }
            flip ^= kFlip;
        }
    } else if constexpr (kTerms == 1) {
        // Two steps s, s + 1 multiply the stages of one half of the LDS, store
        // tiles s + 2, s + 3 into the other and load tiles s + 4, s + 5 into the
        // registers this frees.  The workgroup meets once, before the last
        // quarter, whose fragments are then read: behind it the stored half may
        // be read and this one stored.
        constexpr int kFrags = MI + NI;
        struct Frags {
            bf16x8 x[MI], y[NI];
        };
        // fragment b in the order of their use: x 0, all y, the other x
        auto read = [&](Frags& f, int flip, int stage, int part, int b) {
            if (b >= 1 && b <= NI) f.y[b - 1] = read_y(flip, stage, part, 0, b - 1);
            else f.x[b ? b - NI : 0] = read_x(flip, stage, part, b ? b - NI : 0);
        };
        Stage r[2];
        Frags f0, f1;
        load_stage(r[0]);
        load_stage(r[1]);
        store_stage(r[0], 0, 0);
        load_stage(r[0]);
        store_stage(r[1], 0, 1);
        load_stage(r[1]);
        barrier();
#pragma unroll
        for (int b = 0; b < kFrags; ++b) read(f0, 0, 0, 0, b);
        int flip = 0;
        for (uint32_t k = 0; k < left; k += 2 * kStepT) {
            half(f0.x, f0.y, kFrags, [&](int b) { read(f1, flip, 0, 1, b); }, kPieces,
                 [&](int a) { store_piece(r[0], flip ^ kFlip, 0, a); });
            open_stage();
            half(f1.x, f1.y, kFrags, [&](int b) { read(f0, flip, 1, 0, b); }, kPieces,
                 [&](int a) { load_piece(r[0], a); });
            half(f0.x, f0.y, kFrags, [&](int b) { read(f1, flip, 1, 1, b); }, kPieces,
                 [&](int a) { store_piece(r[1], flip ^ kFlip, 1, a); });
            open_stage();
            barrier();
            flip ^= kFlip;
            half(f1.x, f1.y, kFrags, [&](int b) { read(f0, flip, 0, 0, b); }, kPieces,
                 [&](int a) { load_piece(r[1], a); });
        }
    } else {
        // A step multiplies the codes' fragments by the three terms' in turn,
        // stores the next tile into the other half and loads the one after into
        // the registers this frees; the workgroup meets before the last sixth.
        Stage r;
        bf16x8 x0[MI], x1[MI], y0[NI], y1[NI];
        load_stage(r);
        store_stage(r, 0, 0);
        load_stage(r);
        barrier();
#pragma unroll
        for (int b = 0; b < MI; ++b) x0[b] = read_x(0, 0, 0, b);
#pragma unroll
        for (int b = 0; b < NI; ++b) y0[b] = read_y(0, 0, 0, 0, b);
        int flip = 0;
        constexpr int kFirst = (kPieces + 2) / 3, kThen = 2 * kFirst < kPieces ? kFirst : kPieces - kFirst;
        constexpr int kLast = kPieces - kFirst - kThen;  // pieces of three sixths
        auto nothing = [](int) {};
        for (uint32_t k = 0; k < left; k += kStepT) {
            const int other = flip ^ kFlip;
            half(x0, y0, NI, [&](int b) { y1[b] = read_y(flip, 0, 0, 1, b); }, kFirst,
                 [&](int a) { store_piece(r, other, 0, a); });
            half(x0, y1, NI, [&](int b) { y0[b] = read_y(flip, 0, 0, 2, b); }, kThen,
                 [&](int a) { store_piece(r, other, 0, kFirst + a); });
            half(x0, y0, NI + MI,
                 [&](int b) {
                     if (b < NI) y1[b] = read_y(flip, 0, 1, 0, b);
                     else x1[b - NI] = read_x(flip, 0, 1, b - NI);
                 },
                 kLast, [&](int a) { store_piece(r, other, 0, kFirst + kThen + a); });
            open_stage();
            half(x1, y1, NI, [&](int b) { y0[b] = read_y(flip, 0, 1, 1, b); }, kFirst,
                 [&](int a) { load_piece(r, a); });
            half(x1, y0, NI, [&](int b) { y1[b] = read_y(flip, 0, 1, 2, b); }, kPieces - kFirst,
                 [&](int a) { load_piece(r, kFirst + a); });
            barrier();
            flip = other;
            half(x1, y1, NI + MI,
                 [&](int b) {
                     if (b < NI) y0[b] = read_y(flip, 0, 0, 0, b);
                     else x0[b - NI] = read_x(flip, 0, 0, b - NI);
                 },
                 0, nothing);
        }
    }

    // A lane holds 4 x 4 consecutive columns of one row of every 32 x 32 block.
    // Through LDS, a wavefront's own part of it, they become whole row pieces:
    // 32 rows at a time, padded by 16 bytes against bank conflicts.
    // Rows on 64-byte boundaries are written past the caches; the pieces of others
    // meet there with their neighbours' (2 x 270 tokens, 6279 x 5110 fp32: 121 us past
    // the caches, 91 through them; 6279 x 5120: 69, 79).
    const bool past = ((uintptr_t)(static_cast<typename G::T*>(p.grads.p) + i * p.grads.ld +
                                   p.grads.offset) |
                       (uintptr_t)(p.h * (int64_t)sizeof(typename G::T))) % 64 == 0;
    constexpr int kWide = MI * 32, kPadded = kWide + 4;
    static_assert(kWide == 64 && WO * WH * 32 * kPadded * 4 <= kLds, "LDS of the end");
    barrier();
    float* mine = reinterpret_cast<float*>(lds) + wave * 32 * kPadded;
#pragma unroll
    for (int c = 0; c < NI; ++c) {
        typedef typename G::T GT;
        constexpr int U = 16 / (int)sizeof(GT), kLanes = kWide / U, kRows = kWave / kLanes;
        const int64_t h = h0 + wh + lane % kLanes * U;
        GT* d = static_cast<GT*>(p.grads.p) + i * p.grads.ld + p.grads.offset +
                (o0 + wo + c * 32 + lane / kLanes) * p.h + h;
        const int64_t rows = p.o - (o0 + wo + c * 32 + lane / kLanes);  // from d on
        // what is added to, all loads at once
        Packed<GT, U> old[32 / kRows] = {};
        if (p.accumulate && !apart) {
#pragma unroll
            for (int r = 0; r < 32; r += kRows)
                if (r < rows && p.h - h >= U)
                    old[r / kRows] = load_packed<GT, U, false>(d + r * p.h);
        }
#pragma unroll
        for (int a = 0; a < MI; ++a)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = acc[a][c][e * 4 + k];
                __builtin_memcpy(__builtin_assume_aligned(
                                     mine + lane % 32 * kPadded + a * 32 + e * 8 + lane / 32 * 4, 16),
                                 v, 16);
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (apart) {
            float* part = g.part + ticket * TO * TH + (wo + c * 32) * TH + wh;
#pragma unroll
            for (int r = lane / 16; r < 32; r += 4) {
                float v[4];
                __builtin_memcpy(v, __builtin_assume_aligned(mine + r * kPadded + lane % 16 * 4, 16), 16);
                store_unit<float, 4, false>(part + r * TH + lane % 16 * 4, 4, v);
            }
        } else {
#pragma unroll
            for (int r = 0; r < 32; r += kRows) {
                float v[U], x[U];
                __builtin_memcpy(v, __builtin_assume_aligned(mine + (r + lane / kLanes) * kPadded +
                                                                 lane % kLanes * U, 16),
                                 sizeof(v));
                widen(old[r / kRows], x);
                if (r >= rows || h >= p.h) continue;
                if (p.h - h < U) {
                    put_sums<G, U>(p, i, p.o - rows + r, h, v);
                    continue;
                }
#pragma unroll
                for (int k = 0; k < U; ++k)
                    v[k] = p.accumulate ? __builtin_fmaf(p.scale, v[k], x[k]) : p.scale * v[k];
                // unlike barriers, or the compiler makes one store of both, through
                // the caches
                if (past) {
                    __builtin_amdgcn_sched_barrier(0);
                    store_whole<GT, U, true>(d + r * p.h, v);
                    __builtin_amdgcn_sched_barrier(0);
                } else {
                    __builtin_amdgcn_sched_barrier(1);
                    store_whole<GT, U, false>(d + r * p.h, v);
                    __builtin_amdgcn_sched_barrier(1);
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// The tile of a workgroup.  TAILS: o or h is not a multiple of 8; the tiles that
// end there take a slower loop (4097 x 4099 x 4096 tokens: 158 us, 200 where all
// tiles are 128 x 128; 4096 x 4096 with no such tile 116), which the others need not.
template <class Y, class G, int EDGE, int WO, int WH, bool TAILS, bool LIGHT = false>
__device__ __forceinline__ void wgrad_block(const WgradParams& p, const WgradPlan& g, uint8_t* lds) {
    const bool apart = g.runs > 1 && blockIdx.x >= g.whole;
    const int64_t ticket = apart ? blockIdx.x - g.whole : blockIdx.x;
    const int run = apart ? (int)(ticket % g.runs) : 0;
    const Tile tile =
        tile_at<EDGE, EDGE>(g, apart ? g.whole + ticket / g.runs : spread(ticket, g.whole));
    if (TAILS && ((p.o % 8 && p.o - tile.o0 < EDGE) || (p.h % 8 && p.h - tile.h0 < EDGE)))
        wgrad_tile<Y, G, EDGE, EDGE, WO, WH, true, LIGHT>(p, g, tile, ticket, run, apart, lds);
    else
        wgrad_tile<Y, G, EDGE, EDGE, WO, WH, false, LIGHT>(p, g, tile, ticket, run, apart, lds);
}

template <class Y, class G>
__global__ __launch_bounds__(512, 1) void k_act_wgrad_256(WgradParams p, WgradPlan g) {
    __shared__ __attribute__((aligned(16))) uint8_t lds[lds_bytes<256>()];
    wgrad_block<Y, G, 256, 2, 4, false>(p, g, lds);
}

template <class Y, class G>
__global__ __launch_bounds__(512, 1) void k_act_wgrad_256_tails(WgradParams p, WgradPlan g) {
    __shared__ __attribute__((aligned(16))) uint8_t lds[lds_bytes<256>()];
    wgrad_block<Y, G, 256, 2, 4, true>(p, g, lds);
}

template <class Y, class G>
__global__ __launch_bounds__(256, 2) void k_act_wgrad_128(WgradParams p, WgradPlan g) {
    __shared__ __attribute__((aligned(16))) uint8_t lds[lds_bytes<128>()];
    wgrad_block<Y, G, 128, 2, 2, true>(p, g, lds);
}

template <class G>
__global__ __launch_bounds__(256, 4) void k_act_wgrad_light(WgradParams p, WgradPlan g) {
    __shared__ __attribute__((aligned(16))) uint8_t lds[kLightLds];
    wgrad_block<El16, G, 128, 2, 2, true, true>(p, g, lds);
}

// Sum of the runs of the tiles that were summed apart, in order.
template <class G, int EDGE>
__device__ __forceinline__ void join_tile(const WgradParams& p, const WgradPlan& g) {
    constexpr int U = 4, kUnits = EDGE * EDGE / U, kBlocks = kUnits / kBlock;
    const int64_t which = blockIdx.x / kBlocks;
    const int at = (int)(blockIdx.x % kBlocks * kBlock + threadIdx.x) * U;
    const Tile tile = tile_at<EDGE, EDGE>(g, g.whole + which);
    const int64_t o = tile.o0 + at / EDGE, h = tile.h0 + at % EDGE;
    if (o >= p.o || h >= p.h) return;
    const float* part = g.part + which * g.runs * EDGE * EDGE + at;
    float sum[U] = {};
    constexpr int kAhead = 8;  // runs whose loads are in flight
    for (int s = 0; s < g.runs; s += kAhead) {
        float v[kAhead][U];
#pragma unroll
        for (int a = 0; a < kAhead; ++a)
            if (s + a < g.runs) load_unit<float, U, true>(part + (int64_t)(s + a) * EDGE * EDGE, U, v[a]);
#pragma unroll
        for (int a = 0; a < kAhead; ++a)
            if (s + a < g.runs)
#pragma unroll
                for (int k = 0; k < U; ++k) sum[k] += v[a][k];
    }
    put_sums<G, U>(p, tile.i, o, h, sum);
}

template <class G>
__global__ __launch_bounds__(kBlock) void k_act_wgrad_join(WgradParams p, WgradPlan g) {
    if (g.edge == 256) join_tile<G, 256>(p, g);
    else join_tile<G, 128>(p, g);
}

}  // namespace

size_t act_wgrad_workspace(int64_t n, int64_t t, int64_t o, int64_t h) {
    size_t most = 0;  // of either type of dy
    for (int bf16 = 0; bf16 < 2; ++bf16) {
        WgradPlan g = {};
        wgrad_plan(n, t, o, h, bf16, &g);
        const size_t bytes = wgrad_part_bytes(g);
        most = bytes > most ? bytes : most;
    }
    return most;
}

hipError_t launch_act_wgrad(const WgradParams& p, void* ws, hipStream_t s) {
    WgradPlan g = {};
    wgrad_plan(p.n, p.t, p.o, p.h, p.dy.bf16, &g);
    g.part = static_cast<float*>(ws);
    const int64_t blocks = g.whole + g.rest * g.runs;
    if (blocks > 0xFFFFFFFFll / 512) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)blocks);
    if (g.light) {
        if (p.grads.bf16)
            hipLaunchKernelGGL((k_act_wgrad_light<El16>), grid, dim3(256), 0, s, p, g);
        else
            hipLaunchKernelGGL((k_act_wgrad_light<El32>), grid, dim3(256), 0, s, p, g);
    } else if (g.edge == 256 && (p.o % 8 || p.h % 8)) {
        LOSSY_LAUNCH2(k_act_wgrad_256_tails, p.dy.bf16, p.grads.bf16, grid, dim3(512), s, p, g);
    } else if (g.edge == 256) {
        LOSSY_LAUNCH2(k_act_wgrad_256, p.dy.bf16, p.grads.bf16, grid, dim3(512), s, p, g);
    } else {
        LOSSY_LAUNCH2(k_act_wgrad_128, p.dy.bf16, p.grads.bf16, grid, dim3(256), s, p, g);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || g.runs == 1) return e;
    const dim3 join((unsigned)(g.rest * (g.edge * g.edge / 4 / kBlock)));
    if (p.grads.bf16)
        hipLaunchKernelGGL((k_act_wgrad_join<El16>), join, dim3(kBlock), 0, s, p, g);
    else
        hipLaunchKernelGGL((k_act_wgrad_join<El32>), join, dim3(kBlock), 0, s, p, g);
    return hipGetLastError();
}

}  // namespace lossy
