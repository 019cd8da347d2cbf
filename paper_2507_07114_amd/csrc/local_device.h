// Device helpers shared by the local-gradient kernels: element types, 16-byte
// units of any alignment, token batches, e4m3 codes.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "local.h"

namespace lossy {

constexpr int kBlock = 256;
constexpr int kWave = 64;

// Element types of rows and activations.
struct El32 {
    typedef float T;
};
struct El16 {
    typedef __bf16 T;
};

template <class T>
__device__ __forceinline__ T narrow(float x) {
    return (T)x;  // round to nearest even
}

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Descriptor word of a raw buffer (offsets in bytes, no format, no swizzle).
constexpr int kBufferRaw = 0x00020000;

// Raw memory accesses of 4, 8 or 16 bytes at any element's alignment: global
// memory takes such vectors at any address, so rows that start anywhere need no
// element-by-element form.  STREAM: non-temporal, for data that the call touches once.
template <int BYTES>
struct RawOf;
template <>
struct RawOf<4> {
    typedef uint32_t T;
};
template <>
struct RawOf<8> {
    typedef u32x2 T;
};
template <>
struct RawOf<16> {
    typedef u32x4 T;
};

template <int BYTES, int ALIGN, bool STREAM>
__device__ __forceinline__ typename RawOf<BYTES>::T load_raw(const void* p) {
    typedef typename RawOf<BYTES>::T V __attribute__((aligned(ALIGN)));
    if (STREAM) return __builtin_nontemporal_load(static_cast<const V*>(p));
    return *static_cast<const V*>(p);
}

template <int BYTES, int ALIGN, bool STREAM>
__device__ __forceinline__ void store_raw(void* p, typename RawOf<BYTES>::T v) {
    typedef typename RawOf<BYTES>::T V __attribute__((aligned(ALIGN)));
    if (STREAM) __builtin_nontemporal_store(v, static_cast<V*>(p));
    else *static_cast<V*>(p) = v;
}

// U consecutive elements as they lie in memory, in words: loads that are to be in
// flight together give these.  A conversion inside a branch, elements that a
// branch leaves apart too, would wait for their load.
template <class T, int U>
struct Packed {
    uint32_t w[U * (int)sizeof(T) / 4];
};

// U elements from p, all of which exist.
template <class T, int U, bool STREAM>
__device__ __forceinline__ Packed<T, U> load_packed(const T* p) {
    constexpr int kBytes = U * (int)sizeof(T), kStep = kBytes < 16 ? kBytes : 16;
    Packed<T, U> r;
#pragma unroll
    for (int a = 0; a < kBytes; a += kStep) {
        auto v = load_raw<kStep, (int)sizeof(T), STREAM>(reinterpret_cast<const uint8_t*>(p) + a);
        __builtin_memcpy(r.w + a / 4, &v, sizeof(v));
    }
    return r;
}

template <int U>
__device__ __forceinline__ void widen(const Packed<float, U>& r, float (&x)[U]) {
#pragma unroll
    for (int c = 0; c < U; ++c) x[c] = __uint_as_float(r.w[c]);
}

template <int U>
__device__ __forceinline__ void widen(const Packed<__bf16, U>& r, float (&x)[U]) {
#pragma unroll
    for (int c = 0; c < U; c += 2) {
        x[c] = __uint_as_float(r.w[c / 2] << 16);
        x[c + 1] = __uint_as_float(r.w[c / 2] & 0xFFFF0000u);
    }
}

// U elements to p, rounded to T.
template <class T, int U, bool STREAM>
__device__ __forceinline__ void store_whole(T* p, const float (&x)[U]) {
    constexpr int kStep = U * (int)sizeof(T) < 16 ? U : 16 / (int)sizeof(T);
    T e[U];
#pragma unroll
    for (int c = 0; c < U; ++c) e[c] = narrow<T>(x[c]);
#pragma unroll
    for (int a = 0; a < U; a += kStep) {
        typename RawOf<kStep*(int)sizeof(T)>::T v;
        __builtin_memcpy(&v, e + a, sizeof(v));
        store_raw<kStep*(int)sizeof(T), (int)sizeof(T), STREAM>(p + a, v);
    }
}

// A lane's U columns of a row of h, those from c0 on being its own: it holds
// columns at() .. at() + U, moved back to the row's last U where c0 + U passes
// its end (then the first of them are another lane's, too).  A row shorter than U
// is held from its first column.
template <int U>
struct Columns {
    int64_t c0, h;
    __device__ __forceinline__ int64_t at() const {
        const int64_t last = h < U ? 0 : h - U;
        return c0 < last ? c0 : last;
    }
    __device__ __forceinline__ bool whole() const { return h - c0 >= U; }
    // the held columns of a row at p; NARROW: h < U, of which the last is repeated
    template <class T, bool STREAM, bool NARROW>
    __device__ __forceinline__ Packed<T, U> load(const T* p) const {
        if (!NARROW) return load_packed<T, U, STREAM>(p + at());
        T e[U];
#pragma unroll
        for (int c = 0; c < U; ++c) e[c] = p[c < h ? c : h - 1];
        Packed<T, U> r;
        __builtin_memcpy(r.w, e, sizeof(r.w));
        return r;
    }
    // the lane's own of the held columns
    template <class T, bool STREAM>
    __device__ __forceinline__ void store(T* p, const float (&x)[U]) const {
        if (whole()) {
            store_whole<T, U, STREAM>(p + c0, x);
        } else {
            const int64_t c1 = at();
#pragma unroll
            for (int c = 0; c < U; ++c)
                if (c1 + c >= c0 && c1 + c < h) p[c1 + c] = narrow<T>(x[c]);
        }
    }
};

// U consecutive elements from p, of which the first `have` exist (the others
// read as 0).
template <class T, int U, bool STREAM>
__device__ __forceinline__ void load_unit(const T* p, int64_t have, float (&x)[U]) {
    if (have >= U) {
        widen(load_packed<T, U, STREAM>(p), x);
    } else {
#pragma unroll
        for (int c = 0; c < U; ++c) x[c] = c < have ? (float)p[c] : 0.0f;
    }
}

// The first `have` of U consecutive elements, rounded to T.
template <class T, int U, bool STREAM>
__device__ __forceinline__ void store_unit(T* p, int64_t have, const float (&x)[U]) {
    if (have >= U) {
        store_whole<T, U, STREAM>(p, x);
    } else {
#pragma unroll
        for (int c = 0; c < U; ++c)
            if (c < have) p[c] = narrow<T>(x[c]);
    }
}

// Tokens of worker i's batch.
__device__ __forceinline__ int64_t batch_len(const int32_t* lengths, int i, int64_t t) {
    if (!lengths) return t;
    const int64_t m = lengths[i];
    return m < 0 ? 0 : (m > t ? t : m);
}

// Table row of a token, or -1 where the table does not hold it.  Held ids are
// first .. first + v - 1; the unsigned difference wraps where id < first, and
// where id - first would overflow.
__device__ __forceinline__ int64_t table_row(const TokenView& tok, int64_t id) {
    const uint64_t row = (uint64_t)id - (uint64_t)tok.first;
    return row < (uint64_t)tok.v ? (int64_t)row : -1;
}

// Token j of worker i.
__device__ __forceinline__ int64_t token_id(const TokenView& tok, int i, int64_t j) {
    const int64_t at = (int64_t)i * tok.ld + j;
    return tok.wide ? static_cast<const int64_t*>(tok.ids)[at]
                    : (int64_t) static_cast<const int32_t*>(tok.ids)[at];
}

__device__ __forceinline__ int64_t table_row(const TokenView& tok, int i, int64_t j) {
    return table_row(tok, token_id(tok, i, j));
}

// Launch K<A, B> for the element types given as truth values (bf16?), with `lds`
// bytes of LDS besides the kernel's own.
#define LOSSY_LAUNCH2_LDS(K, a, b, grid, block, lds, s, ...)                                \
    do {                                                                                    \
        if ((a) && (b))                                                                     \
            hipLaunchKernelGGL((K<El16, El16>), grid, block, lds, s, __VA_ARGS__);          \
        else if (a)                                                                         \
            hipLaunchKernelGGL((K<El16, El32>), grid, block, lds, s, __VA_ARGS__);          \
        else if (b)                                                                         \
            hipLaunchKernelGGL((K<El32, El16>), grid, block, lds, s, __VA_ARGS__);          \
        else                                                                                \
            hipLaunchKernelGGL((K<El32, El32>), grid, block, lds, s, __VA_ARGS__);          \
    } while (0)
#define LOSSY_LAUNCH2(K, a, b, grid, block, s, ...) \
    LOSSY_LAUNCH2_LDS(K, a, b, grid, block, 0, s, __VA_ARGS__)

// A grid of at most 2^20 workgroups (kernels stride over the rest).
inline unsigned grid_for(int64_t blocks) {
    const int64_t cap = 1 << 20;
    return (unsigned)(blocks < 1 ? 1 : (blocks > cap ? cap : blocks));
}

// Lanes that walk a row of that many units: a power of two from 8 to 128.
inline int lanes_per_row(int64_t units) {
    int lanes = 8;
    while (lanes < kBlock / 2 && lanes < units) lanes *= 2;
    return lanes;
}

// Units of token rows, dealt out flat: a workgroup takes kBlock * PER consecutive
// units of a group of rows, whatever rows they belong to, so that the chip
// as a whole works on one stretch of memory (a wavefront walking a row of its
// own reads 4.8 TB/s where this reads 6).  Rows are grouped so that a unit's
// number inside the group has 31 bits; grid.x runs through a group, grid.y over
// the groups.
struct FlatRows {
    uint32_t units, rows;  // units of a row, rows of a group
    uint32_t mul, shift;   // unit / units = unit * mul >> shift
    int64_t total;         // rows of all groups
};

__device__ __forceinline__ uint32_t flat_row(const FlatRows& f, uint32_t unit) {
    return (uint32_t)(((uint64_t)unit * f.mul) >> f.shift);
}

// With s = ceil(log2 units) and mul = ceil(2^(31 + s) / units) the quotient is
// exact for 31-bit numbers: the excess mul * units - 2^(31 + s) is below 2^s.
// Returns the grid; false where the rows are too many for one.
inline bool flat_rows(int64_t total, int64_t units, int per, FlatRows* f, dim3* grid) {
    int s = 0;
    while ((1ll << s) < units) ++s;
    f->units = (uint32_t)units;
    f->mul = (uint32_t)(((1ull << (31 + s)) + units - 1) / units);
    f->shift = 31 + s;
    f->total = total;
    const int64_t span = kBlock * (int64_t)per;
    int64_t rows = (0x7FFFFFFFll - span) / units;
    rows = rows < total ? rows : total;
    // 2^23 workgroups of 256 threads stay below 2^32 threads
    if (rows * units > span << 23) rows = (span << 23) / units;
    if (rows < 1) return false;
    f->rows = (uint32_t)rows;
    const int64_t y = (total + rows - 1) / rows;
    if (y > 65535) return false;
    *grid = dim3((unsigned)((rows * units + span - 1) / span), (unsigned)y);
    return true;
}

}  // namespace lossy
