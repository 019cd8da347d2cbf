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
__device__ __forceinline__ float widen(T x) {
    return (float)x;
}

template <class T>
__device__ __forceinline__ T narrow(float x) {
    return (T)x;  // round to nearest even
}

// Columns of one unit: 16 bytes of the narrowest of its types, so that a
// wavefront's access to that type is 1 KiB of consecutive memory.
template <class A, class B>
constexpr int unit_of() {
    return 16 / (int)(sizeof(typename A::T) < sizeof(typename B::T) ? sizeof(typename A::T)
                                                                   : sizeof(typename B::T));
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

// U consecutive elements from p, of which the first `have` exist (the others
// read as 0).
template <class T, int U, bool STREAM>
__device__ __forceinline__ void load_unit(const T* p, int64_t have, float (&x)[U]) {
    constexpr int kPer = 16 / (int)sizeof(T);  // elements of one access
    constexpr int kStep = U < kPer ? U : kPer;
    if (have >= U) {
        T e[U];
#pragma unroll
        for (int a = 0; a < U; a += kStep) {
            auto v = load_raw<kStep*(int)sizeof(T), (int)sizeof(T), STREAM>(p + a);
            __builtin_memcpy(e + a, &v, sizeof(v));
        }
#pragma unroll
        for (int c = 0; c < U; ++c) x[c] = widen(e[c]);
    } else {
#pragma unroll
        for (int c = 0; c < U; ++c) x[c] = c < have ? widen(p[c]) : 0.0f;
    }
}

// The first `have` of U consecutive elements, rounded to T.
template <class T, int U, bool STREAM>
__device__ __forceinline__ void store_unit(T* p, int64_t have, const float (&x)[U]) {
    constexpr int kPer = 16 / (int)sizeof(T);
    constexpr int kStep = U < kPer ? U : kPer;
    if (have >= U) {
        T e[U];
#pragma unroll
        for (int c = 0; c < U; ++c) e[c] = narrow<T>(x[c]);
#pragma unroll
        for (int a = 0; a < U; a += kStep) {
            typename RawOf<kStep*(int)sizeof(T)>::T v;
            __builtin_memcpy(&v, e + a, sizeof(v));
            store_raw<kStep*(int)sizeof(T), (int)sizeof(T), STREAM>(p + a, v);
        }
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

// Whether token row tk = i * t + j lies inside its worker's batch.
__device__ __forceinline__ bool in_batch(const int32_t* lengths, uint32_t tk, int64_t t) {
    if (!lengths) return true;
    const uint32_t i = tk / (uint32_t)t;
    return (int64_t)(tk - i * (uint32_t)t) < lengths[i];
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

// Launch K<A, B> for the element types given as truth values (bf16?).
#define LOSSY_LAUNCH2(K, a, b, grid, block, s, ...)                                         \
    do {                                                                                    \
        if ((a) && (b))                                                                     \
            hipLaunchKernelGGL((K<El16, El16>), grid, block, 0, s, __VA_ARGS__);            \
        else if (a)                                                                         \
            hipLaunchKernelGGL((K<El16, El32>), grid, block, 0, s, __VA_ARGS__);            \
        else if (b)                                                                         \
            hipLaunchKernelGGL((K<El32, El16>), grid, block, 0, s, __VA_ARGS__);            \
        else                                                                                \
            hipLaunchKernelGGL((K<El32, El32>), grid, block, 0, s, __VA_ARGS__);            \
    } while (0)

// A grid of at most 2^20 workgroups (kernels stride over the rest).
inline unsigned grid_for(int64_t blocks) {
    const int64_t cap = 1 << 20;
    return (unsigned)(blocks < 1 ? 1 : (blocks > cap ? cap : blocks));
}

// Threads along a row's units (a power of two from 8 to kBlock) when a
// workgroup takes kBlock / lanes rows: as many as a short row has units; a
// whole wavefront per row where the rows alone fill the chip (each lane then has
// several accesses in flight), the whole workgroup where they do not.
inline int lanes_per_row(int64_t rows, int64_t units) {
    const int most = rows >= 4096 ? kWave : kBlock;
    int lanes = 8;
    while (lanes < most && lanes < units) lanes *= 2;
    return lanes;
}

}  // namespace lossy
