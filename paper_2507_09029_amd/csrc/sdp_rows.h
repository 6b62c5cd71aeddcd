// Rows of any length and alignment, read and written in pieces of 16 bytes (device code): what the norms, the embedding and the
// token loss share.
//
// A piece is 8 bf16 or 4 fp32 values.  Rows of a matrix whose width is no whole number of pieces start at any element; the memory
// instructions of 16 bytes take such addresses, and rows of 1501 bf16 stream at the rate of aligned ones, so there is one form for
// both.  The last piece of a row may be short: its values are moved one by one.
//
// Stores are non-temporal: what is written here is far more than a cache holds, or read next by another kernel, and pushes what is being
// read out of it (embedding of 16384 x 2048 bf16 22.0 -> 17.0 us, its gradient's sums 44 -> 34, norm 50.1 -> 48.8, loss of 8192 x 32000 186 -> 182).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "sdp_internal.h"

namespace sdp {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 __attribute__((aligned(2))) u32x4_at2;
typedef u32x4 __attribute__((aligned(4))) u32x4_at4;
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Whether rows of `row_bytes` in these matrices are read around the caches: more than they hold (the eight L2s 32 MB), and rows of whole
// lines, since a line that two rows share is else fetched twice.  Norm forward of 16384 x 2048 bf16 with / without 46.9 / 48.4 us, loss of
// 8192 x 32000 185 / 190; but rows that are no whole lines: loss of 1000 x 50001 57.6 / 49.6.
inline bool read_once(std::initializer_list<Extent> of, size_t row_bytes) {
    size_t all = 0;
    for (const Extent& m : of) {
        if (m.bytes && !aligned_to(m.p, 128)) return false;
        all += m.bytes;
    }
    return row_bytes % 128 == 0 && all >= (size_t)1 << 26;
}

template <int BF16>
struct Row;

template <>
struct Row<1> {
    typedef uint16_t Elem;
    static constexpr int N = 8; // values of a piece

    static __device__ inline float one(const Elem* p) { return __uint_as_float((uint32_t)*p << 16); }
    static __device__ inline void put(Elem* p, float v) { *p = __builtin_bit_cast(uint16_t, (__bf16)v); }

    // the piece from value e on of a row of n; values past its end are `fill`'s (two bf16 in a word); ONCE: read_once's answer, at compile time (of two loads
    // behind a condition the compiler makes one)
    template <int ONCE = 0>
    static __device__ inline u32x4 load(const Elem* row, int e, int n, uint32_t fill = 0) {
        if (e + N <= n) return ONCE ? __builtin_nontemporal_load((const u32x4_at2*)(row + e)) : *(const u32x4_at2*)(row + e);
        u32x4 w = {fill, fill, fill, fill};
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (e + i < n) w[i / 2] = i % 2 ? (w[i / 2] & 0xFFFFu) | (uint32_t)row[e + i] << 16 : (w[i / 2] & 0xFFFF0000u) | row[e + i];
        return w;
    }
    static __device__ inline void store(Elem* row, int e, int n, const u32x4& w) {
        if (e + N <= n) {
            __builtin_nontemporal_store(w, (u32x4_at2*)(row + e));
            return;
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (e + i < n) row[e + i] = (uint16_t)(i % 2 ? w[i / 2] >> 16 : w[i / 2]);
    }
    // a bf16 is the high half of an fp32: even values sit in the low 16 bits of each word
    static __device__ inline void unpack(const u32x4& w, float (&v)[N]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
    static __device__ inline u32x4 pack(const float (&v)[N]) {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bf16x2 p = {(__bf16)v[2 * i], (__bf16)v[2 * i + 1]}; // to nearest, ties to even
            w[i] = __builtin_bit_cast(uint32_t, p);
        }
        return w;
    }
};

template <>
struct Row<0> {
    typedef float Elem;
    static constexpr int N = 4;

    static __device__ inline float one(const Elem* p) { return *p; }
    static __device__ inline void put(Elem* p, float v) { *p = v; }

    template <int ONCE = 0>
    static __device__ inline u32x4 load(const Elem* row, int e, int n, uint32_t fill = 0) {
        if (e + N <= n) return ONCE ? __builtin_nontemporal_load((const u32x4_at4*)(row + e)) : *(const u32x4_at4*)(row + e);
        u32x4 w = {fill, fill, fill, fill};
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (e + i < n) w[i] = __float_as_uint(row[e + i]);
        return w;
    }
    static __device__ inline void store(Elem* row, int e, int n, const u32x4& w) {
        if (e + N <= n) {
            __builtin_nontemporal_store(w, (u32x4_at4*)(row + e));
            return;
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (e + i < n) row[e + i] = __uint_as_float(w[i]);
    }
    static __device__ inline void unpack(const u32x4& w, float (&v)[N]) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = __uint_as_float(w[i]);
    }
    static __device__ inline u32x4 pack(const float (&v)[N]) {
        return {__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    }
};

// Sums over a wave, in a fixed order; every lane has the result.
__device__ inline float wave_sum(float x) {
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) x += __shfl_xor(x, d, 64);
    return x;
}
__device__ inline float wave_max(float x) {
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) x = fmaxf(x, __shfl_xor(x, d, 64));
    return x;
}

// Token id or label t; anything outside [0, V) is -1.  Where many are loaded at once the type has to be known at compile time: with a
// branch around each load the next waits for the last.
template <int WIDE>
__device__ inline int token_id(const void* ids, int64_t t, int V) {
    typedef std::conditional_t<WIDE, uint64_t, uint32_t> Id;
    const Id v = ((const Id*)ids)[t];
    return v < (Id)V ? (int)v : -1;
}
__device__ inline int token_id(const void* ids, int wide, int64_t t, int V) {
    return wide ? token_id<1>(ids, t, V) : token_id<0>(ids, t, V);
}

} // namespace sdp
