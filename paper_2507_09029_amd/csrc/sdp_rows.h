// Rows of any length and alignment, read and written in pieces of 16 bytes (device code): what the norms, the embedding and the
// token loss share.
//
// A piece is 8 bf16 or 4 fp32 values.  Rows of a matrix whose width is no whole number of pieces start at any element; the memory
// instructions of 16 bytes take such addresses, and rows of 1501 bf16 stream at the rate of aligned ones, so there is one form for
// both.  The values behind the last whole piece, 7 at most, are a lane's each.  A lane without a piece reads the last one again, which costs no
// traffic, and looks away when it uses it: a load is then one instruction without a condition.  (Where the row's end was looked
// for as it was loaded, every load of its wave waited for the one before: norm backward of 16384 x 768 bf16 49 us, now 22.)
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

// Whether rows of `row_bytes` in these matrices are read around the caches: far more than the eight L2s' 32 MB, and rows of whole lines, since
// a line that two rows share is else fetched twice.  With / without, us: norm forward of 16384 x 2048 bf16 and a sum (134 MB) 47.5 / 49.3,
// backward with the skip connection (201 MB) 49.4 / 51.6, loss of 8192 x 32000 (524 MB) 177.7 / 182.1; but norm forward of 16384 x 768
// (50 MB) 20.2 / 16.6, backward (75 MB) 24.1 / 22.4, and loss of 1000 x 50001, no whole lines, 57.6 / 49.6.
inline bool read_once(std::initializer_list<Extent> of, size_t row_bytes) {
    size_t all = 0;
    for (const Extent& m : of) {
        if (m.bytes && !aligned_to(m.p, 128)) return false;
        all += m.bytes;
    }
    return row_bytes % 128 == 0 && all >= (size_t)1 << 27;
}

// A launch of up to 2^32 - 1 workgroups: one dimension of a grid holds less than 2^32 threads.  Rows of a fixed length, so that no
// kernel waits for the grid's size (reading it, and dividing in 64 bits, cost 0.1 to 0.4 us a launch).
constexpr int kGridRow = 20; // 2^20 workgroups of at most 1024 threads
inline dim3 grid_of(int64_t groups) {
    return dim3((unsigned)(groups < (1 << kGridRow) ? groups : 1 << kGridRow), (unsigned)((groups - 1) >> kGridRow) + 1);
}
__device__ inline uint32_t group_id() { return blockIdx.y << kGridRow | blockIdx.x; } // the grid's last row may have more than are needed

template <int BF16>
struct Row {
    typedef std::conditional_t<BF16, uint16_t, float> Elem;
    typedef std::conditional_t<BF16, u32x4_at2, u32x4_at4> Piece;
    static constexpr int N = BF16 ? 8 : 4; // values of a piece

    static __device__ inline float one(const Elem* p) {
        if constexpr (BF16) return __uint_as_float((uint32_t)*p << 16);
        else return *p;
    }
    static __device__ inline float rounded(float v) { return BF16 ? (float)(__bf16)v : v; }
    static __device__ inline void put(Elem* p, float v) {
        if constexpr (BF16) *p = __builtin_bit_cast(uint16_t, (__bf16)v);
        else *p = v;
    }
    // values of a row of n that whole pieces hold
    static __host__ __device__ inline int whole(int n) { return n / N * N; }

    // The piece from value e (a multiple of N) on of a row whose whole pieces hold `whole` values; the last one for lanes behind it.  ONCE:
    // read_once's answer, at compile time (of two loads behind a condition the compiler makes one).
    template <int ONCE = 0>
    static __device__ inline u32x4 load(const Elem* row, int e, int whole) {
        return whole ? load_some<ONCE>(row, e, whole) : u32x4{0, 0, 0, 0};
    }
    // the same of a row that has a whole piece
    template <int ONCE = 0>
    static __device__ inline u32x4 load_some(const Elem* row, int e, int whole) {
        const Piece* p = (const Piece*)((const char*)row + (uint32_t)min(e, whole - N) * (uint32_t)sizeof(Elem));
        return ONCE ? __builtin_nontemporal_load(p) : *p;
    }
    // what load gave, or `fill` (every value of a word) in lanes behind the row's whole pieces
    static __device__ inline u32x4 mine(const u32x4& w, int e, int whole, uint32_t fill = 0) {
        return e < whole ? w : u32x4{fill, fill, fill, fill};
    }
    static __device__ inline void store(Elem* row, int e, int whole, const u32x4& w) {
        if (e < whole) __builtin_nontemporal_store(w, (Piece*)((char*)row + (uint32_t)e * (uint32_t)sizeof(Elem)));
    }
    static __device__ inline void unpack(const u32x4& w, float (&v)[N]) {
        if constexpr (BF16) { // a bf16 is the high half of an fp32: even values sit in the low 16 bits of each word
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = __uint_as_float(w[i] << 16);
                v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(w[i]);
        }
    }
    static __device__ inline u32x4 pack(const float (&v)[N]) {
        u32x4 w;
        if constexpr (BF16) {
            typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bf16x2 p = {(__bf16)v[2 * i], (__bf16)v[2 * i + 1]}; // to nearest, ties to even
                w[i] = __builtin_bit_cast(uint32_t, p);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(v[i]);
        }
        return w;
    }
};

// Pieces are unpacked anew from here on: the compiler would rather keep their fp32 values, twice the registers (16 pieces of logits 177
// instead of 99, two waves a SIMD instead of four).
template <int P>
__device__ inline void again(u32x4 (&w)[P]) {
#pragma unroll
    for (int i = 0; i < P; ++i) asm volatile("" : "+v"(w[i]));
}
// These sums are made here, not where they are next looked at: what they are made of would stay in registers till then.
template <int P, int N>
__device__ inline void settle(float (&x)[P][N]) {
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
        for (int k = 0; k < N; ++k) asm volatile("" : "+v"(x[i][k]));
}

// Sum and maximum over a wave, in a fixed order; every lane has the result.  Six steps on the vector unit's own lane moves (down the rows of
// 16 lanes, then from row to row), not through LDS.
template <int CTRL>
__device__ inline float from_lane(float none, float x) { // x of the lane that CTRL names, `none` where there is none
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(none), __float_as_int(x), CTRL, 0xF, 0xF, false));
}
__device__ inline float wave_sum(float x) {
    x += from_lane<0x111>(0.f, x); // row_shr 1, 2, 4, 8: a row's last lane has the row's sum
    x += from_lane<0x112>(0.f, x);
    x += from_lane<0x114>(0.f, x);
    x += from_lane<0x118>(0.f, x);
    x += from_lane<0x142>(0.f, x); // row_bcast 15, 31: the sums of the rows before
    x += from_lane<0x143>(0.f, x);
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}
__device__ inline float wave_max(float x) {
    x = fmaxf(x, from_lane<0x111>(x, x));
    x = fmaxf(x, from_lane<0x112>(x, x));
    x = fmaxf(x, from_lane<0x114>(x, x));
    x = fmaxf(x, from_lane<0x118>(x, x));
    x = fmaxf(x, from_lane<0x142>(x, x));
    x = fmaxf(x, from_lane<0x143>(x, x));
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
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
