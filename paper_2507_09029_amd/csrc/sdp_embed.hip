// Token embedding: rows of a matrix by token id, scaled, and the gradient of the matrix.
//
//   forward   Y[t] = scale E[id_t]            backward  dE[v] = scale sum_{t : id_t = v} dY[t]
//
// Both are bound by memory.  The backward pass turns the scatter into a gather: tokens are sorted by id, and the rows of dY that
// belong to one row of dE are then neighbours in the sorted order, to be summed by one wave in registers.  No atomics on floats: each
// row's sum has one order, given by the ids alone.
//
// Batches of up to kSmall tokens have a launch of their own (embed_small_kernel).  Otherwise the sort is one launch in which no workgroup
// waits for another.  Each owns a share of the ids and goes through all T ids itself: it counts how many belong to workgroups before it
// (where its part of the order starts) and lists its own, counts how often each id occurs, and writes the listed tokens to their
// places.  The ids are few bytes and come from the cache for all workgroups but the first, so that T / 1024 steps a workgroup take
// less than the launches and the waiting of a sort by digits: 10 us for 16384 ids of 32000 whose frequencies fall as 1 / rank (9 where
// all are as frequent, 7 with none to sort, 16 with one id alone), 40 for 131072 (112 with one id alone: one workgroup places them).
//
// A token that occurs often (the most frequent of a text are several percent of it; in a padded batch one may be all) would be
// one wave's long sum.  The sorted order is therefore cut into chunks of kChunk tokens, of a workgroup each (for 512 columns of bf16): a
// row whose tokens lie within a chunk is finished there, the others leave partial sums in fp32, which a last launch adds up.
#include <cmath>
#include <type_traits>

#include "sdp_internal.h"
#include "sdp_rows.h"

namespace {

using sdp::Row;
using sdp::u32x4;

struct EmbedFwd {
    const void *E, *ids;
    void* Y;
    int T, V, d, wide;
    float scale;
};

// One wave copies a row.
template <int BF16>
__global__ __launch_bounds__(256) void embed_fwd_kernel(EmbedFwd a) {
    typedef Row<BF16> Rw;
    typedef typename Rw::Elem Elem;
    constexpr int N = Rw::N, B = 4; // pieces in flight
    const int64_t t = (int64_t)sdp::group_id() * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    if (t >= a.T) return;
    const int lane = threadIdx.x & 63, id = sdp::token_id(a.ids, a.wide, t, a.V), whole = Rw::whole(a.d);
    const Elem* in = (const Elem*)a.E + (int64_t)id * a.d;
    Elem* out = (Elem*)a.Y + t * a.d;
    const bool tail = whole + lane < a.d; // this lane has a value behind the whole pieces
    const float last = tail && id >= 0 ? Rw::one(in + whole + lane) : 0.f;
    for (int e0 = lane * N; e0 - lane * N < whole; e0 += B * 64 * N) {
        u32x4 w[B] = {};
        if (id >= 0)
#pragma unroll
            for (int i = 0; i < B; ++i) w[i] = Rw::load(in, e0 + i * 64 * N, whole);
#pragma unroll
        for (int i = 0; i < B; ++i) {
            float v[N];
            Rw::unpack(w[i], v);
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] *= a.scale;
            Rw::store(out, e0 + i * 64 * N, whole, Rw::pack(v));
        }
    }
    if (tail) Rw::put(out + whole + lane, last * a.scale);
}

constexpr int kSortWaves = 16, kSortShift = 8, kMaxRange = 960, kAhead = 16;
// sorted tokens of a wave, all of whose rows are in flight at once, and of a workgroup
constexpr int kPiece = 16, kSumWaves = 8, kChunk = kPiece * kSumWaves;
// Rows that a wave clears if they do not occur: few, since waves that store once or twice and end write memory in its order, and faster
// (whole gradient of 16384 tokens, 32000 x 2048 bf16, and of 1200, 64000 x 2048: two rows 42.3 and 50.1 us, eight 45.8 and 52.3, 64 47.7 and 63.9).
constexpr int kClear = 2;

struct Sorted {
    int32_t* order; // [T] tokens, by key of their id, then by place
    int32_t* ids;   // [T] their ids
    int32_t* start; // [keys + 1] where the tokens of a key's row start; start[keys] = number of tokens that have an id
    int2* spans;    // [chunks] {row, last chunk} of the row that starts in the chunk and goes on in the next, or {-1, 0}
};

// What a workgroup sorts: `range` ids, one of each (1 << shift) neighbours, since the frequent ids of a vocabulary often are neighbours.  Which of
// them changes from one to the next, so that rows written one after the other are not all a power of two apart.  The order is that of
// the keys: ids of workgroup 0, of 1, ...; the last ones may lie beyond V.  Whole gradient, bf16, frequencies as 1 / rank, ids in order of
// frequency and in any order: 16384 tokens, 32000 x 2048: 42.2 and 42.3 us, with neighbours in one workgroup 49.3 and 41.2; 131072
// tokens: 184 and 185, 266 and 178.  Without the change 5000 tokens, 50001 x 1600 take 39.8 and 38.1, with it 38.0 and 36.8.
struct Split {
    int range, shift;
    __host__ __device__ int groups() const { return 1 << shift; }
    __host__ __device__ int keys() const { return range << shift; }
    __device__ uint32_t place(uint32_t id) const { return id >> shift; }
    __device__ uint32_t group(uint32_t id) const { return (id ^ place(id)) & (groups() - 1); }
    __device__ uint32_t id(uint32_t group, uint32_t place) const { return place << shift | ((group ^ place) & (groups() - 1)); }
    __device__ int key(uint32_t id) const { return (int)(group(id) * range + place(id)); }
};
Split split_of(int V) {
    int shift = kSortShift;
    const auto range = [&] { return (int)(((int64_t)V + (1 << shift) - 1) >> shift); };
    while (range() > kMaxRange) ++shift;
    return {range(), shift};
}
Split small_split_of(int V) { return {(int)(((int64_t)V + (1 << kSortShift) - 1) >> kSortShift), kSortShift}; } // of any range
constexpr int kBlock = 64 * kAhead; // tokens of a wave that are requested at once
constexpr size_t kSortLds = 159744; // LDS of the lists and counts: a CU's, less what is declared

// orders a wave's own reads and writes of LDS, for the compiler: the instructions themselves take place in order
__device__ inline void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// ONCE: a wave has kBlock tokens at most, requested before anything else.  `room`: tokens that a wave's list holds, kBlock at least.  A wave whose
// part of the range is longer counts each list that is full and starts another; it goes through its ids again to place them.
template <int WIDE, int ONCE>
__global__ __launch_bounds__(kSortWaves * 64) void embed_sort_kernel(const void* __restrict__ ids, int T, int V, Split split, int bits, int room,
                                                                     Sorted out) {
    extern __shared__ int lds[];
    const int range = split.range;
    __shared__ int sums[kSortWaves], below_all[kSortWaves];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const uint64_t lanes_below = (1ull << lane) - 1;
    int* hist = lds + kSortWaves * room; // [kSortWaves][range]: a wave's tokens of each id, then where its next one goes
    int* mine = hist + wave * range;
    int* list = lds + wave * room;       // the wave's tokens of the range, in order: place among the wave's tokens, id's place in the range (10 bits)
    const uint32_t lo = blockIdx.x * range;
    // each wave has an unbroken piece of the tokens, of which a lane takes every 64th
    const int64_t piece = ((int64_t)T + kSortWaves * 64 - 1) / (kSortWaves * 64) * 64;
    const int64_t begin = wave * piece, end = begin + piece < T ? begin + piece : T;
    uint32_t id[kAhead], group[kAhead]; // an id outside [0, V) belongs to a workgroup behind all that there are
    auto request = [&](int64_t b) { // kAhead loads in flight: one after the other, their latency would be most of the time
        if (b >= end) { // a wave without tokens
#pragma unroll
            for (int i = 0; i < kAhead; ++i) group[i] = 0xFFFFFFFFu;
            return;
        }
        std::conditional_t<WIDE, uint64_t, uint32_t> v[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) v[i] = ((const std::conditional_t<WIDE, uint64_t, uint32_t>*)ids)[min(b + i * 64 + lane, end - 1)];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            id[i] = (uint32_t)v[i];
            group[i] = b + i * 64 + lane < end && v[i] < (uint32_t)V ? split.group(id[i]) : 0xFFFFFFFFu;
        }
    };
    int below = 0;
    auto add_to_list = [&](int& m, uint32_t at) { // of what was requested, the wave's tokens from `at` on
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            below += __popcll(__ballot(group[i] < blockIdx.x));
            const uint64_t hits = __ballot(group[i] == blockIdx.x);
            if (hits == 0) continue;
            if (group[i] == blockIdx.x) list[m + __popcll(hits & lanes_below)] = (int)((at + i * 64 + lane) << 10 | split.place(id[i]));
            m += __popcll(hits);
        }
        wave_fence(); // read by other lanes of the wave
    };
    // 64 tokens of the list at a time: a token's place is the wave's count of its id and its rank among the lanes with the same id: all of
    // them (a frequent token), or found by the bits of the id
    auto take_list = [&](int m, bool write) {
        for (int g = 0; g < m; g += 64) {
            const bool live = g + lane < m;
            const uint32_t entry = list[g + lane < m ? g + lane : g];
            const int k = entry & 1023;
            uint64_t peers = __ballot(live);
            if (__ballot(live && k == __builtin_amdgcn_readfirstlane(k)) != peers)
                for (int j = 0; j < bits; ++j) {
                    const uint64_t set = __ballot((k >> j) & 1);
                    peers &= (k >> j) & 1 ? set : ~set;
                }
            const int rank = __popcll(peers & lanes_below), at = mine[k] + rank;
            wave_fence(); // everyone's count is read before it is raised
            if (live) {
                if (write) {
                    out.order[at] = (int)(begin + (entry >> 10));
                    out.ids[at] = (int)split.id(blockIdx.x, k);
                }
                if (rank == 0) mine[k] = at + __popcll(peers);
            }
            wave_fence();
        }
    };
    int listed = 0;
    bool again = false; // the list does not hold them all
    if (ONCE) request(begin);
    for (int i = tid; i < kSortWaves * range; i += kSortWaves * 64) hist[i] = 0;
    __syncthreads();
    for (int64_t b = begin; b < end; b += kBlock) {
        if (!ONCE) {
            request(b);
            if (listed > room - kBlock) {
                take_list(listed, false);
                listed = 0, again = true;
            }
        }
        add_to_list(listed, (uint32_t)(b - begin));
    }
    take_list(listed, false);
    if (lane == 0) below_all[wave] = below;
    __syncthreads();
    // an id per thread (kMaxRange <= threads): its tokens, then exclusive sums over the ids before it
    int total = 0;
    if (tid < range)
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) total += hist[w * range + tid];
    int before = total;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        const int v = __shfl_up(before, s, 64);
        if (lane >= s) before += v;
    }
    if (lane == 63) sums[wave] = before;
    __syncthreads();
    int at = before - total;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) at += below_all[w] + (w < wave ? sums[w] : 0);
    if (tid < range) {
        out.start[lo + tid] = at;
        if (lo + tid == split.keys() - 1) out.start[split.keys()] = at + total;
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) {
            const int c = hist[w * range + tid];
            hist[w * range + tid] = at;
            at += c;
        }
    }
    __syncthreads();
    if (ONCE || !again) {
        take_list(listed, true);
        return;
    }
    listed = 0;
    for (int64_t b = begin; b < end; b += kBlock) {
        request(b);
        if (listed > room - kBlock) {
            take_list(listed, true);
            listed = 0;
        }
        add_to_list(listed, (uint32_t)(b - begin));
    }
    take_list(listed, true);
}

struct EmbedBwd {
    const void* dY;
    void* dE;
    Sorted s;
    Split split;
    float* part; // [chunks][2][d]: of a row that starts in an earlier chunk, of one that goes on in the next
    int T, V, d, chunks, slabs;
    float scale;
};

// What a lane has of a row in a slab of 64 pieces: a piece, and where rows have values behind their whole pieces, in the first slab, one
// of those
template <int BF16, int TAIL>
struct Lane {
    typedef Row<BF16> Rw;
    typedef typename Rw::Elem Elem;
    static constexpr int N = Rw::N, M = N + TAIL;
    int e, whole, et;
    bool tail;
    __device__ Lane(int d, int slab, int lane)
        : e((slab * 64 + lane) * N), whole(Rw::whole(d)), et(whole + lane), tail(TAIL && slab == 0 && et < d) {}

    __device__ void write(const EmbedBwd& a, int id, const float (&acc)[M]) const {
        Elem* row = (Elem*)a.dE + (int64_t)id * a.d;
        float v[N];
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = acc[k] * a.scale;
        Rw::store(row, e, whole, Rw::pack(v));
        if constexpr (TAIL)
            if (tail) Rw::put(row + et, acc[N] * a.scale);
    }
    // a row of partial sums
    __device__ void write_part(float* row, const float (&acc)[M]) const {
        if (e < whole)
#pragma unroll
            for (int k = 0; k < N; ++k) row[e + k] = acc[k];
        if constexpr (TAIL)
            if (tail) row[et] = acc[N];
    }
    __device__ void read_part(const float* row, float (&v)[M]) const {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = e < whole ? row[e + k] : 0.f;
        if constexpr (TAIL) v[N] = tail ? row[et] : 0.f;
    }
};

// A workgroup has a chunk of the sorted tokens, a wave a piece of it, or kClear rows of dE for each wave to clear; and a slab of 64 pieces of
// the columns.  What a wave has of a row that starts in an earlier one goes through LDS to the wave that has its start, and to memory
// only where that lies in another chunk.
//
// Piece: the wave's sorted tokens: lane i < cnt has token `tok` of row `id`; `prev` and `next`: the rows of the tokens before and behind
// them, -1 where there are none.
struct Piece {
    int tok, id, cnt, prev, next;
};
template <int BF16, int TAIL, int WAVES>
struct Chunk {
    static constexpr int N = Row<BF16>::N, M = N + TAIL;
    float heads[WAVES][M][64];
    int head_of[WAVES]; // 0: the wave starts with a row of its own; 1: its first row started earlier, 2: and goes on

    // goes_on(sum): of a row that starts here and does not end here; came(sum, ends): of the one that started in an earlier chunk.  One wave at
    // most calls each.
    template <class On, class Came>
    __device__ void sum(const EmbedBwd& a, const Lane<BF16, TAIL>& mine, const Piece& p, int wave, int lane, On&& goes_on, Came&& came) {
        typedef Row<BF16> Rw;
        typedef typename Rw::Elem Elem;
        float acc[M] = {};
        bool own = p.prev < 0 || __builtin_amdgcn_readlane(p.id, 0) != p.prev; // the row at hand starts in this piece
        int head = 0, tail = -1; // tail: the row that starts here and goes on; acc is its sum then
        u32x4 w[kPiece];
        float wt[kPiece];
#pragma unroll
        for (int j = 0; j < kPiece; ++j) {
            w[j] = u32x4{0, 0, 0, 0}, wt[j] = 0.f;
            if (j < p.cnt) {
                const Elem* row = (const Elem*)a.dY + (int64_t)__builtin_amdgcn_readlane(p.tok, j) * a.d;
                w[j] = Rw::load(row, mine.e, mine.whole);
                if constexpr (TAIL)
                    if (mine.tail) wt[j] = Rw::one(row + mine.et);
            }
        }
#pragma unroll
        for (int j = 0; j < kPiece; ++j) {
            if (j < p.cnt) {
                float v[N];
                Rw::unpack(w[j], v);
#pragma unroll
                for (int k = 0; k < N; ++k) acc[k] += v[k];
                if constexpr (TAIL) acc[N] += wt[j];
                const int row = __builtin_amdgcn_readlane(p.id, j);
                const int after = j == p.cnt - 1 ? p.next : __builtin_amdgcn_readlane(p.id, (j + 1) % kPiece);
                if (j == p.cnt - 1 && row == after && own) {
                    tail = row;
                } else if (j == p.cnt - 1 || row != after) {
                    if (own) {
                        mine.write(a, row, acc);
                    } else {
                        head = row == after ? 2 : 1;
#pragma unroll
                        for (int k = 0; k < M; ++k) heads[wave][k][lane] = acc[k];
                    }
                    own = true;
#pragma unroll
                    for (int k = 0; k < M; ++k) acc[k] = 0.f;
                }
            }
        }
        if (lane == 0) head_of[wave] = head;
        __syncthreads();
        // adds what the waves from `from` on have of a row that goes on in them; whether it ends there
        auto follow = [&](float (&s)[M], int from) {
            const uint64_t ends = __ballot(lane >= from && lane < WAVES && head_of[lane % WAVES] != 2);
            const int last = ends ? __builtin_ctzll(ends) : WAVES - 1;
#pragma unroll 2
            for (int u = from; u <= last; ++u)
#pragma unroll
                for (int k = 0; k < M; ++k) s[k] += heads[u][k][lane];
            return ends != 0;
        };
        if (tail >= 0) {
            if (follow(acc, wave + 1)) mine.write(a, tail, acc);
            else goes_on(acc);
        }
        if (wave == 0 && head) {
#pragma unroll
            for (int k = 0; k < M; ++k) acc[k] = heads[0][k][lane];
            const bool ends = head == 1 || follow(acc, 1);
            came(acc, ends);
        }
    }
};

template <int BF16, int TAIL>
__global__ __launch_bounds__(kSumWaves * 64) void embed_sum_kernel(EmbedBwd a) {
    __shared__ Chunk<BF16, TAIL, kSumWaves> chunk;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int64_t job = sdp::group_id() / (uint32_t)a.slabs;
    const int slab = (int)(sdp::group_id() - (uint32_t)job * (uint32_t)a.slabs);
    const Lane<BF16, TAIL> mine(a.d, slab, lane);
    if (job >= a.chunks) {
        const int64_t first = ((job - a.chunks) * kSumWaves + wave) * kClear;
        if (first >= a.V) return;
        int keys[kClear];
#pragma unroll
        for (int i = 0; i < kClear; ++i) keys[i] = a.split.key((uint32_t)first + i);
        const float zeros[Lane<BF16, TAIL>::M] = {};
#pragma unroll
        for (int i = 0; i < kClear; ++i)
            if (first + i < a.V && a.s.start[keys[i]] == a.s.start[keys[i] + 1]) mine.write(a, (int)first + i, zeros);
        return;
    }
    // requested before it is known how many tokens there are: what lies behind the last one is not used
    const int p0 = (int)job * kChunk + wave * kPiece, at = min(p0 + lane, a.T - 1);
    Piece p{a.s.order[at], a.s.ids[at], 0, a.s.ids[max(min(p0, a.T) - 1, 0)], a.s.ids[min(p0 + kPiece, a.T - 1)]};
    const int n = a.s.start[a.split.keys()];
    if (job * kChunk >= n) return;
    p.cnt = max(0, min(kPiece, n - p0));
    if (p0 == 0) p.prev = -1;
    if (p0 + p.cnt >= n) p.next = -1;
    if (job > 0 && wave == 0 && slab == 0 && lane == 0) {
        // what goes on from the chunk before, if it starts there
        const int before = (int)(job - 1) * kChunk;
        const int key = a.split.key(p.id);
        a.s.spans[job - 1] = p.id == p.prev && a.s.start[key] >= before ? make_int2(p.id, (a.s.start[key + 1] - 1) / kChunk) : make_int2(-1, 0);
    }
    float* part = a.part + job * 2 * a.d;
    chunk.sum(a, mine, p, wave, lane, [&](const auto& s) { mine.write_part(part + a.d, s); }, [&](const auto& s, bool) { mine.write_part(part, s); });
}

// A batch of kSmall tokens at most, in one launch: a workgroup has a share of the ids, dealt out as in the sort, and a slab of the columns.  Its
// tokens are put in order and summed a chunk at a time; a row that goes over a chunk's end is carried in LDS.  The order comes from counting,
// for each token, those before it; where that is many, which a few ids' tokens are, from splitting by each bit in which places differ.
// One launch / three, us, bf16, frequencies as 1 / rank: 512 tokens, 1024 rows of 256 7.2 / 15.1; 1000 tokens of these 8.4 / 16.4; 1024 tokens, 32000 x 768
// 14.8 / 18.8, x 2048 24.7 / 30.6.  All tokens of one id are one workgroup's: 512 tokens 16.6 / 14.3, 1000 29.1 / 15.7.
constexpr int kSmallWaves = 16, kSmall = kSmallWaves * 64, kSmallChunk = kSmallWaves * kPiece, kCounted = 256;

template <int BF16, int TAIL>
__global__ __launch_bounds__(kSmallWaves * 64) void embed_small_kernel(EmbedBwd a, const void* ids, int wide, Split split) {
    constexpr int M = Lane<BF16, TAIL>::M;
    __shared__ Chunk<BF16, TAIL, kSmallWaves> chunk;
    __shared__ __align__(16) uint32_t key[kSmall]; // of the share's tokens: place of the id, then token; behind the last one the largest
    __shared__ uint32_t sorted[kSmall];
    __shared__ int present[kSmall];
    __shared__ int counts[2][kSmallWaves];
    __shared__ float carry[2][M][64]; // from one chunk to the next: a chunk may read one and write one
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t job = sdp::group_id() / (uint32_t)a.slabs;
    if (job >= (uint32_t)split.groups()) return;
    const Lane<BF16, TAIL> mine(a.d, (int)(sdp::group_id() - job * (uint32_t)a.slabs), lane);
    // where a wave's lanes with `bit` go among those of all waves; `all`: how many there are
    auto among = [&](bool bit, int turn, int& all) {
        const uint64_t set = __ballot(bit);
        if (lane == 0) counts[turn][wave] = __popcll(set);
        __syncthreads();
        int before = 0;
        all = 0;
#pragma unroll
        for (int w = 0; w < kSmallWaves; ++w) before += w < wave ? counts[turn][w] : 0, all += counts[turn][w];
        return before + __popcll(set & ((1ull << lane) - 1));
    };
    const int id = tid < a.T ? sdp::token_id(ids, wide, tid, a.V) : -1;
    const bool held = id >= 0 && split.group(id) == job;
    int m;
    const int at = among(held, 0, m);
    if (held) key[at] = split.place(id) << 10 | tid;
    if (tid < (-m & 3)) key[m + tid] = 0xFFFFFFFFu;
    __syncthreads();
    if (m <= kCounted) {
        if (tid < m) {
            const uint32_t own = key[tid];
            int rank = 0;
#pragma unroll 4
            for (int j = 0; j < m; j += 4) {
                const u32x4 k = *(const u32x4*)(key + j);
                rank += (k[0] < own) + (k[1] < own) + (k[2] < own) + (k[3] < own);
            }
            sorted[rank] = own;
        }
    } else {
        uint32_t own = tid < m ? key[tid] : 0, differ = tid < m ? own ^ key[0] : 0;
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) differ |= __shfl_xor(differ, s, 64);
        if (lane == 0) counts[1][wave] = (int)differ;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kSmallWaves; ++w) differ |= (uint32_t)counts[1][w];
        int turn = 0; // counts[0] was read before a barrier, counts[1] is free once a bit was split by
        for (int b = 10; b < 32; ++b) {
            if (!(__builtin_amdgcn_readfirstlane(differ) >> b & 1)) continue;
            const bool low = tid < m && !(own >> b & 1);
            int lows;
            const int l = among(low, turn, lows);
            if (tid < m) key[low ? l : lows + tid - l] = own;
            __syncthreads();
            own = tid < m ? key[tid] : 0;
            turn ^= 1;
        }
        if (tid < m) sorted[tid] = own;
    }
    __syncthreads();
    auto row_of = [&](int i) { return (int)split.id(job, sorted[i] >> 10); };
    // Rows that do not occur, of an unbroken range of split.range of them: memory is faster written in its order (256 tokens, 32000 x 2048 bf16
    // 24.2 us, 25.6 where a workgroup clears rows of its share).  `present`: the tokens whose ids lie there.
    const int lo = (int)job * split.range;
    int n;
    const bool in = id >= lo && id - lo < split.range;
    const int place = among(in, 1, n);
    if (in) present[place] = id - lo;
    __syncthreads();
    const float zeros[M] = {};
    for (int v = wave; v < min(split.range, a.V - lo); v += kSmallWaves) {
        bool occurs = false;
        for (int i = lane; i < n; i += 64) occurs |= present[i] == v;
        if (__ballot(occurs) == 0) mine.write(a, lo + v, zeros);
    }
    for (int c0 = 0; c0 < m; c0 += kSmallChunk) {
        const int p0 = c0 + wave * kPiece, cnt = max(0, min(kPiece, m - p0)), i = min(p0 + lane, m - 1), turn = c0 / kSmallChunk & 1;
        const Piece p{(int)(sorted[i] & 1023), row_of(i), cnt, p0 > 0 && cnt ? row_of(p0 - 1) : -1, p0 + cnt < m ? row_of(p0 + cnt) : -1};
        auto put = [&](const float (&s)[M]) {
#pragma unroll
            for (int k = 0; k < M; ++k) carry[turn ^ 1][k][lane] = s[k];
        };
        chunk.sum(a, mine, p, wave, lane, put, [&](float (&s)[M], bool ends) {
#pragma unroll
            for (int k = 0; k < M; ++k) s[k] += carry[turn][k][lane];
            if (ends) mine.write(a, row_of(c0), s);
            else put(s);
        });
        if (c0 + kSmallChunk < m) __syncthreads(); // before the next chunk's sums take the place of this one's
    }
}

// A workgroup looks at a chunk and a slab: if a row starts there and goes on, it adds up the row's partial sums.  Each wave adds every
// fourth chunk's, in their order, and the waves' sums follow in theirs.
template <int BF16, int TAIL>
__global__ __launch_bounds__(256) void embed_join_kernel(EmbedBwd a) {
    constexpr int M = Lane<BF16, TAIL>::M, B = 4;
    __shared__ float lds[4][M][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int64_t job = sdp::group_id() / (uint32_t)a.slabs;
    if (job >= a.chunks - 1) return;
    const Lane<BF16, TAIL> mine(a.d, (int)(sdp::group_id() - (uint32_t)job * (uint32_t)a.slabs), lane);
    const int n = a.s.start[a.split.keys()];
    const int2 span = a.s.spans[job]; // written by the sums of the next chunk, where that has a token
    if ((job + 1) * kChunk >= n || span.x < 0) return;
    float acc[M] = {};
    // the row's parts: of chunk `job`, then of those up to span.y
    for (int64_t c = job + wave; c <= span.y; c += 4 * B) {
        float v[B][M] = {};
#pragma unroll
        for (int j = 0; j < B; ++j) {
            const int64_t at = c + 4 * j;
            if (at <= span.y) mine.read_part(a.part + (at * 2 + (at == job)) * a.d, v[j]);
        }
#pragma unroll
        for (int j = 0; j < B; ++j)
#pragma unroll
            for (int k = 0; k < M; ++k) acc[k] += v[j][k]; // zeros behind the last
    }
#pragma unroll
    for (int k = 0; k < M; ++k) lds[wave][k][lane] = acc[k];
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int k = 0; k < M; ++k) acc[k] = ((lds[0][k][lane] + lds[1][k][lane]) + lds[2][k][lane]) + lds[3][k][lane];
    mine.write(a, span.x, acc);
}

int check_embed(int dtype, int id_type, int T, int V, int d) {
    if (dtype != SDP_F32 && dtype != SDP_BF16) return SDP_ERR_INVALID_ARG;
    if (id_type != SDP_I32 && id_type != SDP_I64) return SDP_ERR_INVALID_ARG;
    if (T < 0 || V < 1 || d < 1) return SDP_ERR_INVALID_ARG;
    return T > SDP_EMBED_MAX_TOKENS || V > SDP_MAX_EXTENT || d > SDP_MAX_EXTENT ? SDP_ERR_SHAPE : SDP_OK;
}

int chunks_of(int T) { return (int)(((int64_t)T + kChunk - 1) / kChunk); }
int slabs_of(int dtype, int d) { // one of a row of less than a piece, which is all tail
    const int s = dtype == SDP_BF16 ? (Row<1>::whole(d) + 511) / 512 : (Row<0>::whole(d) + 255) / 256;
    return s > 0 ? s : 1;
}

struct Layout {
    size_t ids, start, spans, part, all;
};
Layout layout(int T, int V, int d) {
    Layout l;
    l.ids = sdp::round_up((size_t)T * 4, 256);
    l.start = 2 * l.ids;
    l.spans = l.start + sdp::round_up(((size_t)split_of(V).keys() + 1) * 4, 256);
    l.part = l.spans + sdp::round_up((size_t)chunks_of(T) * sizeof(int2), 256);
    l.all = l.part + sdp::round_up((size_t)chunks_of(T) * 2 * d * sizeof(float), 256);
    return l;
}

} // namespace

extern "C" int sdp_embed_fwd(int dtype, int id_type, int T, int V, int d, float scale, const void* E, const void* ids, void* Y,
                             void* stream) {
    const int rc = check_embed(dtype, id_type, T, V, d);
    if (rc != SDP_OK) return rc;
    if (!std::isfinite(scale)) return SDP_ERR_INVALID_ARG;
    if (T == 0) return SDP_OK;
    const size_t es = dtype == SDP_BF16 ? 2 : 4, is = id_type == SDP_I64 ? 8 : 4;
    if (!E || !ids || !Y || !sdp::aligned_to(E, es) || !sdp::aligned_to(Y, es) || !sdp::aligned_to(ids, is)) return SDP_ERR_INVALID_ARG;
    if (sdp::overlap({{Y, (size_t)T * d * es}}, {{E, (size_t)V * d * es}, {ids, (size_t)T * is}})) return SDP_ERR_INVALID_ARG;
    hipStream_t s = (hipStream_t)stream;
    const EmbedFwd a{E, ids, Y, T, V, d, id_type == SDP_I64, scale};
    sdp::ProfileScope ps("embed_fwd", s);
    const dim3 groups = sdp::grid_of(((int64_t)T + 3) / 4);
    if (dtype == SDP_BF16) embed_fwd_kernel<1><<<groups, 256, 0, s>>>(a);
    else embed_fwd_kernel<0><<<groups, 256, 0, s>>>(a);
    return sdp::launch_status();
}

extern "C" size_t sdp_embed_bwd_workspace_bytes(int dtype, int T, int V, int d) {
    if (check_embed(dtype, SDP_I32, T, V, d) != SDP_OK) return 0;
    return layout(T, V, d).all;
}

extern "C" int sdp_embed_bwd(int dtype, int id_type, int T, int V, int d, float scale, const void* dY, const void* ids, void* dE,
                             void* ws, size_t ws_bytes, void* stream) {
    const int rc = check_embed(dtype, id_type, T, V, d);
    if (rc != SDP_OK) return rc;
    if (!std::isfinite(scale)) return SDP_ERR_INVALID_ARG;
    const size_t es = dtype == SDP_BF16 ? 2 : 4, is = id_type == SDP_I64 ? 8 : 4;
    if (!dE || (T > 0 && (!dY || !ids))) return SDP_ERR_INVALID_ARG;
    EmbedBwd a{dY, dE, {}, split_of(V), nullptr, T, V, d, chunks_of(T), slabs_of(dtype, d), scale};
    const int64_t sum = ((int64_t)a.chunks + ((int64_t)V + kSumWaves * kClear - 1) / (kSumWaves * kClear)) * a.slabs;
    const int64_t join = (int64_t)(a.chunks - 1) * a.slabs;
    if (sum > UINT32_MAX) return SDP_ERR_SHAPE; // workgroups; no memory holds such a dE
    if (!sdp::aligned_to(dE, es) || !sdp::aligned_to(dY, es) || !sdp::aligned_to(ids, is)) return SDP_ERR_INVALID_ARG;
    if (T > 0 && sdp::overlap({{dE, (size_t)V * d * es}}, {{dY, (size_t)T * d * es}, {ids, (size_t)T * is}})) return SDP_ERR_INVALID_ARG;
    const Layout l = layout(T, V, d);
    if (!ws || !sdp::aligned16(ws) || ws_bytes < l.all) return SDP_ERR_WORKSPACE;
    hipStream_t s = (hipStream_t)stream;
    char* w = (char*)ws;
    a.s = {(int32_t*)w, (int32_t*)(w + l.ids), (int32_t*)(w + l.start), (int2*)(w + l.spans)};
    a.part = (float*)(w + l.part);
    sdp::ProfileScope ps("embed_bwd", s);
    const auto by_form = [&](auto&& go) {
        auto of = [&](auto bf16) {
            return d % Row<bf16.value>::N ? go(bf16, std::integral_constant<int, 1>{}) : go(bf16, std::integral_constant<int, 0>{});
        };
        return dtype == SDP_BF16 ? of(std::integral_constant<int, 1>{}) : of(std::integral_constant<int, 0>{});
    };
    if (T <= kSmall) {
        const Split share = small_split_of(V);
        const dim3 groups = sdp::grid_of((int64_t)share.groups() * a.slabs);
        return by_form([&](auto bf16, auto tail) {
            embed_small_kernel<bf16.value, tail.value><<<groups, kSmallWaves * 64, 0, s>>>(a, ids, id_type == SDP_I64, share);
            return sdp::launch_status();
        });
    }
    const int range = a.split.range;
    int bits = 0;
    while ((1 << bits) < range) ++bits;
    // one block's list for the shorter batches, so that two workgroups share a CU; else all that the counts leave
    const int room = T <= kSortWaves * kBlock ? kBlock : (int)(kSortLds / (kSortWaves * sizeof(int))) - range;
    const size_t lds = (size_t)kSortWaves * (room + range) * sizeof(int);
    auto sort = [&](auto wide, auto once) {
        const auto kern = embed_sort_kernel<wide.value, once.value>;
        static const hipError_t attr =
            hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)kSortLds);
        if (attr != hipSuccess) return sdp::hip_status(attr);
        kern<<<a.split.groups(), kSortWaves * 64, lds, s>>>(ids, T, V, a.split, bits, room, a.s);
        return sdp::launch_status();
    };
    auto sort_of = [&](auto wide) {
        return T <= kSortWaves * kBlock ? sort(wide, std::integral_constant<int, 1>{}) : sort(wide, std::integral_constant<int, 0>{});
    };
    if (const int st = id_type == SDP_I64 ? sort_of(std::integral_constant<int, 1>{}) : sort_of(std::integral_constant<int, 0>{}); st != SDP_OK)
        return st;
    return by_form([&](auto bf16, auto tail) {
        embed_sum_kernel<bf16.value, tail.value><<<sdp::grid_of(sum), kSumWaves * 64, 0, s>>>(a);
        const int rc = sdp::launch_status();
        if (rc != SDP_OK || a.chunks < 2) return rc;
        embed_join_kernel<bf16.value, tail.value><<<sdp::grid_of(join), 256, 0, s>>>(a);
        return sdp::launch_status();
    });
}
