// The output head and its loss in one: logits Z = X W^T of the tokens that have a target, their loss, dX = dZ W and dW = dZ^T X, without Z.
//
// 6 T V d operations, three contractions of the same size, with [T][V] between them.  Bound by the matrix cores as soon as tokens are some
// hundreds; by reading W and writing dW for a few.  The logits exist for a piece of tokens at a time, as large as SDP_HEAD_PIECE_BYTES: all V
// columns of it are there before anything goes on, so that no contraction is done twice (pieces of the vocabulary would need the first one
// again behind the softmax: 8 T V d).  A piece:
//   gather   rows of X of its tokens, side by side; tokens without a target are left out, at the cost of a copy of X (one part in
//            thousands of the contractions' time)
//   logits   bf16: the contraction's epilogue takes each block's maximum and sum in fp32 and keeps a logit as 16 bits (kCodeRange)
//   rows     a row's blocks -> its lse and loss; its codes -> its gradient, bf16, in their place.  4 bytes a logit moved beside 6 d operations
//   dX, dW   contractions on what is stored; dW goes on from piece to piece in fp32 (head.sums), and is rounded once
// fp32: the same with the logits themselves in fp32 (target_rows) and the fp32 contractions, over all tokens, of which those without a target are rows of
// zeros: nothing waits for their number then (a list's launch less: 1023 x 5003 x 511 184 -> 180 us).
#include <cmath>

#include "sdp_internal.h"
#include "sdp_loss_rows.h"
#include "sdp_rows.h"
#include "sdp_targets.h"

namespace {

using sdp::Row;
using sdp::Targets;
using sdp::u32x4;

// tokens of a turn in the list's kernel: 16 a thread
constexpr int kListTurn = 1024 * 16;

// whether a token has an entry; a wave a token
__global__ __launch_bounds__(256) void entries_kernel(Targets t, int T, int V, uint8_t* __restrict__ has) {
    const int64_t token = (int64_t)sdp::group_id() * 4 + (threadIdx.x >> 6);
    if (token >= T) return;
    const bool any = sdp::has_entry(t, token, V);
    if ((threadIdx.x & 63) == 0) has[token] = any;
}

// The sizes that the pieces' contractions are planned from
struct Shapes {
    sdp::HeadTiles dx, dw;
    int rows, pieces, V, d;
};

// by a whole wave
__device__ inline void plan_piece(const Shapes& g, int rows, sdp::HeadPiece* to) {
    auto tiles = [](const sdp::HeadTiles& t, int m, int n) { return ((m + t.bm - 1) / t.bm) * ((n + t.bn - 1) / t.bn); };
    const bool two = rows <= sdp::kTwoTermRows; // dX's cut tiles have room for them
    const int held = two ? 2 * rows : rows;
    const sdp::HeadCut dx = sdp::head_cut(g.dx, tiles(g.dx, held, g.d), (g.V + 63) / 64, two);
    const sdp::HeadCut dw = sdp::head_cut(g.dw, tiles(g.dw, g.V, g.d), (held + 63) / 64);
    if ((threadIdx.x & 63) == 0) *to = {rows, two ? 2 : 1, {}, dx, dw};
}

// list: the tokens with a target in order, from its front; the others as -1 - token, from its end.  pieces: what each of them has of the former.
// One workgroup: 16384 tokens are one turn.  FROM: 0, 1 labels of 32, 64 bits, 2 what entries_kernel wrote.
template <int FROM>
__global__ __launch_bounds__(1024) void list_kernel(const void* __restrict__ from, int T, int V, int32_t* __restrict__ list, sdp::HeadPiece* pieces, Shapes g) {
    __shared__ int wave_sums[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int before = 0; // tokens with a target in earlier turns
    for (int64_t t0 = 0; t0 < T; t0 += kListTurn) {
        // a wave's 1024 tokens, 64 at a time: loads without conditions
        const int64_t first = t0 + wave * 1024 + lane;
        bool has[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int64_t t = first + 64 * i < T ? first + 64 * i : T - 1;
            if constexpr (FROM == 2) has[i] = ((const uint8_t*)from)[t] != 0;
            else has[i] = sdp::token_id<FROM>(from, t, V) >= 0;
        }
        uint64_t mask[16];
        int n = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) mask[i] = __ballot(has[i] && first + 64 * i < T), n += __popcll(mask[i]);
        if (lane == 0) wave_sums[wave] = n;
        __syncthreads();
        int at = before, all = 0;
#pragma unroll
        for (int w = 0; w < 16; ++w) {
            if (w < wave) at += wave_sums[w];
            all += wave_sums[w];
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int64_t t = first + 64 * i;
            const int mine = at + __popcll(mask[i] & ((1ull << lane) - 1)); // those with a target before token t
            if (t < T) {
                if (mask[i] >> lane & 1) list[mine] = (int32_t)t;
                else list[T - 1 - (t - mine)] = -1 - (int32_t)t;
            }
            at += __popcll(mask[i]);
        }
        before += all;
        __syncthreads();
    }
    for (int p = wave; p < g.pieces; p += 16) {
        const int left = before - p * g.rows;
        plan_piece(g, left < 0 ? 0 : left < g.rows ? left : g.rows, pieces + p);
    }
}

// The list of at most kSmallList tokens, by every workgroup of 256 threads that needs it, in its own LDS; returns how many have a target.  `has`: what
// entries_kernel wrote, null with labels.
constexpr int kSmallList = 1024;
__device__ int small_list(const void* labels, int wide, const uint8_t* has, int T, int V, int32_t* list) {
    __shared__ uint64_t masks[kSmallList / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int c = 0; c < kSmallList / 64; c += 4) {
        const int t = (c + wave) * 64 + lane;
        const int at = t < T ? t : T - 1;
        const uint64_t mask = __ballot((has ? has[at] != 0 : sdp::token_id(labels, wide, at, V) >= 0) && t < T);
        if (lane == 0) masks[c + wave] = mask;
    }
    __syncthreads();
    int before = 0;
    for (int c = 0; c * 64 < T; ++c) {
        const uint64_t mask = masks[c];
        if (c % 4 == wave) {
            const int t = c * 64 + lane, mine = before + __popcll(mask & ((1ull << lane) - 1));
            if (t < T) list[mask >> lane & 1 ? mine : T - 1 - (t - mine)] = mask >> lane & 1 ? t : -1 - t;
        }
        before += __popcll(mask);
    }
    __syncthreads();
    return before;
}

struct Gather {
    const void* X;
    void *Xc, *Xt, *dX; // Xt: may be null; dX: zeros for tokens without a target, may be null
    int64_t ldt;
    int32_t* list; // SMALL: made here, of T = rows tokens
    sdp::HeadPiece* piece;
    Shapes shapes;
    const void* labels_in;
    int wide;
    const uint8_t* has;
    int32_t* labels; // [row], -1 for none; may be null
    int rows, V, d;
};

// Rows of X in the list's order, and (bf16) the same column by column for dW, whose depth they are: read along it, they need one LDS read a
// fragment where rows need two (a depth step of 256 x 256 1.67 -> 1.45 us with one transposed operand instead of two).  A workgroup takes
// 64 tokens x 64 columns; tokens without a target are zeros.  d a multiple of 8, 16-byte aligned.  With two terms (HeadPiece) the columns behind
// the last token are those of all tokens again.  SMALL: the list and the plan of the other kernels are made here as well, a launch less.
template <int SMALL>
__global__ __launch_bounds__(256) void gather_kernel(Gather a) {
    __shared__ uint16_t tile[64][72]; // rows of 144 bytes: 16 of them start on different banks
    __shared__ int32_t small[SMALL ? kSmallList : 1];
    const int tid = threadIdx.x, r0 = blockIdx.x * 64, c0 = blockIdx.y * 64;
    const int32_t* list = a.list;
    int live, terms;
    if constexpr (SMALL) {
        live = small_list(a.labels_in, a.wide, a.has, a.rows, a.V, small);
        list = small;
        if (r0 == 0 && c0 == 0) {
            for (int i = tid; i < a.rows; i += 256) a.list[i] = small[i];
            if (tid < 64) plan_piece(a.shapes, live, a.piece);
        }
        terms = live <= sdp::kTwoTermRows ? 2 : 1;
    } else {
        live = a.piece->rows, terms = a.piece->terms;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int r = 32 * h + tid / 8, c = c0 + tid % 8 * 8;
        const int listed = r0 + r < a.rows ? list[r0 + r] : -1;
        u32x4 w = {0, 0, 0, 0};
        if (c < a.d) {
            if (r0 + r < a.rows && listed >= 0) {
                w = *(const u32x4*)((const uint16_t*)a.X + (int64_t)listed * a.d + c);
                *(u32x4*)((uint16_t*)a.Xc + (int64_t)(r0 + r) * a.d + c) = w; // read next
            } else {
                if (r0 + r < a.rows && a.dX) *(u32x4*)((uint16_t*)a.dX + (int64_t)(-1 - listed) * a.d + c) = w;
                if (r0 + r < live * terms) w = *(const u32x4*)((const uint16_t*)a.X + (int64_t)list[r0 + r - live] * a.d + c);
            }
        }
        if (a.labels && c0 == 0 && tid % 8 == 0 && r0 + r < a.rows) a.labels[r0 + r] = listed < 0 ? -1 : sdp::token_id(a.labels_in, a.wide, listed, a.V);
        if (a.Xt) *(u32x4*)&tile[r][tid % 8 * 8] = w;
    }
    if (!a.Xt) return;
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int c = 32 * h + tid / 8, r = tid % 8 * 8;
        if (c0 + c >= a.d) continue;
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = tile[r + 2 * i][c] | (uint32_t)tile[r + 2 * i + 1][c] << 16;
        *(u32x4*)((uint16_t*)a.Xt + (int64_t)(c0 + c) * a.ldt + r0 + r) = u32x4{w[0], w[1], w[2], w[3]};
    }
}

// fp32: rows of X with zeros for tokens without a target, whose products are computed all the same, in their places; list says which have one.  A wave a
// row, of any width and alignment.
struct Clean {
    const float* X;
    float *Xc, *dX; // dX: zeros for those tokens, may be null
    int32_t* list;  // of all tokens
    Targets t;
    int base, rows, V, d; // the piece's first token
};
__global__ __launch_bounds__(64) void clean_f32_kernel(Clean a) {
    typedef Row<0> Rw;
    constexpr int N = Rw::N;
    const int64_t row = sdp::group_id();
    if (row >= a.rows) return;
    const int tid = threadIdx.x, d = a.d, whole = Rw::whole(d), token = a.base + (int)row;
    const bool live = sdp::has_entry(a.t, token, a.V);
    if (tid == 0) a.list[token] = live ? token : -1 - token;
    const float* x = a.X + (int64_t)token * d;
    float *xc = a.Xc + row * d, *dx = a.dX + (int64_t)token * d;
    const u32x4 none = {0, 0, 0, 0};
    for (int e = tid * N; e < whole; e += 64 * N) {
        const u32x4 w = Rw::load_some(x, e, whole);
        if (!live && a.dX) *(Rw::Piece*)(dx + e) = none;
        *(Rw::Piece*)(xc + e) = live ? w : none;
    }
    if (whole + tid < d) {
        const float w = x[whole + tid];
        if (!live && a.dX) dx[whole + tid] = 0.f;
        xc[whole + tid] = live ? w : 0.f;
    }
}

struct EntryLogits {
    const uint16_t *X, *W; // [row][d], [V][d]
    const int32_t* list;
    Targets t;
    float* z; // [row][k]
    int rows, V, d;
    int parts; // workgroups of a row
};
// The entries' logits in fp32: a workgroup a row, of few rows several, LANES lanes four entries at a time, as few as hold a row of W: 10000 tokens of 109 entries, d = 80
// 84.7 us with 64 lanes, 34.6 with 16; 6200 of 104, d = 304 52.5 with 64, 46.4 with 32; 76 of 84, d = 832 11.9 with a workgroup a row, 4.5 with six.
template <int LANES>
__global__ __launch_bounds__(256) void entry_logits_kernel(EntryLogits a) {
    typedef Row<1> Rw;
    constexpr int GROUPS = 256 / LANES, M = 4;
    const uint32_t at = sdp::group_id();
    const int64_t row = at / (uint32_t)a.parts;
    if (row >= a.rows) return;
    const int listed = a.list[row], lane = threadIdx.x % LANES, group = (int)(at % (uint32_t)a.parts) * GROUPS + threadIdx.x / LANES, k = a.t.k;
    if (listed < 0) return;
    const uint16_t* x = a.X + row * a.d;
    for (int i0 = group * M; i0 - group % (64 / LANES) * M < k; i0 += a.parts * GROUPS * M) { // (whole waves stay for the sums)
        const uint16_t* w[M];
        float sum[M];
#pragma unroll
        for (int j = 0; j < M; ++j) {
            const int id = i0 + j < k ? sdp::token_id(a.t.ids, a.t.wide, (int64_t)listed * k + i0 + j, a.V) : -1;
            w[j] = a.W + (int64_t)(id < 0 ? 0 : id) * a.d;
            sum[j] = 0.f;
        }
        for (int e = lane * 8; e < a.d; e += LANES * 8) {
            float xv[8];
            Rw::unpack(*(const u32x4*)(x + e), xv);
#pragma unroll
            for (int j = 0; j < M; ++j) {
                float wv[8];
                Rw::unpack(*(const u32x4*)(w[j] + e), wv);
#pragma unroll
                for (int n = 0; n < 8; ++n) sum[j] = fmaf(xv[n], wv[n], sum[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < M; ++j) {
            float z = sum[j];
            if constexpr (LANES == 64) {
                z = sdp::wave_sum(z);
            } else {
#pragma unroll
                for (int d = LANES / 2; d >= 1; d >>= 1) z += __shfl_xor(z, d, 64);
            }
            if (lane == 0 && i0 + j < k) a.z[row * k + i0 + j] = z;
        }
    }
}

struct CodeRows {
    uint16_t* P; // may be null: the loss alone
    int64_t ldp;
    const float2* stats;
    int nblk, shift; // columns of a block: 1 << shift
    const float* z;  // [row][k]
    Targets t;
    const int32_t* list;
    const sdp::HeadPiece* piece;
    float *kl, *lse;
    int rows, V;
    int parts, columns; // a row is that many workgroups', of so many columns each
};

// A row of codes and its blocks' statistics -> its loss, lse and gradient.  One workgroup a row.  ONCE: around the caches, where the codes are far
// more than the 256 MB behind the L2s hold: 16384 x 32000 444 -> 396 us, but 3350 x 50001 123 -> 136.
// Few rows are several workgroups' each, of which all find the row's sum.  Many short ones are a wave's each (TH = 64): 15397 x 963 38.1 -> 17.6 us,
// 14187 x 413 33.2 -> 14.3, 6200 x 2442 22.2 -> 14.7, 2000 x 3500 12.5 -> 10.7, but 800 x 3000 7.0 -> 7.6.
template <int TH, int ONCE>
__global__ __launch_bounds__(TH) void code_rows_kernel(CodeRows a) {
    typedef Row<1> Rw;
    constexpr int WAVES = TH / 64;
    __shared__ float lds[3][2][WAVES];
    extern __shared__ unsigned char entry_lds[];
    const uint32_t group = sdp::group_id();
    const int64_t row = group / (uint32_t)a.parts;
    if (row >= a.rows) return;
    const int tid = threadIdx.x, k = a.t.k, listed = a.list[row], first = (int)(group % (uint32_t)a.parts) * a.columns;
    if (listed < 0) {
        if (tid == 0 && first == 0) {
            a.kl[-1 - listed] = 0.f;
            if (a.lse) a.lse[-1 - listed] = 0.f;
        }
        return;
    }
    const sdp::Entries en(entry_lds, k);
    const float2* stats = a.stats + row * a.nblk;
    const int piece_rows = a.P ? a.piece->rows : 0, terms = a.P ? a.piece->terms : 1;
    float vmax = en.load<TH>(a.t, listed, a.V);
    for (int i = tid; i < k; i += TH) en.z[i] = en.id[i] >= 0 ? a.z[row * k + i] : 0.f;
    const float rate = sdp::kLog2e * a.t.inv_tau;
    constexpr float kLn2 = 0.69314718055994530942f;
    float m = -INFINITY, sum = 0.f; // powers of two from here on
    for (int b = tid; b < a.nblk; b += TH) {
        const float2 s = stats[b];
        const float top = fmaxf(m, s.x), from = top == -INFINITY ? 0.f : top;
        sum = sum * __builtin_amdgcn_exp2f(m - from) + s.y * __builtin_amdgcn_exp2f(s.x - from);
        m = top;
    }
    const float mine = m;
    sdp::group_both<WAVES, true>(m, vmax, lds[0]);
    // a thread without blocks, or with nothing but -inf: 0; nothing but -inf in the whole row: NaN
    sum *= __builtin_amdgcn_exp2f(mine - m);
    float of_entries = en.sum<TH>(a.t, vmax);
    sdp::group_both<WAVES, false>(sum, of_entries, lds[1]);
    const float log_sum = logf(sum);
    float mass = 0.f, kl = 0.f;
    en.masses<TH>(a.t, listed, vmax, of_entries, [&](int i, float q, float log_q) {
        mass += q;
        if (q != 0.f) kl += q * ((log_q - fmaf(en.z[i], rate, -m) * kLn2) + log_sum);
    });
    sdp::group_both<WAVES, false>(mass, kl, lds[2]);
    if (!a.t.top_lse && mass == mass) mass = 1.f;
    if (tid == 0 && first == 0) {
        a.kl[listed] = !a.t.top && kl < 0.f ? 0.f : kl; // a label's logit that is all of its row's sum, but for roundings
        if (a.lse) a.lse[listed] = fmaf(m, kLn2, log_sum);
    }
    if (!a.P) return;
    // The gradient's factor c / tau comes in fp32 with the products' results: mass p - q is rounded by itself, which keeps a label's 1 - p, that most of a
    // row's length lies in, at the fine end of bf16's steps where p is small (1 / 3350 of it may lie anywhere: dX 2.5e-3 off instead of 2.1e-3),
    // and keeps a small factor out of bf16's range.
    const float inv = mass / sum;
    uint16_t* p = a.P + row * a.ldp;
    uint16_t* second = terms == 2 ? p + piece_rows * a.ldp : nullptr; // the second term's row
    constexpr float kStep = sdp::kCodeRange / 65535.f;
    const int all = (a.V + 7) / 8 * 8, end = min(first + a.columns, all); // codes of columns behind V say 0
    // (0 times a sum that is no number is NaN, as every other element of such a row)
    auto value = [&](uint32_t code, float from) { return (code == 65535u ? 0.f : __builtin_amdgcn_exp2f(fmaf((float)code, -kStep, from))) * inv; };
    auto turn = [&](int e, const u32x4& w, float block) {
        const float from = block - m;
        float v[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[2 * i] = value(w[i] & 0xFFFFu, from), v[2 * i + 1] = value(w[i] >> 16, from);
        if (ONCE) __builtin_nontemporal_store(Rw::pack(v), (u32x4*)(p + e));
        else *(u32x4*)(p + e) = Rw::pack(v); // read next
        if (!second) return;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] -= Rw::rounded(v[i]);
        *(u32x4*)(second + e) = Rw::pack(v);
    };
    constexpr int U = 4;
    for (int e0 = first + tid * 8; e0 < end; e0 += U * TH * 8) {
        u32x4 w[U];
        float block[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int e = min(e0 + u * TH * 8, end - 8);
            w[u] = ONCE ? __builtin_nontemporal_load((const u32x4*)(p + e)) : *(const u32x4*)(p + e);
            block[u] = stats[e >> a.shift].x;
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (e0 + u * TH * 8 < end) turn(e0 + u * TH * 8, w[u], block[u]);
    }
    // The entries' elements are written twice: the first time has to have reached memory, whichever wave it came from.
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    for (int i = tid; i < k; i += TH) {
        if (en.id[i] < first || en.id[i] >= end) continue;
        const float v = __builtin_amdgcn_exp2f(fmaf(en.z[i], rate, -m)) * inv - en.all_of(i, k);
        Rw::put(p + en.id[i], v);
        if (second) Rw::put(second + en.id[i], v - Rw::rounded(v));
    }
}

// Depth ranges of fp32 dX, whose outputs are few and whose depth is the vocabulary: a launch of few tiles runs as up to four problems.  1023 x 511, 5003
// deep 97 -> 53 us, and 6 for their sums.
int f32_dx_ranges(int rows, int V, int d) {
    const int64_t tiles = (int64_t)((rows + 63) / 64) * ((d + 63) / 64);
    int r = tiles > 0 && tiles <= 256 ? (int)(512 / tiles) : 1;
    r = r > sdp::kMaxBatch ? sdp::kMaxBatch : r;
    while (r > 1 && V / r < 512) --r;
    return r;
}
// their sums, in their order, and the vocabulary's last tokens, which no range has -> the tokens' rows; a workgroup a row
__global__ __launch_bounds__(256) void f32_dx_sum_kernel(const float* __restrict__ part, int ranges, int rows, int d, const float* __restrict__ Z, int64_t ldz,
                                                         const float* __restrict__ W, int first, int V, const int32_t* __restrict__ list, float* dX,
                                                         sdp::HeadLoss loss) {
    const int64_t row = (int64_t)sdp::group_id() - 1;
    if (row < 0) sdp::sum_loss(loss);
    if (row < 0 || row >= rows) return;
    const int token = list[row];
    if (token < 0) return; // zeros are there
    for (int c = threadIdx.x; c < d; c += 256) {
        float of[sdp::kMaxBatch];
#pragma unroll
        for (int r = 0; r < sdp::kMaxBatch; ++r) of[r] = part[((int64_t)min(r, ranges - 1) * rows + row) * d + c];
        float x = of[0];
#pragma unroll
        for (int r = 1; r < sdp::kMaxBatch; ++r) x += r < ranges ? of[r] : 0.f;
#pragma unroll 4
        for (int v = first; v < V; ++v) x = fmaf(Z[row * ldz + v], W[(int64_t)v * d + c], x);
        dX[(int64_t)token * d + c] = x;
    }
}

__global__ __launch_bounds__(256) void zero_kernel(uint16_t* p, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += 4096 * 256) p[i] = 0;
}

// What a call needs, and where it lies in the workspace
struct Plan {
    int rows = 0, pieces = 0, block = 0, nblk = 0; // tokens of a piece; columns of a statistic's block
    int64_t ldz = 0;                               // of the codes, or of the fp32 logits
    int64_t ldt = 0;
    sdp::HeadTiles tx{}, tw{};
    size_t list = 0, piece = 0, has = 0, X = 0, Xt = 0, Z = 0, stats = 0, labels = 0, z = 0, sums = 0, cut = 0, bytes = 0;
};
Plan plan(int dtype, int T, int V, int d, int k, bool teacher, bool dx, bool dw) {
    Plan p;
    const bool bf16 = dtype == SDP_BF16, grads = dx || dw;
    const size_t row = bf16 ? (grads ? (size_t)sdp::line_ld(V, 1) * 2 : ((size_t)V + 31) / 32 * 8) : ((size_t)V + 3) * 4;
    const size_t wide = (size_t)d * (bf16 ? 2 : 4);
    const int64_t most = (int64_t)(SDP_HEAD_PIECE_BYTES / (row > wide ? row : wide)) / 64 * 64;
    const int64_t rows_max = most < 64 ? 64 : most < SDP_HEAD_PIECE_TOKENS ? most : SDP_HEAD_PIECE_TOKENS;
    p.pieces = (int)((T + rows_max - 1) / rows_max);
    p.rows = T;
    if (p.pieces > 1) {
        p.rows = (int)(((T + p.pieces - 1) / p.pieces + 63) / 64 * 64); // equal pieces
        p.pieces = (T + p.rows - 1) / p.rows;
    }
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += sdp::round_up(bytes, 256);
        return here;
    };
    const size_t rows = (size_t)p.rows;
    p.list = take((size_t)T * 4);
    if (bf16 && teacher) p.has = take((size_t)T);
    p.X = take(rows * d * (bf16 ? 2 : 4));
    if (bf16) {
        p.ldz = sdp::line_ld(V, p.rows);
        const size_t held = (size_t)sdp::head_held(p.rows);
        p.ldt = sdp::line_ld((int64_t)held, d);
        if (dw) p.Xt = take((size_t)p.ldt * d * 2);
        p.block = sdp::head_block(p.rows, V, d), p.nblk = (V + p.block - 1) / p.block;
        if (grads) p.Z = take(held * p.ldz * 2);
        p.stats = take(rows * p.nblk * 8);
        if (!teacher) p.labels = take(rows * 4);
        p.z = take(rows * k * 4);
        p.piece = take((size_t)p.pieces * sizeof(sdp::HeadPiece));
        p.tx = sdp::head_dx_tiles(p.rows, V, d), p.tw = sdp::head_dw_tiles(p.rows, V, d, p.pieces);
        if (dw && p.pieces > 1) p.sums = take(sdp::head_sums_bytes(p.tw, V, d));
        // both contractions' cut tiles, one after the other
        const size_t bx = dx ? sdp::head_cut_bytes(p.tx) : 0, bw = dw ? sdp::head_cut_bytes(p.tw) : 0;
        p.cut = take(bx > bw ? bx : bw);
    } else {
        p.ldz = (V + 3) / 4 * 4;
        p.Z = take(rows * p.ldz * 4);
        const int r = f32_dx_ranges(p.rows, V, d);
        if (dx && r > 1) p.cut = take((size_t)r * rows * d * 4);
    }
    p.bytes = at;
    return p;
}

struct Call {
    int dtype, T, V, d;
    const void *X, *W;
    Targets t;
    float *kl, *lse;
    void *dX, *dW;
    float* loss;
};

int run(const Call& c, unsigned char* ws, hipStream_t s) {
    const bool bf16 = c.dtype == SDP_BF16, teacher = c.t.top != nullptr, grads = c.dX || c.dW;
    const Plan p = plan(c.dtype, c.T, c.V, c.d, c.t.k, teacher, c.dX, c.dW);
    int32_t* list = (int32_t*)(ws + p.list);
    sdp::HeadPiece* pieces = (sdp::HeadPiece*)(ws + p.piece); // bf16
    const Shapes shapes{p.tx, p.tw, p.rows, p.pieces, c.V, c.d};
    const bool small = p.pieces == 1 && c.T <= kSmallList; // listed by what gathers
    const bool with_loss = sdp::head_sums_loss(p.rows, p.pieces, c.dX, bf16 && c.dW);
    const sdp::HeadLoss loss{with_loss ? c.loss : nullptr, c.kl, c.T, c.t.scale, c.t.scale_dev};
    bool summed = bf16 && with_loss;
    uint8_t* has = bf16 && teacher ? ws + p.has : nullptr;
    if (has) {
        sdp::ProfileScope ps("head_entries", s);
        entries_kernel<<<sdp::grid_of((c.T + 3) / 4), 256, 0, s>>>(c.t, c.T, c.V, has);
    }
    if (bf16 && !small) {
        sdp::ProfileScope ps("head_list", s);
        if (teacher) list_kernel<2><<<1, 1024, 0, s>>>(has, c.T, c.V, list, pieces, shapes);
        else if (c.t.wide) list_kernel<1><<<1, 1024, 0, s>>>(c.t.ids, c.T, c.V, list, pieces, shapes);
        else list_kernel<0><<<1, 1024, 0, s>>>(c.t.ids, c.T, c.V, list, pieces, shapes);
    }
    int rc = sdp::launch_status();
    for (int i = 0; i < p.pieces && rc == SDP_OK; ++i) {
        const int base = i * p.rows, rows = c.T - base < p.rows ? c.T - base : p.rows;
        Gather g{c.X, ws + p.X, c.dW && bf16 ? ws + p.Xt : nullptr, c.dX, p.ldt, list + base, pieces + i, shapes, c.t.ids, c.t.wide, has, nullptr, rows, c.V, c.d};
        if (bf16 && !teacher) g.labels = (int32_t*)(ws + p.labels);
        {
            sdp::ProfileScope ps("head_gather", s);
            const dim3 grid((sdp::head_held(rows) + 63) / 64, (c.d + 63) / 64);
            if (!bf16) clean_f32_kernel<<<sdp::grid_of(rows), 64, 0, s>>>({(const float*)c.X, (float*)(ws + p.X), (float*)c.dX, list, c.t, base, rows, c.V, c.d});
            else if (small) gather_kernel<1><<<grid, 256, 0, s>>>(g);
            else gather_kernel<0><<<grid, 256, 0, s>>>(g);
        }
        rc = sdp::launch_status();
        if (rc != SDP_OK) return rc;
        if (bf16) {
            sdp::HeadGemm h;
            // p.rows, of the last piece as well: its tiles, statistics and sums lie as those that the plan is made for
            h.X = ws + p.X, h.W = c.W, h.P = ws + p.Z, h.ldp = p.ldz, h.rows = p.rows, h.V = c.V, h.d = c.d, h.piece = pieces + i;
            h.Xt = ws + p.Xt, h.ldt = p.ldt;
            h.scale = c.t.scale * c.t.inv_tau, h.scale_dev = c.t.scale_dev;
            float2* stats = (float2*)(ws + p.stats);
            float* z = (float*)(ws + p.z);
            if (teacher) {
                sdp::ProfileScope ps("head_entry_logits", s);
                const int lanes = c.d <= 128 ? 16 : c.d <= 512 ? 32 : 64, at_once = 256 / lanes * 4;
                const EntryLogits e{(const uint16_t*)h.X, (const uint16_t*)c.W, list + base, c.t, z, rows, c.V, c.d, rows < 512 ? (c.t.k + at_once - 1) / at_once : 1};
                const dim3 grid = sdp::grid_of((int64_t)rows * e.parts);
                if (lanes == 16) entry_logits_kernel<16><<<grid, 256, 0, s>>>(e);
                else if (lanes == 32) entry_logits_kernel<32><<<grid, 256, 0, s>>>(e);
                else entry_logits_kernel<64><<<grid, 256, 0, s>>>(e);
            }
            rc = sdp::gemm_head_logits(h, sdp::kLog2e * c.t.inv_tau, grads, stats, p.nblk, g.labels, z, s);
            if (rc != SDP_OK) return rc;
            const int columns = rows < 512 ? 8192 : (c.V + 7) / 8 * 8, parts = grads ? (c.V + columns - 1) / columns : 1;
            const CodeRows r{grads ? (uint16_t*)h.P : nullptr, p.ldz, stats, p.nblk, p.block == 64 ? 6 : 5, z, c.t, list + base, pieces + i, c.kl, c.lse, rows, c.V,
                             parts, columns};
            {
                sdp::ProfileScope ps("head_rows", s);
                const size_t lds = sdp::Entries::bytes(c.t.k);
                const dim3 grid = sdp::grid_of((int64_t)rows * parts);
                if (grads && (size_t)rows * p.ldz * 2 >= (size_t)1 << 29) code_rows_kernel<256, 1><<<grid, 256, lds, s>>>(r);
                else if (rows < 1024 || c.V > 4096) code_rows_kernel<256, 0><<<grid, 256, lds, s>>>(r);
                else code_rows_kernel<64, 0><<<grid, 64, lds, s>>>(r);
            }
            rc = sdp::launch_status();
            h.loss = loss;
            const bool few = c.dX && c.dW && sdp::head_dw_few(p.rows, p.pieces);
            if (rc == SDP_OK && c.dX) rc = sdp::gemm_head_dx(h, list + base, c.dX, (float*)(ws + p.cut), few ? c.dW : nullptr, s);
            if (rc == SDP_OK && c.dW && !few)
                rc = sdp::gemm_head_dw(h, c.dW, (float*)(ws + p.sums), p.pieces == 1 ? 0 : i == 0 ? 1 : i == p.pieces - 1 ? 3 : 2, (float*)(ws + p.cut), s);
            continue;
        }
        sdp::GemmDesc d;
        d.M = rows, d.N = c.V, d.K = c.d, d.A = ws + p.X, d.lda = c.d, d.B = c.W, d.ldb = c.d, d.C = ws + p.Z, d.ldc = p.ldz, d.name = "head_logits";
        rc = sdp::gemm_f32(d, s);
        if (rc != SDP_OK) return rc;
        sdp::TargetRows of;
        of.Z = ws + p.Z, of.dZ = grads ? ws + p.Z : nullptr, of.ldz = p.ldz, of.t = c.t, of.kl = c.kl, of.lse = c.lse, of.rows = rows, of.V = c.V, of.list = list + base;
        rc = sdp::target_rows(SDP_F32, of, "head_rows", s);
        sdp::GemmDesc both[2];
        sdp::GemmDesc &x = both[0], &w = both[1];
        x.M = rows, x.N = c.d, x.K = c.V, x.A = ws + p.Z, x.lda = p.ldz, x.B = c.W, x.ldb = c.d, x.b_km = 1, x.C = c.dX, x.ldc = c.d;
        x.c_scatter = list + base, x.name = "head_dx";
        w.M = c.V, w.N = c.d, w.K = rows, w.A = ws + p.Z, w.lda = p.ldz, w.a_km = 1, w.B = ws + p.X, w.ldb = c.d, w.b_km = 1, w.C = c.dW, w.ldc = c.d;
        if (i > 0) w.R = c.dW, w.ldr = c.d; // the pieces before
        w.name = "head_dw";
        if (rc != SDP_OK) return rc;
        const int r = f32_dx_ranges(p.rows, c.V, c.d);
        // in one launch where dX's depth is not what takes longest: 256 x 256, 1024 deep 8.3 us, but 12 x 225, 5083 deep 38.6,
        // where dX takes 12.4 in ranges and 3.9 for their sums, with the loss, and dW 12.8; 1 x 66, 7746 deep 53.4 and 16.8, 4.0, 8.6
        rc = c.dX && c.dW && (r == 1 || c.V <= 1536) ? sdp::gemm_f32_group(both, 2, "head_dx_dw", s) : SDP_ERR_UNSUPPORTED;
        if (rc == SDP_ERR_UNSUPPORTED) {
            if (c.dX && r > 1) {
                const int depth = c.V / r / 4 * 4;
                float* part = (float*)(ws + p.cut);
                x.nbatch = r, x.K = depth, x.c_scatter = nullptr;
                for (int z = 0; z < r; ++z)
                    x.Ab[z] = (const float*)x.A + z * depth, x.Bb[z] = (const float*)x.B + (int64_t)z * depth * c.d, x.Cb[z] = part + (int64_t)z * rows * c.d;
                rc = sdp::gemm_f32(x, s);
                if (rc != SDP_OK) return rc;
                sdp::ProfileScope ps("head_dx_sum", s);
                f32_dx_sum_kernel<<<sdp::grid_of((int64_t)rows + 1), 256, 0, s>>>(part, r, rows, c.d, (const float*)(ws + p.Z), p.ldz, (const float*)c.W, r * depth, c.V,
                                                                     list + base, (float*)c.dX, loss);
                rc = sdp::launch_status();
                summed = with_loss;
            } else {
                rc = c.dX ? sdp::gemm_f32(x, s) : SDP_OK;
            }
            if (rc == SDP_OK && c.dW) rc = sdp::gemm_f32(w, s);
        }
    }
    if (rc != SDP_OK || !c.loss || summed) return rc;
    return sdp::loss_sum(c.kl, c.T, c.t.scale, c.t.scale_dev, c.loss, s);
}

bool sizes_ok(int dtype, int T, int V, int d, int k) {
    if (T > SDP_EMBED_MAX_TOKENS || V >= 1 << 22 || d > 1 << 20 || k > SDP_MAX_ENTRIES) return false;
    if ((int64_t)V * d >= (int64_t)1 << 31) return false;
    return dtype != SDP_BF16 || d % 8 == 0;
}
size_t workspace(int dtype, int T, int V, int d, int k, bool teacher, bool dx, bool dw) {
    if ((dtype != SDP_F32 && dtype != SDP_BF16) || T < 1 || V < 1 || d < 1 || k < 1 || !sizes_ok(dtype, T, V, d, k)) return 0;
    return plan(dtype, T, V, d, k, teacher, dx, dw).bytes;
}

int head(const Call& c, int id_type, int top_dtype, float temperature, void* ws, size_t ws_bytes, void* stream) {
    const bool teacher = top_dtype >= 0;
    if ((c.dtype != SDP_F32 && c.dtype != SDP_BF16) || (id_type != SDP_I32 && id_type != SDP_I64)) return SDP_ERR_INVALID_ARG;
    if (teacher && top_dtype != SDP_F32 && top_dtype != SDP_BF16) return SDP_ERR_INVALID_ARG;
    if (c.T < 0 || c.V < 1 || c.d < 1 || c.t.k < 1 || !sdp::temperature_ok(temperature) || !std::isfinite(c.t.scale)) return SDP_ERR_INVALID_ARG;
    if (!sizes_ok(c.dtype, c.T, c.V, c.d, c.t.k)) return SDP_ERR_SHAPE;
    const bool bf16 = c.dtype == SDP_BF16;
    const size_t es = bf16 ? 2 : 4, is = id_type == SDP_I64 ? 8 : 4, ts = top_dtype == SDP_BF16 ? 2 : 4, st = (size_t)c.T * 4;
    if (!c.W || (c.T > 0 && (!c.X || !c.t.ids || (teacher && !c.t.top) || !c.kl))) return SDP_ERR_INVALID_ARG;
    for (const void* p : {c.X, c.W, (const void*)c.dX, (const void*)c.dW})
        if (!sdp::aligned_to(p, bf16 ? 16 : 4)) return SDP_ERR_INVALID_ARG;
    if (!sdp::aligned_to(c.t.ids, is) || (teacher && !sdp::aligned_to(c.t.top, ts))) return SDP_ERR_INVALID_ARG;
    for (const float* p : {c.t.top_lse, c.t.scale_dev, (const float*)c.kl, (const float*)c.lse, (const float*)c.loss})
        if (!sdp::aligned_to(p, 4)) return SDP_ERR_INVALID_ARG;
    const size_t tokens = (size_t)c.T * c.d * es, vocabulary = (size_t)c.V * c.d * es, entries = (size_t)c.T * c.t.k;
    const size_t need = workspace(c.dtype, c.T, c.V, c.d, c.t.k, teacher, c.dX, c.dW);
    const sdp::Extent eX{c.X, tokens}, eW{c.W, vocabulary}, ei{c.t.ids, entries * is}, ev{c.t.top, teacher ? entries * ts : 0},
        eL{c.t.top_lse, c.t.top_lse ? st : 0}, ec{c.t.scale_dev, c.t.scale_dev ? 4u : 0u}, on{c.kl, st}, os{c.lse, c.lse ? st : 0},
        ox{c.dX, c.dX ? tokens : 0}, ow{c.dW, c.dW ? vocabulary : 0}, o1{c.loss, c.loss ? 4u : 0u};
    if ((c.dX != c.X && sdp::overlap({ox}, {eX})) || sdp::overlap({on, os, ow, o1}, {eX}) || sdp::overlap({on, os, ox, ow, o1}, {eW, ei, ev, eL, ec}) ||
        sdp::overlap({on}, {os, ox, ow, o1}) || sdp::overlap({os}, {ox, ow, o1}) || sdp::overlap({ox}, {ow, o1}) || sdp::overlap({ow}, {o1}))
        return SDP_ERR_INVALID_ARG;
    hipStream_t s = (hipStream_t)stream;
    if (c.T == 0) {
        if (c.dW) { // no token: zeros
            zero_kernel<<<4096, 256, 0, s>>>((uint16_t*)c.dW, (int64_t)(vocabulary / 2));
            const int rc = sdp::launch_status();
            if (rc != SDP_OK) return rc;
        }
        return c.loss ? sdp::loss_sum(c.kl, 0, c.t.scale, c.t.scale_dev, c.loss, s) : SDP_OK;
    }
    if (!ws || ws_bytes < need || !sdp::aligned_to(ws, 256)) return SDP_ERR_WORKSPACE;
    const sdp::Extent scratch{ws, need};
    if (sdp::overlap({scratch}, {eX, eW, ei, ev, eL, ec, on, os, ox, ow, o1})) return SDP_ERR_INVALID_ARG;
    return run(c, (unsigned char*)ws, s);
}

} // namespace

extern "C" size_t sdp_head_loss_workspace_bytes(int dtype, int T, int V, int d, int want_dx, int want_dw) {
    return workspace(dtype, T, V, d, 1, false, want_dx, want_dw);
}

extern "C" int sdp_head_loss(int dtype, int id_type, int T, int V, int d, float scale, const void* X, const void* W, const void* labels,
                             const float* scale_dev, float* nll, float* lse, void* dX, void* dW, float* loss, void* ws, size_t ws_bytes,
                             void* stream) {
    const Call c{dtype, T, V, d, X, W, {labels, nullptr, nullptr, 1, id_type == SDP_I64, 0, 1.f, scale, scale_dev}, nll, lse, dX, dW, loss};
    return head(c, id_type, -1, 1.f, ws, ws_bytes, stream);
}

extern "C" size_t sdp_head_distill_workspace_bytes(int dtype, int T, int V, int d, int k, int want_dx, int want_dw) {
    return workspace(dtype, T, V, d, k, true, want_dx, want_dw);
}

extern "C" int sdp_head_distill(int dtype, int id_type, int top_dtype, int T, int V, int d, int k, float temperature, float scale, const void* X,
                                const void* W, const void* ids, const void* top, const float* top_lse, const float* scale_dev, float* kl,
                                float* lse, void* dX, void* dW, float* loss, void* ws, size_t ws_bytes, void* stream) {
    if (top_dtype < 0) return SDP_ERR_INVALID_ARG;
    const Call c{dtype, T, V, d, X, W, {ids, top, top_lse, k, id_type == SDP_I64, top_dtype == SDP_BF16, 1.f / temperature, scale, scale_dev},
                 kl, lse, dX, dW, loss};
    return head(c, id_type, top_dtype, temperature, ws, ws_bytes, stream);
}
