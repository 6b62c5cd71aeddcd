// Layer and root-mean-square norm of tokens, alone or of a sum with the skip connection, and the backward pass.
//
//   forward   h = x + r (rounded), mu = mean(h) (0 for the root-mean-square form), s = 1 / sqrt(mean((h - mu)^2) + eps),
//             y = (h - mu) s gamma + beta
//   backward  xh = (h - mu) s, g = dy gamma, dx = s (g - mean(g) - xh mean(g xh)) + dh (mean(g) only in the layer form),
//             dgamma = sum_t dy xh, dbeta = sum_t dy
//
// Both are bound by memory: a row is read once into registers, its sums are taken over the lanes that hold it, and it is written
// once.  A row belongs to WPR waves, each lane holding up to VPL pieces of 16 bytes (fwd_shape, bwd_shape).  16384 x 2048 bf16 with the
// skip connection, four matrices of 67 MB: forward 47.3 us, 5.7 TB/s; backward 49.1, 5.5, of which the sums of the weight's gradients
// are 4.8.  Small batches are bound by the launch: 256 x 256 fp32 forward 4.4 us, most of it the call's.
#include <cmath>
#include <type_traits>

#include "sdp_internal.h"
#include "sdp_rows.h"

namespace {

using sdp::Row;
using sdp::u32x4;

struct NormFwd {
    const void *X, *R, *gamma, *beta;
    void *H, *Y;
    float *mean, *rstd;
    int T, d, layer;
    float eps;
};

struct NormBwd {
    const void *H, *dY, *dH, *gamma;
    const float *mean, *rstd;
    void *dX, *dgamma, *dbeta;
    float* partial; // [workgroups][2][d]: dgamma, dbeta
    int T, d;
    int want_dw;
};

// waves of a workgroup in the forward pass: four rows of one wave each, or one row of four or sixteen
constexpr int waves_of(int WPR) { return WPR > 4 ? WPR : 4; }

// and in the backward pass.  us, eight / four / sixteen: 16384 x 2048 bf16 50.9 / 61.7 / 50.4, 1024 x 2048 10.9 / 11.8 / 11.4, 8192 x 2000
// 27.4 / 33.6 / 28.3, fp32 8192 x 2048 47.6 / 47.4 / 50.1; but bf16 4096 x 3200 25.7 / 25.6 / 22.6.
constexpr int kBwdWaves = 8;
constexpr int bwd_waves(int WPR) { return WPR > kBwdWaves ? WPR : WPR == 3 ? 9 : kBwdWaves; }

// Sum over the WPR waves of a row; every lane has the result.  `lds` holds one float a wave; two calls in a row need two of them.
template <int WPR>
__device__ inline float row_sum(float x, float* lds) {
    x = sdp::wave_sum(x);
    if (WPR == 1) return x;
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) lds[wave] = x;
    __syncthreads();
    const int first = wave / WPR * WPR;
    float s = lds[first];
#pragma unroll
    for (int i = 1; i < WPR; ++i) s += lds[first + i];
    return s;
}

// two sums at once
template <int WPR>
__device__ inline void row_sums(float& x, float& y, float2* lds) {
    x = sdp::wave_sum(x), y = sdp::wave_sum(y);
    if (WPR == 1) return;
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) lds[wave] = make_float2(x, y);
    __syncthreads();
    const int first = wave / WPR * WPR;
    float2 s = lds[first];
#pragma unroll
    for (int i = 1; i < WPR; ++i) s.x += lds[first + i].x, s.y += lds[first + i].y;
    x = s.x, y = s.y;
}

// FORM: rows of whole pieces, such rows read once (read_once), rows with values behind them, rows of less than a piece
constexpr int FORM_WHOLE = 0, FORM_ONCE = 1, FORM_TAIL = 2, FORM_SHORT = 3;

template <int BF16, int WPR, int VPL, int FORM>
__global__ __launch_bounds__(waves_of(WPR) * 64) void norm_fwd_kernel(NormFwd a) {
    typedef Row<BF16> Rw;
    typedef typename Rw::Elem Elem;
    constexpr int N = Rw::N, ROWS = waves_of(WPR) / WPR, STEP = WPR * 64 * N, ONCE = FORM == FORM_ONCE;
    __shared__ float lds[2][waves_of(WPR)];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int64_t row = (int64_t)sdp::group_id() * ROWS + wave / WPR;
    if (row >= a.T) return; // whole workgroups, or waves where a row has one: no barrier waits for them
    const int d = a.d, whole = Rw::whole(d), at = (wave % WPR * 64 + lane) * N, et = whole + lane;
    const bool tail = FORM >= FORM_TAIL && wave % WPR == 0 && et < d; // this lane has a value behind the whole pieces
    const int64_t off = row * d;
    u32x4 x[VPL];
    float h[VPL][N], ht = 0.f;
#pragma unroll
    for (int i = 0; i < VPL; ++i) x[i] = Rw::template load<ONCE>((const Elem*)a.X + off, at + i * STEP, whole);
    if (tail) ht = Rw::one((const Elem*)a.X + off + et);
    if (a.R) {
        u32x4 r[VPL];
#pragma unroll
        for (int i = 0; i < VPL; ++i) r[i] = Rw::template load<ONCE>((const Elem*)a.R + off, at + i * STEP, whole);
        if (tail) {
            ht = Rw::rounded(ht + Rw::one((const Elem*)a.R + off + et));
            Rw::put((Elem*)a.H + off + et, ht);
        }
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            float p[N], q[N];
            Rw::unpack(x[i], p), Rw::unpack(r[i], q);
#pragma unroll
            for (int k = 0; k < N; ++k) p[k] += q[k];
            x[i] = Rw::pack(p); // the statistics are those of what is stored
            Rw::store((Elem*)a.H + off, at + i * STEP, whole, x[i]);
        }
    }
    float sum = ht;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        Rw::unpack(Rw::mine(x[i], at + i * STEP, whole), h[i]);
#pragma unroll
        for (int k = 0; k < N; ++k) sum += h[i][k];
    }
    const float mu = a.layer ? row_sum<WPR>(sum, lds[0]) / (float)d : 0.f;
    ht -= mu;
    float sq = tail ? ht * ht : 0.f;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        const bool live = at + i * STEP < whole;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            h[i][k] = live ? h[i][k] - mu : 0.f;
            sq = __builtin_fmaf(h[i][k], h[i][k], sq);
        }
    }
    const float rstd = 1.0f / __builtin_sqrtf(row_sum<WPR>(sq, lds[1]) / (float)d + a.eps);
    if (wave % WPR == 0 && lane == 0) {
        a.rstd[row] = rstd;
        if (a.layer) a.mean[row] = mu;
    }
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        const int e = at + i * STEP;
        float ga[N], be[N] = {};
        Rw::unpack(Rw::load((const Elem*)a.gamma, e, whole), ga);
        if (a.beta) Rw::unpack(Rw::load((const Elem*)a.beta, e, whole), be);
#pragma unroll
        for (int k = 0; k < N; ++k) h[i][k] = __builtin_fmaf(h[i][k] * rstd, ga[k], be[k]);
        Rw::store((Elem*)a.Y + off, e, whole, Rw::pack(h[i]));
    }
    if (tail) {
        ht = ht * rstd * Rw::one((const Elem*)a.gamma + et);
        if (a.beta) ht += Rw::one((const Elem*)a.beta + et);
        Rw::put((Elem*)a.Y + off + et, ht);
    }
}

// What a lane has of a row in the backward pass
template <int BF16, int VPL>
struct Held {
    u32x4 h[VPL], dy[VPL], skip[VPL];
    float ht, dyt, skipt; // behind the whole pieces
    float rstd, mu;
};

// A workgroup of kBwdWaves waves (or those of a row) takes rows in turn and keeps its columns' share of dgamma and dbeta in registers; at
// the end the shares of the workgroup's rows are added up, in the order of its waves, and written as one row of `partial`.  The next row is
// requested before the one at hand is worked on, by the same number of loads whatever the row: with loads behind a condition the
// wait for the row at hand would be one for the next as well.
//
// ROOM: registers are enough for that, and to keep what the sums are made of for the second use.  With more than 8 values of a matrix a lane
// they are not, and spill: rows of more than 8192, us, each row requested as it is needed and values made again / otherwise: 2048 x 16384
// fp32 114 / 248, bf16 74 / 133.  Where there is room, 16384 x 2048 bf16: values kept 51, made again 60.
template <int BF16, int WPR, int VPL, int FORM, int SKIP>
__global__ __launch_bounds__(bwd_waves(WPR) * 64) void norm_bwd_kernel(NormBwd a) {
    typedef Row<BF16> Rw;
    typedef typename Rw::Elem Elem;
    typedef Held<BF16, VPL> Row1;
    constexpr int N = Rw::N, WAVES = bwd_waves(WPR), ROWS = WAVES / WPR, STEP = WPR * 64 * N;
    constexpr bool ROOM = VPL * N <= 8;
    __shared__ float2 lds[2][WAVES]; // the two sums of a row, and the next row's
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int d = a.d, whole = Rw::whole(d), at = (wave % WPR * 64 + lane) * N, et = whole + lane;
    const bool tail = FORM >= FORM_TAIL && wave % WPR == 0 && et < d;
    const float width = (float)d;
    u32x4 ga[VPL];
    float dga[VPL][N] = {}, dbe[VPL][N] = {}, gat = 0.f, dgat = 0.f, dbet = 0.f;
#pragma unroll
    for (int i = 0; i < VPL; ++i) { // 0 behind the row's whole pieces: g = gamma dy has to be 0 there, whatever the last piece's gamma is
        const int e = at + i * STEP;
        ga[i] = FORM == FORM_SHORT ? u32x4{0, 0, 0, 0} : Rw::mine(Rw::load((const Elem*)a.gamma, e, whole), e, whole);
    }
    if (tail) gat = Rw::one((const Elem*)a.gamma + et);
    const int64_t step = (int64_t)gridDim.x * ROWS;
    int64_t row = (int64_t)blockIdx.x * ROWS + wave / WPR;
    const float* means = a.mean ? a.mean : a.rstd; // no mean: read, not used
    const int ett = FORM >= FORM_TAIL ? min(et, d - 1) : 0;
    auto request = [&](int64_t r, Row1& w) {
        r = r < a.T ? r : a.T - 1; // behind the last row: read, not used
        const int64_t off = r * d;
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            if constexpr (FORM == FORM_SHORT) {
                w.h[i] = w.dy[i] = w.skip[i] = u32x4{0, 0, 0, 0};
            } else {
                w.h[i] = Rw::template load_some<FORM == FORM_ONCE>((const Elem*)a.H + off, at + i * STEP, whole);
                w.dy[i] = Rw::template load_some<FORM == FORM_ONCE>((const Elem*)a.dY + off, at + i * STEP, whole);
                if constexpr (SKIP) w.skip[i] = Rw::template load_some<FORM == FORM_ONCE>((const Elem*)a.dH + off, at + i * STEP, whole);
            }
        }
        if constexpr (FORM >= FORM_TAIL) {
            w.ht = Rw::one((const Elem*)a.H + off + ett), w.dyt = Rw::one((const Elem*)a.dY + off + ett);
            if constexpr (SKIP) w.skipt = Rw::one((const Elem*)a.dH + off + ett);
        }
        w.rstd = a.rstd[r], w.mu = means[r];
    };
    // the row in `now`, while the one after it is on its way to `next`
    auto take = [&](Row1& now, Row1& next, float2* sums) {
        if (ROOM) request(row + step, next);
        const bool live = ROWS == 1 || row < a.T;
        const int held = live ? whole : 0;
        const float mu = live && a.mean ? now.mu : 0.f, rstd = live ? now.rstd : 0.f;
        float s1 = 0.f, s2 = 0.f, xht = 0.f, gt = 0.f;
        if constexpr (FORM >= FORM_TAIL) {
            const float dyt = tail && live ? now.dyt : 0.f;
            xht = tail && live ? (now.ht - mu) * rstd : 0.f, gt = gat * dyt;
            s1 = gt * xht, s2 = gt;
            dgat += dyt * xht, dbet += dyt;
        }
        float xh[VPL][N], g[VPL][N];
        // A lane without values of the row has dy = 0 and the last piece's xh: one of the row's own, where (0 - mu) rstd may be no fp32 value
        // and its product with 0 NaN.  Behind the last row xh is 0: what was read there may have been written over (dX in the place of H).
        auto centre = [&](int i, float (&dy)[N]) {
            Rw::unpack(FORM != FORM_SHORT && live ? now.h[i] : u32x4{0, 0, 0, 0}, xh[i]), Rw::unpack(Rw::mine(now.dy[i], at + i * STEP, held), dy);
            Rw::unpack(ga[i], g[i]);
#pragma unroll
            for (int k = 0; k < N; ++k) xh[i][k] = FORM == FORM_SHORT ? 0.f : (xh[i][k] - mu) * rstd, g[i][k] *= dy[k];
        };
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            float dy[N];
            centre(i, dy);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                s1 = __builtin_fmaf(g[i][k], xh[i][k], s1);
                s2 += g[i][k];
                dga[i][k] = __builtin_fmaf(dy[k], xh[i][k], dga[i][k]);
                dbe[i][k] += dy[k];
            }
        }
        sdp::settle(dga), sdp::settle(dbe);
        row_sums<WPR>(s1, s2, sums);
        s1 /= width, s2 = a.mean ? s2 / width : 0.f;
        // xh and g: kept, or made again
        if (!ROOM) sdp::again(now.h), sdp::again(now.dy), sdp::again(ga);
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            float dx[N], skip[N] = {};
            if (!ROOM) centre(i, dx);
            if constexpr (SKIP) Rw::unpack(now.skip[i], skip);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                dx[k] = __builtin_fmaf(-xh[i][k], s1, g[i][k] - s2);
                dx[k] = SKIP ? __builtin_fmaf(dx[k], rstd, skip[k]) : dx[k] * rstd;
            }
            Rw::store((Elem*)a.dX + row * d, at + i * STEP, held, Rw::pack(dx));
        }
        if (tail && live) Rw::put((Elem*)a.dX + row * d + et, rstd * (gt - s2 - xht * s1) + (SKIP ? now.skipt : 0.f));
        row += step;
    };
    Row1 one, two;
    if (ROOM) request(row, one);
    // all waves of a workgroup take the same number of turns: their sums of a row go through a barrier.  Two rows a round: handed over from
    // `next` to `now`, a row would have to have arrived.
    for (int64_t first = (int64_t)blockIdx.x * ROWS; first < a.T; first += 2 * step) {
        if (!ROOM) request(row, one);
        take(one, two, lds[0]);
        if (first + step < a.T) {
            if (!ROOM) request(row, two);
            take(two, one, lds[1]);
        }
    }
    if (!a.want_dw) return;
    // one workgroup alone has the sums
    const bool alone = gridDim.x == 1;
    float* out = a.partial + (int64_t)blockIdx.x * 2 * d;
    auto give = [&](int part, int e, float x) {
        if (!alone) out[part * d + e] = x;
        else if (part == 0) Rw::put((Elem*)a.dgamma + e, x);
        else if (a.dbeta) Rw::put((Elem*)a.dbeta + e, x);
    };
    extern __shared__ float share[]; // [ROWS][2][d] where a workgroup has several rows
    float* mine = share + wave / WPR * 2 * d;
    auto add = [&](int e, float g, float b) {
        if (ROWS == 1) give(0, e, g), give(1, e, b);
        else mine[e] = g, mine[d + e] = b;
    };
#pragma unroll
    for (int i = 0; i < VPL; ++i)
        if (at + i * STEP < whole)
#pragma unroll
            for (int k = 0; k < N; ++k) add(at + i * STEP + k, dga[i][k], dbe[i][k]);
    if (tail) add(et, dgat, dbet);
    if (ROWS == 1) return;
    __syncthreads();
    for (int e = threadIdx.x; e < 2 * d; e += WAVES * 64) {
        float x = share[e];
#pragma unroll
        for (int r = 1; r < ROWS; ++r) x += share[r * 2 * d + e];
        give(e >= d, e >= d ? e - d : e, x);
    }
}

// Sums of the workgroups' shares, in their order: 64 columns a workgroup, sixteen waves with every sixteenth share.  n = 0: zeros.
template <int BF16>
__global__ __launch_bounds__(1024) void norm_dw_kernel(const float* __restrict__ partial, int n, int d, void* dgamma, void* dbeta) {
    typedef typename Row<BF16>::Elem Elem;
    constexpr int WAVES = 16, B = 8;
    __shared__ float lds[WAVES][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int e = blockIdx.x * 64 + lane, part = blockIdx.y;
    float s = 0.f;
    if (e < d)
        for (int i0 = wave; i0 < n; i0 += WAVES * B) { // B shares in flight
            float v[B];
#pragma unroll
            for (int j = 0; j < B; ++j) v[j] = i0 + j * WAVES < n ? partial[((int64_t)(i0 + j * WAVES) * 2 + part) * d + e] : 0.f;
#pragma unroll
            for (int j = 0; j < B; ++j) s += v[j];
        }
    lds[wave][lane] = s;
    __syncthreads();
    if (wave != 0 || e >= d) return;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) s += lds[w][lane];
    Row<BF16>::put((Elem*)(part ? dbeta : dgamma) + e, s);
}

// Waves of a row and pieces of a lane.
struct Shape {
    int wpr, vpl;
};
// One wave where it can hold the row: its sums need no barrier.  us, one wave / four: 16384 x 768 bf16 16.5 / 22.6, 8192 x 1024 11.3 / 15.5,
// 16384 x 2048 47.8 / 49.5, though 8192 x 2000 23.0 / 22.3.  Else four, if they can: four / sixteen: 8192 x 4096 46.6 / 60.6, 4096 x 3200 17.0 / 24.7.
Shape fwd_shape(int dtype, int d) {
    const int n = dtype == SDP_BF16 ? 8 : 4, pieces = (d + n - 1) / n;
    if (pieces <= 256) return {1, (pieces + 63) / 64};
    if (pieces <= 1024) return {4, pieces <= 512 ? 2 : 4};
    return {16, pieces <= 2048 ? 2 : 4};
}
// A row of whole waves' pieces, one a lane in bf16 and two in fp32, eight values of each matrix either way: more waves leave lanes idle, fewer
// take more registers.  us, bf16, one piece / two: 16384 x 2048 51.2 / 55.8, 16384 x 1200 34.7 / 38.0; but 16384 x 768
// 21.7 / 20.8, 4096 x 3200 25.9 / 23.7.
Shape bwd_shape(int dtype, int d) {
    const int n = dtype == SDP_BF16 ? 8 : 4, pieces = (d + n - 1) / n, most = dtype == SDP_BF16 ? 1 : 2;
    if (pieces <= 64 * most) return {1, (pieces + 63) / 64};
    for (int w : {2, 3, 4, 8})
        if (pieces <= 64 * most * w) return {w, most};
    return {16, pieces <= 1024 * most ? most : 2 * most};
}
int fwd_rows(const Shape& s) { return s.wpr == 1 ? 4 : 1; }
int bwd_rows(const Shape& s) { return bwd_waves(s.wpr) / s.wpr; }

// Workgroups of the backward pass: one on every CU; with two, twice the shares are written and added up: 16384 x 2048 bf16 51.2 and 55.1 us,
// 8192 x 8192 99.8 and 112.9.  Where one alone has kBwdAlone turns at most they take less than a second launch, and it writes the sums itself:
// 16 x 768 one launch 5.8 us, two 7.7.
constexpr int kBwdGroups = 256, kBwdAlone = 4;
int bwd_groups(int T, const Shape& s) {
    const int64_t all = ((int64_t)T + bwd_rows(s) - 1) / bwd_rows(s);
    return all <= kBwdAlone ? (all > 0) : (int)(all < kBwdGroups ? all : kBwdGroups);
}

#define SDP_NORM_SHAPE(W, V) \
    if (s.wpr == W && s.vpl == V) return launch(bf16, std::integral_constant<int, W>{}, std::integral_constant<int, V>{})
template <class F>
int by_fwd_shape(int dtype, const Shape& s, F&& launch) {
    auto with = [&](auto bf16) {
        SDP_NORM_SHAPE(1, 1);
        SDP_NORM_SHAPE(1, 2);
        SDP_NORM_SHAPE(1, 3);
        SDP_NORM_SHAPE(1, 4);
        SDP_NORM_SHAPE(4, 2);
        SDP_NORM_SHAPE(4, 4);
        SDP_NORM_SHAPE(16, 2);
        if constexpr (!bf16.value) SDP_NORM_SHAPE(16, 4);
        return (int)SDP_ERR_UNSUPPORTED;
    };
    return dtype == SDP_BF16 ? with(std::integral_constant<int, 1>{}) : with(std::integral_constant<int, 0>{});
}
template <class F>
int by_bwd_shape(int dtype, const Shape& s, F&& launch) {
    auto with = [&](auto bf16) {
        constexpr int M = bf16.value ? 1 : 2;
        SDP_NORM_SHAPE(1, 1);
        if constexpr (!bf16.value) SDP_NORM_SHAPE(1, 2);
        SDP_NORM_SHAPE(2, M);
        SDP_NORM_SHAPE(3, M);
        SDP_NORM_SHAPE(4, M);
        SDP_NORM_SHAPE(8, M);
        SDP_NORM_SHAPE(16, M);
        SDP_NORM_SHAPE(16, 2 * M);
        return (int)SDP_ERR_UNSUPPORTED;
    };
    return dtype == SDP_BF16 ? with(std::integral_constant<int, 1>{}) : with(std::integral_constant<int, 0>{});
}
#undef SDP_NORM_SHAPE

int check_norm(int kind, int dtype, int T, int d) {
    if (kind != SDP_NORM_LAYER && kind != SDP_NORM_RMS) return SDP_ERR_INVALID_ARG;
    if (dtype != SDP_F32 && dtype != SDP_BF16) return SDP_ERR_INVALID_ARG;
    if (T < 0 || d < 1) return SDP_ERR_INVALID_ARG;
    return d > SDP_NORM_MAX_WIDTH || T > SDP_MAX_EXTENT ? SDP_ERR_SHAPE : SDP_OK;
}

} // namespace

extern "C" int sdp_norm_fwd(int kind, int dtype, int T, int d, float eps, const void* X, const void* R, const void* gamma,
                            const void* beta, void* H, void* Y, float* mean, float* rstd, void* stream) {
    const int rc = check_norm(kind, dtype, T, d);
    if (rc != SDP_OK) return rc;
    if (!(eps >= 0.f) || !std::isfinite(eps)) return SDP_ERR_INVALID_ARG;
    const bool layer = kind == SDP_NORM_LAYER;
    if (T == 0) return SDP_OK;
    if (!X || !gamma || !Y || !rstd || (R != nullptr) != (H != nullptr) || layer != (mean != nullptr)) return SDP_ERR_INVALID_ARG;
    const size_t es = dtype == SDP_BF16 ? 2 : 4, rows = (size_t)T * d * es, w = (size_t)d * es, st = (size_t)T * 4;
    for (const void* p : {X, R, gamma, beta, (const void*)H, (const void*)Y})
        if (!sdp::aligned_to(p, es)) return SDP_ERR_INVALID_ARG;
    if (!sdp::aligned_to(mean, 4) || !sdp::aligned_to(rstd, 4)) return SDP_ERR_INVALID_ARG;
    const sdp::Extent eX{X, rows}, eR{R, R ? rows : 0}, eg{gamma, w}, eb{beta, beta ? w : 0}, eH{H, H ? rows : 0}, eY{Y, rows},
        em{mean, mean ? st : 0}, es_{rstd, st};
    for (const sdp::Extent& o : {eH, eY})
        for (const sdp::Extent& i : {eX, eR})
            if (o.p != i.p && sdp::overlap({o}, {i})) return SDP_ERR_INVALID_ARG;
    if (sdp::overlap({eH, eY, em, es_}, {eg, eb}) || sdp::overlap({em, es_}, {eX, eR, eH, eY}) || sdp::overlap({eH}, {eY}) ||
        sdp::overlap({em}, {es_}))
        return SDP_ERR_INVALID_ARG;
    hipStream_t s = (hipStream_t)stream;
    const Shape sh = fwd_shape(dtype, d);
    const NormFwd a{X, R, gamma, beta, H, Y, mean, rstd, T, d, layer, eps};
    const bool once = sdp::read_once({eX, eR}, w);
    sdp::ProfileScope ps("norm_fwd", s);
    const dim3 groups = sdp::grid_of(((int64_t)T + fwd_rows(sh) - 1) / fwd_rows(sh));
    return by_fwd_shape(dtype, sh, [&](auto bf16, auto wpr, auto vpl) {
        auto go = [&](auto form) {
            norm_fwd_kernel<bf16.value, wpr.value, vpl.value, form.value><<<groups, waves_of(wpr.value) * 64, 0, s>>>(a);
        };
        if (d % Row<bf16.value>::N) go(std::integral_constant<int, FORM_TAIL>{});
        else if (once) go(std::integral_constant<int, FORM_ONCE>{});
        else go(std::integral_constant<int, FORM_WHOLE>{});
        return sdp::launch_status();
    });
}

extern "C" size_t sdp_norm_bwd_workspace_bytes(int dtype, int T, int d) {
    if (check_norm(SDP_NORM_LAYER, dtype, T, d) != SDP_OK) return 0;
    return sdp::round_up((size_t)bwd_groups(T, bwd_shape(dtype, d)) * 2 * d * sizeof(float), 256);
}

extern "C" int sdp_norm_bwd(int kind, int dtype, int T, int d, const void* H, const void* dY, const void* dH, const void* gamma,
                            const float* mean, const float* rstd, void* dX, void* dgamma, void* dbeta, void* ws, size_t ws_bytes,
                            void* stream) {
    const int rc = check_norm(kind, dtype, T, d);
    if (rc != SDP_OK) return rc;
    const size_t es = dtype == SDP_BF16 ? 2 : 4, rows = (size_t)T * d * es, w = (size_t)d * es, st = (size_t)T * 4;
    if (dbeta && !dgamma) return SDP_ERR_INVALID_ARG;
    if (T > 0 && (!H || !dY || !gamma || !rstd || !dX || (kind == SDP_NORM_LAYER) != (mean != nullptr))) return SDP_ERR_INVALID_ARG;
    for (const void* p : {H, dY, dH, gamma, (const void*)dX, (const void*)dgamma, (const void*)dbeta})
        if (!sdp::aligned_to(p, es)) return SDP_ERR_INVALID_ARG;
    if (!sdp::aligned_to(mean, 4) || !sdp::aligned_to(rstd, 4)) return SDP_ERR_INVALID_ARG;
    const size_t need = dgamma ? sdp_norm_bwd_workspace_bytes(dtype, T, d) : 0;
    const sdp::Extent eH{H, H ? rows : 0}, eY{dY, dY ? rows : 0}, eS{dH, dH ? rows : 0}, eg{gamma, gamma ? w : 0},
        em{mean, mean ? st : 0}, er{rstd, rstd ? st : 0}, oX{dX, dX ? rows : 0}, og{dgamma, dgamma ? w : 0}, ob{dbeta, dbeta ? w : 0};
    for (const sdp::Extent& i : {eH, eY, eS})
        if (oX.p != i.p && sdp::overlap({oX}, {i})) return SDP_ERR_INVALID_ARG;
    if (sdp::overlap({og, ob}, {eH, eY, eS, eg, em, er, oX}) || sdp::overlap({oX}, {eg, em, er}) || sdp::overlap({og}, {ob}))
        return SDP_ERR_INVALID_ARG;
    if (need > 0 && (!ws || !sdp::aligned16(ws) || ws_bytes < need)) return SDP_ERR_WORKSPACE;
    hipStream_t s = (hipStream_t)stream;
    const Shape sh = bwd_shape(dtype, d);
    const int groups = bwd_groups(T, sh);
    const bool once = sdp::read_once({eH, eY, eS}, w);
    sdp::ProfileScope ps("norm_bwd", s);
    int st2 = SDP_OK;
    if (groups > 0) {
        const NormBwd a{H, dY, dH, gamma, mean, rstd, dX, dgamma, dbeta, (float*)ws, T, d, dgamma != nullptr};
        const size_t lds = bwd_rows(sh) > 1 && dgamma ? (size_t)bwd_rows(sh) * 2 * d * sizeof(float) : 0;
        st2 = by_bwd_shape(dtype, sh, [&](auto bf16, auto wpr, auto vpl) {
            auto go = [&](auto form) {
                if (dH) norm_bwd_kernel<bf16.value, wpr.value, vpl.value, form.value, 1><<<groups, bwd_waves(wpr.value) * 64, lds, s>>>(a);
                else norm_bwd_kernel<bf16.value, wpr.value, vpl.value, form.value, 0><<<groups, bwd_waves(wpr.value) * 64, lds, s>>>(a);
            };
            if (once) go(std::integral_constant<int, FORM_ONCE>{});
            else if (d % Row<bf16.value>::N == 0) go(std::integral_constant<int, FORM_WHOLE>{});
            else if (wpr.value > 1 || d > Row<bf16.value>::N) go(std::integral_constant<int, FORM_TAIL>{});
            else go(std::integral_constant<int, wpr.value * vpl.value == 1 ? FORM_SHORT : FORM_TAIL>{});
            return sdp::launch_status();
        });
    }
    if (st2 != SDP_OK || !dgamma || groups == 1) return st2;
    const dim3 grid((d + 63) / 64, dbeta ? 2 : 1);
    if (dtype == SDP_BF16) norm_dw_kernel<1><<<grid, 1024, 0, s>>>((const float*)ws, groups, d, dgamma, dbeta);
    else norm_dw_kernel<0><<<grid, 1024, 0, s>>>((const float*)ws, groups, d, dgamma, dbeta);
    return sdp::launch_status();
}
