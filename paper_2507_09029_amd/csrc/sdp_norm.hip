// Layer and root-mean-square norm of tokens, alone or of a sum with the skip connection, and the backward pass.
//
//   forward   h = x + r (rounded), mu = mean(h) (0 for the root-mean-square form), s = 1 / sqrt(mean((h - mu)^2) + eps),
//             y = (h - mu) s gamma + beta
//   backward  xh = (h - mu) s, g = dy gamma, dx = s (g - mean(g) - xh mean(g xh)) + dh (mean(g) only in the layer form),
//             dgamma = sum_t dy xh, dbeta = sum_t dy
//
// Both are bound by memory: a row is read once into registers, its sums are taken over the lanes that hold it, and it is written
// once.  A row belongs to WPR waves, each lane holding up to VPL pieces of 16 bytes.
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

// waves of a workgroup: four rows of one wave each, or one row of four or sixteen
constexpr int waves_of(int WPR) { return WPR > 4 ? WPR : 4; }

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

template <int BF16, int WPR, int VPL, int ONCE>
__global__ __launch_bounds__(waves_of(WPR) * 64) void norm_fwd_kernel(NormFwd a) {
    typedef Row<BF16> Rw;
    typedef typename Rw::Elem Elem;
    constexpr int N = Rw::N, ROWS = waves_of(WPR) / WPR;
    __shared__ float lds[2][waves_of(WPR)];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * ROWS + wave / WPR;
    if (ROWS > 1 && row >= a.T) return; // no barrier where a workgroup has several rows
    const int d = a.d, at = (wave % WPR * 64 + lane) * N;
    const int64_t off = row * d;
    u32x4 x[VPL];
    float h[VPL][N];
#pragma unroll
    for (int i = 0; i < VPL; ++i) x[i] = Rw::template load<ONCE>((const Elem*)a.X + off, at + i * WPR * 64 * N, d);
    if (a.R) {
        u32x4 r[VPL];
#pragma unroll
        for (int i = 0; i < VPL; ++i) r[i] = Rw::template load<ONCE>((const Elem*)a.R + off, at + i * WPR * 64 * N, d);
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            float p[N], q[N];
            Rw::unpack(x[i], p), Rw::unpack(r[i], q);
#pragma unroll
            for (int k = 0; k < N; ++k) p[k] += q[k];
            x[i] = Rw::pack(p); // the statistics are those of what is stored
            Rw::store((Elem*)a.H + off, at + i * WPR * 64 * N, d, x[i]);
        }
    }
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        Rw::unpack(x[i], h[i]);
#pragma unroll
        for (int k = 0; k < N; ++k) sum += h[i][k];
    }
    const float mu = a.layer ? row_sum<WPR>(sum, lds[0]) / (float)d : 0.f;
    float sq = 0.f;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        const int left = d - (at + i * WPR * 64 * N); // what lies behind the row's end has no part in the squares
#pragma unroll
        for (int k = 0; k < N; ++k) {
            h[i][k] -= mu;
            sq += k < left ? h[i][k] * h[i][k] : 0.f;
        }
    }
    const float rstd = 1.0f / __builtin_sqrtf(row_sum<WPR>(sq, lds[1]) / (float)d + a.eps);
    if (wave % WPR == 0 && lane == 0) {
        a.rstd[row] = rstd;
        if (a.layer) a.mean[row] = mu;
    }
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        const int e = at + i * WPR * 64 * N;
        if (e >= d) break;
        float ga[N], be[N];
        Rw::unpack(Rw::load((const Elem*)a.gamma, e, d), ga);
        if (a.beta) Rw::unpack(Rw::load((const Elem*)a.beta, e, d), be);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            h[i][k] = h[i][k] * rstd * ga[k];
            if (a.beta) h[i][k] += be[k];
        }
        Rw::store((Elem*)a.Y + off, e, d, Rw::pack(h[i]));
    }
}

// A workgroup takes rows in turn and keeps its columns' share of dgamma and dbeta in registers; at the end the shares of the
// workgroup's rows are added up, in the order of its waves, and written as one row of `partial`.
template <int BF16, int WPR, int VPL>
__global__ __launch_bounds__(waves_of(WPR) * 64) void norm_bwd_kernel(NormBwd a) {
    typedef Row<BF16> Rw;
    typedef typename Rw::Elem Elem;
    constexpr int N = Rw::N, ROWS = waves_of(WPR) / WPR;
    __shared__ float lds[2][2][waves_of(WPR)]; // two sums of a row, and the next row's
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int d = a.d, at = (wave % WPR * 64 + lane) * N;
    const float width = (float)d;
    u32x4 ga[VPL];
    float dga[VPL][N] = {}, dbe[VPL][N] = {};
#pragma unroll
    for (int i = 0; i < VPL; ++i) ga[i] = Rw::load((const Elem*)a.gamma, at + i * WPR * 64 * N, d);
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * ROWS + wave / WPR; row < a.T; row += (int64_t)gridDim.x * ROWS, turn ^= 1) {
        const int64_t off = row * d;
        u32x4 hw[VPL], yw[VPL];
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            hw[i] = Rw::load((const Elem*)a.H + off, at + i * WPR * 64 * N, d);
            yw[i] = Rw::load((const Elem*)a.dY + off, at + i * WPR * 64 * N, d);
        }
        const float rstd = a.rstd[row], mu = a.mean ? a.mean[row] : 0.f;
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            // behind the row's end dy and gamma are zeros
            float h[N], dy[N], g[N];
            Rw::unpack(hw[i], h), Rw::unpack(yw[i], dy), Rw::unpack(ga[i], g);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const float xh = (h[k] - mu) * rstd;
                g[k] *= dy[k];
                s1 += g[k] * xh;
                s2 += g[k];
                dga[i][k] += dy[k] * xh;
                dbe[i][k] += dy[k];
            }
        }
        s1 = row_sum<WPR>(s1, lds[turn][0]) / width;
        s2 = a.mean ? row_sum<WPR>(s2, lds[turn][1]) / width : 0.f;
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            const int e = at + i * WPR * 64 * N;
            if (e >= d) break;
            float h[N], dy[N], g[N], skip[N];
            Rw::unpack(hw[i], h), Rw::unpack(yw[i], dy), Rw::unpack(ga[i], g);
            if (a.dH) Rw::unpack(Rw::load((const Elem*)a.dH + off, e, d), skip);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                h[k] = rstd * (g[k] * dy[k] - s2 - (h[k] - mu) * rstd * s1);
                if (a.dH) h[k] += skip[k];
            }
            Rw::store((Elem*)a.dX + off, e, d, Rw::pack(h));
        }
    }
    if (!a.want_dw) return;
    extern __shared__ float share[]; // [2][d] where a workgroup has several rows
    if (ROWS > 1) {
        for (int r = 0; r < ROWS; ++r) {
            if (r) __syncthreads();
            if (wave / WPR != r) continue;
#pragma unroll
            for (int i = 0; i < VPL; ++i)
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    const int e = at + i * WPR * 64 * N + k;
                    if (e >= d) continue;
                    share[e] = r ? share[e] + dga[i][k] : dga[i][k];
                    share[d + e] = r ? share[d + e] + dbe[i][k] : dbe[i][k];
                }
        }
        __syncthreads();
        for (int e = threadIdx.x; e < 2 * d; e += waves_of(WPR) * 64) a.partial[(int64_t)blockIdx.x * 2 * d + e] = share[e];
    } else {
#pragma unroll
        for (int i = 0; i < VPL; ++i)
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const int e = at + i * WPR * 64 * N + k;
                if (e >= d) continue;
                a.partial[(int64_t)blockIdx.x * 2 * d + e] = dga[i][k];
                a.partial[(int64_t)blockIdx.x * 2 * d + d + e] = dbe[i][k];
            }
    }
}

// Sums of the workgroups' shares, in their order: 64 columns a workgroup, four waves with every fourth share.  n = 0: zeros.
template <int BF16>
__global__ __launch_bounds__(256) void norm_dw_kernel(const float* __restrict__ partial, int n, int d, void* dgamma, void* dbeta) {
    typedef typename Row<BF16>::Elem Elem;
    __shared__ float lds[4][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int e = blockIdx.x * 64 + lane, part = blockIdx.y;
    float s = 0.f;
    if (e < d)
#pragma unroll 8
        for (int i = wave; i < n; i += 4) s += partial[((int64_t)i * 2 + part) * d + e];
    lds[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && e < d) Row<BF16>::put((Elem*)(part ? dbeta : dgamma) + e, ((lds[0][lane] + lds[1][lane]) + lds[2][lane]) + lds[3][lane]);
}

// waves of a row and pieces of a lane: as few waves as hold it with four pieces a lane (eight where sixteen waves do not)
struct Shape {
    int wpr, vpl;
};
Shape shape(int dtype, int d) {
    const int n = dtype == SDP_BF16 ? 8 : 4, pieces = (d + n - 1) / n;
    if (pieces <= 256) return {1, (pieces + 63) / 64};
    if (pieces <= 1024) return {4, pieces <= 512 ? 2 : 4};
    return {16, pieces <= 4096 ? 4 : 8};
}
int rows_of(const Shape& s) { return s.wpr == 1 ? 4 : 1; }

constexpr int kBwdGroups = 512;
int bwd_groups(int T, const Shape& s) {
    const int64_t all = ((int64_t)T + rows_of(s) - 1) / rows_of(s);
    return (int)(all < kBwdGroups ? all : kBwdGroups);
}

template <class F>
int by_shape(int dtype, const Shape& s, F&& launch) {
    auto with = [&](auto bf16) {
#define SDP_NORM_SHAPE(W, V) \
    if (s.wpr == W && s.vpl == V) return launch(bf16, std::integral_constant<int, W>{}, std::integral_constant<int, V>{})
        SDP_NORM_SHAPE(1, 1);
        SDP_NORM_SHAPE(1, 2);
        SDP_NORM_SHAPE(1, 3);
        SDP_NORM_SHAPE(1, 4);
        SDP_NORM_SHAPE(4, 2);
        SDP_NORM_SHAPE(4, 4);
        SDP_NORM_SHAPE(16, 4);
        if constexpr (!bf16.value) SDP_NORM_SHAPE(16, 8);
#undef SDP_NORM_SHAPE
        return (int)SDP_ERR_UNSUPPORTED;
    };
    return dtype == SDP_BF16 ? with(std::integral_constant<int, 1>{}) : with(std::integral_constant<int, 0>{});
}

int check_norm(int kind, int dtype, int T, int d) {
    if (kind != SDP_NORM_LAYER && kind != SDP_NORM_RMS) return SDP_ERR_INVALID_ARG;
    if (dtype != SDP_F32 && dtype != SDP_BF16) return SDP_ERR_INVALID_ARG;
    if (T < 0 || d < 1) return SDP_ERR_INVALID_ARG;
    return d > SDP_NORM_MAX_WIDTH || T > SDP_MAX_TOKENS ? SDP_ERR_SHAPE : SDP_OK;
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
    const Shape sh = shape(dtype, d);
    const NormFwd a{X, R, gamma, beta, H, Y, mean, rstd, T, d, layer, eps};
    const bool once = sdp::read_once({eX, eR}, w);
    sdp::ProfileScope ps("norm_fwd", s);
    const unsigned groups = (unsigned)(((int64_t)T + rows_of(sh) - 1) / rows_of(sh));
    return by_shape(dtype, sh, [&](auto bf16, auto wpr, auto vpl) {
        if (once) norm_fwd_kernel<bf16.value, wpr.value, vpl.value, 1><<<groups, waves_of(wpr.value) * 64, 0, s>>>(a);
        else norm_fwd_kernel<bf16.value, wpr.value, vpl.value, 0><<<groups, waves_of(wpr.value) * 64, 0, s>>>(a);
        return sdp::launch_status();
    });
}

extern "C" size_t sdp_norm_bwd_workspace_bytes(int dtype, int T, int d) {
    if (check_norm(SDP_NORM_LAYER, dtype, T, d) != SDP_OK) return 0;
    return sdp::round_up((size_t)bwd_groups(T, shape(dtype, d)) * 2 * d * sizeof(float), 256);
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
    const Shape sh = shape(dtype, d);
    const int groups = bwd_groups(T, sh);
    sdp::ProfileScope ps("norm_bwd", s);
    int st2 = SDP_OK;
    if (groups > 0) {
        const NormBwd a{H, dY, dH, gamma, mean, rstd, dX, dgamma, dbeta, (float*)ws, T, d, dgamma != nullptr};
        const size_t lds = sh.wpr == 1 && dgamma ? (size_t)2 * d * sizeof(float) : 0;
        st2 = by_shape(dtype, sh, [&](auto bf16, auto wpr, auto vpl) {
            norm_bwd_kernel<bf16.value, wpr.value, vpl.value><<<groups, waves_of(wpr.value) * 64, lds, s>>>(a);
            return sdp::launch_status();
        });
    }
    if (st2 != SDP_OK || !dgamma) return st2;
    const dim3 grid((d + 63) / 64, dbeta ? 2 : 1);
    if (dtype == SDP_BF16) norm_dw_kernel<1><<<grid, 256, 0, s>>>((const float*)ws, groups, d, dgamma, dbeta);
    else norm_dw_kernel<0><<<grid, 256, 0, s>>>((const float*)ws, groups, d, dgamma, dbeta);
    return sdp::launch_status();
}
