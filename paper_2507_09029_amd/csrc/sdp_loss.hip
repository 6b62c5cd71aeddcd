// Cross-entropy of rows of logits against labels, with the gradient from the same read of the logits.
//
//   lse = log sum_j exp z_j,  nll = lse - z_label,  dz_j = c (exp(z_j - lse) - [j = label])
//
// Bound by memory: the logits are the largest tensor of a training step (8192 x 32000 bf16: 524 MB), and the least that can be
// moved is one read and one write of them.  A workgroup holds a row in registers, as it is stored, from the read to the write: up to 16
// waves with up to 16 pieces of 16 bytes a lane, as many as leave room for several rows on a CU (by_row).  Rows of more than 131072
// bf16 or 65536 fp32 values are read for the maximum, for the sum and for the gradient: 1024 x 152000 bf16 176 us, 89 without a gradient,
// 512 x 128256 fp32 148 and 73.  8192 x 32000 bf16: 177 us with the scale and the sum of the loss, 5.9 TB/s, more than a large copy
// reaches; 1000 x 50001, a quarter without a label: 42 us, 4.1 TB/s, with three rows to read a CU.
//
// exp(z - max) is 2^((z - max) L), L = log2 e, on the hardware's 2^x.  The difference comes first: z L - max L in one step, with max L
// rounded, overflows or is far off where a row's values are near the type's lowest, as masks write them.
#include <cmath>
#include <type_traits>

#include "sdp_internal.h"
#include "sdp_loss_rows.h"
#include "sdp_rows.h"

namespace {

using sdp::group_all;
using sdp::kLog2e;
using sdp::minus_inf;
using sdp::Row;
using sdp::u32x4;

struct Loss {
    const void *Z, *labels;
    const float* scale_dev;
    float *nll, *lse;
    void* dZ;
    int T, V, wide;
    int64_t ldz;
    float scale;
};

// PIECES > 0: pieces a lane holds, the row has no more; 0: the row is read again for the sum, and again for the gradient
template <int BF16, int WAVES, int PIECES, int ONCE>
__global__ __launch_bounds__(WAVES * 64) void token_loss_kernel(Loss a) {
    typedef Row<BF16> Rw;
    typedef typename Rw::Elem Elem;
    constexpr int N = Rw::N, TH = WAVES * 64, P = PIECES ? PIECES : 1;
    __shared__ float lds[2][WAVES], at_label;
    const int64_t row = sdp::group_id();
    if (row >= a.T) return;
    const int tid = threadIdx.x, V = a.V, whole = Rw::whole(V), label = sdp::token_id(a.labels, a.wide, row, V);
    const Elem* z = (const Elem*)a.Z + row * a.ldz;
    Elem* dz = (Elem*)a.dZ + row * a.ldz;
    const bool tail = whole + tid < V; // this lane has a value behind the whole pieces
    if (label < 0) {
        if (tid == 0) {
            a.nll[row] = 0.f;
            if (a.lse) a.lse[row] = 0.f;
        }
        if (a.dZ) {
            for (int64_t e = tid * N; e < whole; e += TH * N) Rw::store(dz, (int)e, whole, u32x4{0, 0, 0, 0});
            if (tail) Rw::put(dz + whole + tid, 0.f);
        }
        return;
    }
    const float c = a.scale * (a.scale_dev ? *a.scale_dev : 1.f);
    u32x4 w[P];
    auto piece = [&](int64_t e) { return Rw::mine(Rw::load(z, (int)e, whole), (int)e, whole, minus_inf<BF16>()); }; // of a row that is read again
    if (PIECES)
#pragma unroll
        for (int i = 0; i < P; ++i) w[i] = Rw::template load<ONCE>(z, (tid + i * TH) * N, whole);
    const float zt = tail ? Rw::one(z + whole + tid) : -INFINITY;
    if (tid == 0) at_label = Rw::one(z + label); // read before anything is written: dZ may be Z
    float m = zt, sum = 0.f;
    if (PIECES) {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            float v[N];
            w[i] = Rw::mine(w[i], (tid + i * TH) * N, whole, minus_inf<BF16>());
            Rw::unpack(w[i], v);
#pragma unroll
            for (int k = 0; k < N; ++k) m = fmaxf(m, v[k]);
        }
    } else {
        for (int64_t e = tid * N; e < whole; e += TH * N) {
            float v[N];
            Rw::unpack(piece(e), v);
#pragma unroll
            for (int k = 0; k < N; ++k) m = fmaxf(m, v[k]);
        }
    }
    m = group_all<WAVES, true>(m, lds[0]);
    if (PIECES) sdp::again(w);
    auto power = [&](float v) { return __builtin_amdgcn_exp2f((v - m) * kLog2e); };
    if (tail) sum = power(zt);
    if (PIECES) {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            float v[N];
            Rw::unpack(w[i], v);
#pragma unroll
            for (int k = 0; k < N; ++k) sum += power(v[k]);
        }
    } else { // up to 2^18 pieces: a running fp32 sum of terms of one size drifts to one side (65536 terms: 1e-3)
        double all = 0.0;
        for (int64_t e = tid * N; e < whole; e += TH * N) {
            float v[N];
            Rw::unpack(piece(e), v);
            float part = 0.f;
#pragma unroll
            for (int k = 0; k < N; ++k) part += power(v[k]);
            all += (double)part;
        }
        sum += (float)all;
    }
    sum = group_all<WAVES, false>(sum, lds[1]);
    if (PIECES) sdp::again(w);
    if (tid == 0) {
        const float log_sum = logf(sum);
        a.nll[row] = (m - at_label) + log_sum;
        if (a.lse) a.lse[row] = m + log_sum;
    }
    if (!a.dZ) return;
    const float inv = c / sum;
    auto gradient = [&](int e, const u32x4& x) {
        float v[N];
        Rw::unpack(x, v);
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = power(v[k]) * inv;
        if ((uint32_t)(label - e) < (uint32_t)N)
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] -= e + k == label ? c : 0.f;
        Rw::store(dz, e, whole, Rw::pack(v));
    };
    if (PIECES) {
#pragma unroll
        for (int i = 0; i < P; ++i) gradient((tid + i * TH) * N, w[i]);
    } else {
        for (int64_t e = tid * N; e < whole; e += TH * N) gradient((int)e, piece(e));
    }
    if (tail) Rw::put(dz + whole + tid, power(zt) * inv - (whole + tid == label ? c : 0.f));
}

// Sum of a double over a workgroup of 1024, in a fixed order; valid in thread 0
template <class S>
__device__ inline S group_sum(S x) {
    __shared__ S lds[16];
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) x += __shfl_xor(x, d, 64);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = lds[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) x += lds[i];
    return x;
}

__global__ __launch_bounds__(1024) void loss_sum_kernel(const float* __restrict__ nll, int T, float scale, const float* scale_dev,
                                                        float* loss) {
    double x = 0.0;
    const int whole = Row<0>::whole(T);
    for (int t0 = threadIdx.x * 4; t0 < whole; t0 += 4 * 4096) {
        u32x4 w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = Row<0>::load_some(nll, t0 + i * 4096, whole);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = Row<0>::mine(w[i], t0 + i * 4096, whole);
#pragma unroll
            for (int k = 0; k < 4; ++k) x += (double)__uint_as_float(w[i][k]);
        }
    }
    if (whole + (int)threadIdx.x < T) x += (double)nll[whole + threadIdx.x];
    x = group_sum(x);
    if (threadIdx.x == 0) *loss = (float)(x * ((double)scale * (scale_dev ? (double)*scale_dev : 1.0)));
}

template <int WIDE>
__global__ __launch_bounds__(1024) void label_scale_kernel(const void* __restrict__ labels, int T, int V, float* scale) {
    int n = 0;
    // 16 bytes at a time, as words
    constexpr int W = WIDE ? 2 : 1, N = 4 / W;
    const int whole = T / N * N;
    for (int t0 = threadIdx.x * N; t0 < whole; t0 += 4 * 1024 * N) {
        u32x4 w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = *(const sdp::u32x4_at4*)((const char*)labels + (int64_t)min(t0 + i * 1024 * N, whole - N) * (4 * W));
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int k = 0; k < 4; k += W)
                n += t0 + i * 1024 * N < whole && w[i][k] < (uint32_t)V && (!WIDE || w[i][(k + 1) % 4] == 0);
    }
    if (whole + (int)threadIdx.x < T) n += sdp::token_id<WIDE>(labels, whole + threadIdx.x, V) >= 0;
    n = group_sum(n);
    if (threadIdx.x == 0) *scale = 1.0f / (float)(n > 1 ? n : 1);
}

} // namespace

int sdp::loss_sum(const float* of, int T, float scale, const float* scale_dev, float* loss, hipStream_t s) {
    loss_sum_kernel<<<1, 1024, 0, s>>>(of, T, scale, scale_dev, loss);
    return launch_status();
}

extern "C" int sdp_token_loss(int dtype, int id_type, int T, int V, int64_t ldz, float scale, const void* Z, const void* labels,
                              const float* scale_dev, float* nll, float* lse, void* dZ, float* loss, void* stream) {
    if (dtype != SDP_F32 && dtype != SDP_BF16) return SDP_ERR_INVALID_ARG;
    if (id_type != SDP_I32 && id_type != SDP_I64) return SDP_ERR_INVALID_ARG;
    if (T < 0 || V < 1 || !std::isfinite(scale)) return SDP_ERR_INVALID_ARG;
    if (T > SDP_MAX_EXTENT || V > SDP_MAX_EXTENT || ldz < V || ldz > ((int64_t)1 << 40)) return SDP_ERR_SHAPE;
    const size_t es = dtype == SDP_BF16 ? 2 : 4, is = id_type == SDP_I64 ? 8 : 4, st = (size_t)T * 4;
    if (T > 0 && (!Z || !labels || !nll)) return SDP_ERR_INVALID_ARG;
    if (!sdp::aligned_to(Z, es) || !sdp::aligned_to(dZ, es) || !sdp::aligned_to(labels, is)) return SDP_ERR_INVALID_ARG;
    for (const float* p : {scale_dev, (const float*)nll, (const float*)lse, (const float*)loss})
        if (!sdp::aligned_to(p, 4)) return SDP_ERR_INVALID_ARG;
    const size_t rows = T > 0 ? ((size_t)(T - 1) * ldz + V) * es : 0;
    const sdp::Extent eZ{Z, rows}, el{labels, (size_t)T * is}, ec{scale_dev, scale_dev ? 4u : 0u}, on{nll, st}, os{lse, lse ? st : 0},
        oz{dZ, dZ ? rows : 0}, o1{loss, loss ? 4u : 0u};
    if (T > 0 && ((dZ != Z && sdp::overlap({oz}, {eZ})) || sdp::overlap({oz, on, os, o1}, {el, ec}) || sdp::overlap({on, os, o1}, {eZ, oz}) ||
                  sdp::overlap({on}, {os, o1}) || sdp::overlap({os}, {o1})))
        return SDP_ERR_INVALID_ARG;
    hipStream_t s = (hipStream_t)stream;
    sdp::ProfileScope ps("token_loss", s);
    int rc = SDP_OK;
    if (T > 0) {
        const Loss a{Z, labels, scale_dev, nll, lse, dZ, T, V, id_type == SDP_I64, ldz, scale};
        const bool once = sdp::read_once({eZ}, (size_t)ldz * es);
        sdp::by_row(dtype == SDP_BF16, V, [&](auto b, auto waves, auto p) {
            if (p.value && once) token_loss_kernel<b.value, waves.value, p.value, p.value != 0><<<sdp::grid_of(T), waves.value * 64, 0, s>>>(a);
            else token_loss_kernel<b.value, waves.value, p.value, 0><<<sdp::grid_of(T), waves.value * 64, 0, s>>>(a);
        });
        rc = sdp::launch_status();
    }
    if (rc != SDP_OK || !loss) return rc;
    return sdp::loss_sum(nll, T, scale, scale_dev, loss, s);
}

extern "C" int sdp_label_scale(int id_type, int T, int V, const void* labels, float* scale, void* stream) {
    if (id_type != SDP_I32 && id_type != SDP_I64) return SDP_ERR_INVALID_ARG;
    if (T < 0 || V < 1 || !scale || (T > 0 && !labels)) return SDP_ERR_INVALID_ARG;
    if (T > SDP_MAX_EXTENT || V > SDP_MAX_EXTENT) return SDP_ERR_SHAPE;
    if (!sdp::aligned_to(labels, id_type == SDP_I64 ? 8 : 4) || !sdp::aligned_to(scale, 4)) return SDP_ERR_INVALID_ARG;
    if (T > 0 && sdp::overlap({{scale, 4}}, {{labels, (size_t)T * (id_type == SDP_I64 ? 8 : 4)}})) return SDP_ERR_INVALID_ARG;
    sdp::ProfileScope ps("label_scale", (hipStream_t)stream);
    if (id_type == SDP_I64) label_scale_kernel<1><<<1, 1024, 0, (hipStream_t)stream>>>(labels, T, V, scale);
    else label_scale_kernel<0><<<1, 1024, 0, (hipStream_t)stream>>>(labels, T, V, scale);
    return sdp::launch_status();
}
