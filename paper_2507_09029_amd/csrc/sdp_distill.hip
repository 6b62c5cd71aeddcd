// Divergence of rows of logits from a teacher of whom k entries a token are known, with the gradient from the same read of the logits.
//
//   q_i = exp(v_i / tau - L),  Q = sum q_i,  lse = log sum_j exp(z_j / tau),  kl = sum_i q_i (log q_i - z_id_i / tau + lse)
//   dz_j = c / tau (Q exp(z_j / tau - lse) - sum_{i : id_i = j} q_i)
//
// Bound by memory, like the token loss: one read and one write of the logits, k entries a row beside them. A workgroup holds a row in
// registers from the read to the write (by_row).  While it arrives, a thread an entry fetches its logit again and makes q, which goes through LDS to the
// wave that holds the entry's element (stored without and written anew behind a barrier by the entry's thread, 8192 x 32000 with 64 entries
// took 252 us).  Above 98304 bf16 logits (fp32 49152) 16 waves of 16 pieces spill 20 (28) registers beside the entries' state: 1000 x 128256 124 us, 4.1 TB/s; above
// 131072 (65536) the row is read three times: 1000 x 131073 186 us.
#include <cmath>
#include <type_traits>

#include "sdp_internal.h"
#include "sdp_loss_rows.h"
#include "sdp_targets.h"

namespace {

using sdp::kLog2e;
using sdp::Row;
using sdp::TargetRows;
using sdp::u32x4;

// PIECES > 0: pieces a lane holds, the row has no more; 0: the row is read again for the sum, and again for the gradient
template <int BF16, int WAVES, int PIECES, int ONCE>
__global__ __launch_bounds__(WAVES * 64) void target_rows_kernel(TargetRows a) {
    typedef Row<BF16> Rw;
    typedef typename Rw::Elem Elem;
    constexpr int N = Rw::N, TH = WAVES * 64, P = PIECES ? PIECES : 1;
    __shared__ float lds[3][2][WAVES];
    extern __shared__ unsigned char entry_lds[];
    const int64_t row = sdp::group_id();
    if (row >= a.rows) return;
    const int tid = threadIdx.x, V = a.V, whole = Rw::whole(V), k = a.t.k;
    const Elem* z = (const Elem*)a.Z + row * a.ldz;
    Elem* dz = (Elem*)a.dZ + row * a.ldz;
    const bool tail = whole + tid < V; // this lane has a value behind the whole pieces
    const int listed = a.list ? a.list[row] : (int)row;
    const int token = listed < 0 ? -1 - listed : listed;
    const sdp::Entries en(entry_lds, k);
    if (listed < 0 || !sdp::has_entry(a.t, token, V)) { // every wave finds out for itself: a barrier less before the row is requested
        if (tid == 0) {
            a.kl[token] = 0.f;
            if (a.lse) a.lse[token] = 0.f;
        }
        if (a.dZ) {
            for (int64_t e = tid * N; e < whole; e += TH * N) Rw::store(dz, (int)e, whole, u32x4{0, 0, 0, 0});
            if (tail) Rw::put(dz + whole + tid, 0.f);
        }
        return;
    }
    u32x4 w[P];
    auto piece = [&](int64_t e) { return Rw::mine(Rw::load(z, (int)e, whole), (int)e, whole, sdp::minus_inf<BF16>()); }; // of a row that is read again
    if (PIECES)
#pragma unroll
        for (int i = 0; i < P; ++i) w[i] = Rw::template load<ONCE>(z, (tid + i * TH) * N, whole);
    const float zt = tail ? Rw::one(z + whole + tid) : -INFINITY;
    float vmax = en.load<TH>(a.t, token, V);
    for (int i = tid; i < k; i += TH) en.z[i] = en.id[i] >= 0 ? Rw::one(z + en.id[i]) : 0.f; // before anything is written: dZ may be Z
    float m = zt, sum = 0.f;
    if (PIECES) {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            float v[N];
            w[i] = Rw::mine(w[i], (tid + i * TH) * N, whole, sdp::minus_inf<BF16>());
            Rw::unpack(w[i], v);
#pragma unroll
            for (int j = 0; j < N; ++j) m = fmaxf(m, v[j]);
        }
    } else {
        for (int64_t e = tid * N; e < whole; e += TH * N) {
            float v[N];
            Rw::unpack(piece(e), v);
#pragma unroll
            for (int j = 0; j < N; ++j) m = fmaxf(m, v[j]);
        }
    }
    sdp::group_both<WAVES, true>(m, vmax, lds[0]);
    if (PIECES) sdp::again(w);
    const float rate = kLog2e * a.t.inv_tau;
    auto power = [&](float v) { return __builtin_amdgcn_exp2f((v - m) * rate); };
    float of_entries = en.sum<TH>(a.t, vmax);
    if (tail) sum = power(zt);
    if (PIECES) {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            float v[N];
            Rw::unpack(w[i], v);
#pragma unroll
            for (int j = 0; j < N; ++j) sum += power(v[j]);
        }
    } else { // as in the token loss: a running fp32 sum would drift
        double all = 0.0;
        for (int64_t e = tid * N; e < whole; e += TH * N) {
            float v[N];
            Rw::unpack(piece(e), v);
            float part = 0.f;
#pragma unroll
            for (int j = 0; j < N; ++j) part += power(v[j]);
            all += (double)part;
        }
        sum += (float)all;
    }
    sdp::group_both<WAVES, false>(sum, of_entries, lds[1]);
    if (PIECES) sdp::again(w);
    const float log_sum = logf(sum);
    float mass = 0.f, kl = 0.f;
    en.masses<TH>(a.t, token, vmax, of_entries, [&](int i, float q, float log_q) {
        mass += q;
        if (q != 0.f) kl += q * ((log_q - (en.z[i] - m) * a.t.inv_tau) + log_sum);
    });
    sdp::group_both<WAVES, false>(mass, kl, lds[2]);
    if (!a.t.top_lse && mass == mass) mass = 1.f;
    if (tid == 0) {
        a.kl[token] = kl;
        if (a.lse) a.lse[token] = m * a.t.inv_tau + log_sum;
    }
    if (!a.dZ) return;
    const float c = a.t.scale * (a.t.scale_dev ? *a.t.scale_dev : 1.f) * a.t.inv_tau, inv = c * mass / sum;
    // A lane looks at one entry in 64 of them; those of the 64 pieces that the wave is about to store are found by a vote and taken off by their lanes.
    const int lane = tid & 63;
    const int id0 = lane < k ? en.id[lane] : -1;
    const float q0 = lane < k ? en.q[lane] * c : 0.f;
    auto gradient = [&](int64_t e, const u32x4& x) { // e: this lane's, the wave's others side by side
        float v[N];
        Rw::unpack(x, v);
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = power(v[j]) * inv;
        const int64_t first = e - (int64_t)lane * N;
        auto take_off = [&](int id, float q) {
            uint64_t hits = __ballot(id >= first && id < first + 64 * N);
            while (hits) {
                const int from = __builtin_ctzll(hits);
                hits &= hits - 1;
                const int at = __builtin_amdgcn_readlane(id, from) - (int)e;
                const float off = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(q), from));
#pragma unroll
                for (int j = 0; j < N; ++j) v[j] -= at == j ? off : 0.f;
            }
        };
        take_off(id0, q0);
        for (int i = 64 + lane; i - lane < k; i += 64) take_off(i < k ? en.id[i] : -1, i < k ? en.q[i] * c : 0.f);
        Rw::store(dz, (int)e, whole, Rw::pack(v));
    };
    if (PIECES) {
#pragma unroll
        for (int i = 0; i < P; ++i) gradient((tid + i * TH) * N, w[i]);
    } else {
        for (int64_t e = tid * N; e - (int64_t)lane * N < whole; e += TH * N) gradient(e, piece(e < whole ? e : whole));
    }
    if (tail) {
        float v = power(zt) * inv;
        for (int i = 0; i < k; ++i) v -= en.id[i] == whole + tid ? en.q[i] * c : 0.f;
        Rw::put(dz + whole + tid, v);
    }
}

} // namespace

int sdp::target_rows(int dtype, const TargetRows& r, const char* name, hipStream_t s) {
    if (r.rows < 1) return SDP_OK;
    ProfileScope ps(name, s);
    const bool bf16 = dtype == SDP_BF16, once = read_once({{r.Z, ((size_t)(r.rows - 1) * r.ldz + r.V) * (bf16 ? 2 : 4)}}, (size_t)r.ldz * (bf16 ? 2 : 4));
    const size_t lds = Entries::bytes(r.t.k);
    by_row<false>(bf16, r.V, [&](auto b, auto waves, auto p) {
        if (p.value && once) target_rows_kernel<b.value, waves.value, p.value, p.value != 0><<<grid_of(r.rows), waves.value * 64, lds, s>>>(r);
        else target_rows_kernel<b.value, waves.value, p.value, 0><<<grid_of(r.rows), waves.value * 64, lds, s>>>(r);
    });
    return launch_status();
}

extern "C" int sdp_distill_loss(int dtype, int id_type, int top_dtype, int T, int V, int k, int64_t ldz, float temperature, float scale,
                                const void* Z, const void* ids, const void* top, const float* top_lse, const float* scale_dev, float* kl,
                                float* lse, void* dZ, float* loss, void* stream) {
    if ((dtype != SDP_F32 && dtype != SDP_BF16) || (top_dtype != SDP_F32 && top_dtype != SDP_BF16)) return SDP_ERR_INVALID_ARG;
    if (id_type != SDP_I32 && id_type != SDP_I64) return SDP_ERR_INVALID_ARG;
    if (T < 0 || V < 1 || k < 1 || !sdp::temperature_ok(temperature) || !std::isfinite(scale)) return SDP_ERR_INVALID_ARG;
    if (T > SDP_MAX_EXTENT || V > SDP_MAX_EXTENT || k > SDP_MAX_ENTRIES || ldz < V || ldz > ((int64_t)1 << 40)) return SDP_ERR_SHAPE;
    const size_t es = dtype == SDP_BF16 ? 2 : 4, is = id_type == SDP_I64 ? 8 : 4, ts = top_dtype == SDP_BF16 ? 2 : 4, st = (size_t)T * 4;
    if (T > 0 && (!Z || !ids || !top || !kl)) return SDP_ERR_INVALID_ARG;
    if (!sdp::aligned_to(Z, es) || !sdp::aligned_to(dZ, es) || !sdp::aligned_to(ids, is) || !sdp::aligned_to(top, ts)) return SDP_ERR_INVALID_ARG;
    for (const float* p : {top_lse, scale_dev, (const float*)kl, (const float*)lse, (const float*)loss})
        if (!sdp::aligned_to(p, 4)) return SDP_ERR_INVALID_ARG;
    const size_t rows = T > 0 ? ((size_t)(T - 1) * ldz + V) * es : 0, entries = (size_t)T * k;
    const sdp::Extent eZ{Z, rows}, ei{ids, entries * is}, ev{top, entries * ts}, eL{top_lse, top_lse ? st : 0}, ec{scale_dev, scale_dev ? 4u : 0u},
        on{kl, st}, os{lse, lse ? st : 0}, oz{dZ, dZ ? rows : 0}, o1{loss, loss ? 4u : 0u};
    if (T > 0 && ((dZ != Z && sdp::overlap({oz}, {eZ})) || sdp::overlap({oz, on, os, o1}, {ei, ev, eL, ec}) || sdp::overlap({on, os, o1}, {eZ, oz}) ||
                  sdp::overlap({on}, {os, o1}) || sdp::overlap({os}, {o1})))
        return SDP_ERR_INVALID_ARG;
    hipStream_t s = (hipStream_t)stream;
    sdp::TargetRows r;
    r.Z = Z, r.dZ = dZ, r.ldz = ldz, r.kl = kl, r.lse = lse, r.rows = T, r.V = V;
    r.t = {ids, top, top_lse, k, id_type == SDP_I64, top_dtype == SDP_BF16, 1.f / temperature, scale, scale_dev};
    const int rc = sdp::target_rows(dtype, r, "distill_loss", s);
    if (rc != SDP_OK || !loss) return rc;
    return sdp::loss_sum(kl, T, scale, scale_dev, loss, s);
}
