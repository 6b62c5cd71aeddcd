// A token's targets in a workgroup (device code): the entries of a teacher, or a label, which is one entry of mass 1.
#pragma once
#include <cmath>

#include "sdp_internal.h"
#include "sdp_loss_rows.h"

namespace sdp {

// 1 / temperature is an ordinary fp32 number and differences of logits over it stay far from overflow
inline bool temperature_ok(float t) { return std::isfinite(t) && t >= 9.5367431640625e-7f; }

// two sums, or two maxima, over a workgroup at once, in a fixed order; every thread has both
template <int WAVES, bool MAX>
__device__ inline void group_both(float& x, float& y, float (*lds)[WAVES]) {
    x = MAX ? wave_max(x) : wave_sum(x);
    y = MAX ? wave_max(y) : wave_sum(y);
    if ((threadIdx.x & 63) == 0) lds[0][threadIdx.x >> 6] = x, lds[1][threadIdx.x >> 6] = y;
    __syncthreads();
    x = lds[0][0], y = lds[1][0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) {
        x = MAX ? fmaxf(x, lds[0][i]) : x + lds[0][i];
        y = MAX ? fmaxf(y, lds[1][i]) : y + lds[1][i];
    }
}

// Whether a token has an entry; the same in all lanes of a wave.
__device__ inline bool has_entry(const Targets& t, int64_t token, int V) {
    for (int i = threadIdx.x & 63; i - (int)(threadIdx.x & 63) < t.k; i += 64) {
        bool any = false;
        if (i < t.k) {
            const int64_t at = token * t.k + i;
            const float v = !t.top ? 0.f : t.top_bf16 ? Row<1>::one((const uint16_t*)t.top + at) : ((const float*)t.top)[at];
            any = token_id(t.ids, t.wide, at, V) >= 0 && !(v == -INFINITY);
        }
        if (__any(any)) return true;
    }
    return false;
}

// The entries of one token in LDS; thread t of TH has entries t, t + TH, ..  All but all_of look at a thread's own alone.
struct Entries {
    int* id;     // -1: none
    float *q, *z; // q: first the teacher's logit, then its probability; z: the student's logit, the caller's
    static constexpr size_t bytes(int k) { return (size_t)k * 12; }
    __device__ Entries(unsigned char* lds, int k) : id((int*)lds), q((float*)lds + k), z((float*)lds + 2 * k) {}

    // fetches them; this thread's largest logit, NaN where one is, -inf where it has no entry
    template <int TH>
    __device__ float load(const Targets& t, int token, int V) const {
        float top = -INFINITY;
        for (int i = threadIdx.x; i < t.k; i += TH) {
            const int64_t at = (int64_t)token * t.k + i;
            int j = token_id(t.ids, t.wide, at, V);
            const float v = !t.top ? 0.f : t.top_bf16 ? Row<1>::one((const uint16_t*)t.top + at) : ((const float*)t.top)[at];
            if (v == -INFINITY) j = -1;
            id[i] = j, q[i] = v;
            if (j >= 0) top = v != v || top != top ? NAN : fmaxf(top, v);
        }
        return top;
    }
    // this thread's part of sum_i exp((v_i - vmax) / tau)
    template <int TH>
    __device__ float sum(const Targets& t, float vmax) const {
        float x = 0.f;
        if (t.top && !t.top_lse)
            for (int i = threadIdx.x; i < t.k; i += TH)
                if (id[i] >= 0) x += __builtin_amdgcn_exp2f((q[i] - vmax) * (kLog2e * t.inv_tau));
        return x;
    }
    // q_i and log q_i of every entry of this thread, to `take`; `all` = the workgroup's sum
    template <int TH, class F>
    __device__ void masses(const Targets& t, int token, float vmax, float all, F&& take) const {
        const float log_all = t.top_lse ? t.top_lse[token] : t.top ? logf(all) : 0.f;
        for (int i = threadIdx.x; i < t.k; i += TH) {
            float p = 0.f;
            if (id[i] >= 0) {
                const float log_q = !t.top ? 0.f : t.top_lse ? q[i] * t.inv_tau - log_all : (q[i] - vmax) * t.inv_tau - log_all;
                p = t.top ? __builtin_amdgcn_exp2f(log_q * kLog2e) : 1.f;
                take(i, p, log_q);
            }
            q[i] = p;
        }
    }
    // mass of all entries of entry i's id (behind a barrier after masses); the same bits for each of them
    __device__ float all_of(int i, int k) const {
        const int mine = id[i];
        float x = 0.f;
        for (int j = 0; j < k; ++j) x += id[j] == mine ? q[j] : 0.f;
        return x;
    }
};

} // namespace sdp
