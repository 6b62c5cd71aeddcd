// Rows of logits in a workgroup's registers (device code): what the token loss and the divergence from a teacher share.
#pragma once
#include <stdint.h>

#include <type_traits>

#include "sdp_rows.h"

namespace sdp {

constexpr float kLog2e = 1.44269504088896340736f;

// maximum / sum over a workgroup, in a fixed order; every thread has the result
template <int WAVES, bool MAX>
__device__ inline float group_all(float x, float* lds) {
    x = MAX ? sdp::wave_max(x) : sdp::wave_sum(x);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = lds[0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) x = MAX ? fmaxf(x, lds[i]) : x + lds[i];
    return x;
}

// value of a piece's word behind the row's end: -inf
template <int BF16>
constexpr uint32_t minus_inf() {
    return BF16 ? 0xFF80FF80u : 0xFF800000u;
}

// Waves of a row and pieces of a lane: the first pair in this order that holds the row.  Few waves leave no lane idle and wait for
// each other less, many keep the registers few enough for two workgroups on a CU, so that one loads while the other computes or stores.  bf16,
// us: 8192 x 1024 two waves of one piece 7, four 12.6; 8192 x 4000 4 x 2 23.3, 8 x 1 30.8; 8192 x 8000 4 x 4 45.7, 8 x 2 48.1, 16 x 1 65.8; 4096 x 16000
// 8 x 4 47.4, 16 x 2 50.9; 8192 x 32000 16 x 4 172, 8 x 8 178, 4 x 16 181; 1000 x 50001 16 x 7 40.5, 8 x 16 43; 1000 x 65536 8 x 16 53.1, 16 x 8 (66
// registers, one workgroup) 59.6.
// LEAN: a kernel that holds five to seven pieces beside all else in 64 registers, of which two workgroups of 16 waves then share a CU (token loss with its sum, 8 x 16
// instead: 1000 x 45001 45.8 -> 50.5 us, 4000 x 50304 141.4 -> 145.1, 16000 x 50304 549 -> 556, fp32 4000 x 25152 137.7 -> 139.9).  The divergence from a
// teacher does not, and does better with 8 x 16: 1000 x 36000 41.7 -> 39.9, 1000 x 50001 52.4 -> 44.8, 4000 x 50304 207 -> 156.
template <bool LEAN = true, class F>
void by_row(int bf16, int V, F&& launch) {
    const int n = bf16 ? 8 : 4;
    auto with = [&](auto b) {
        const int64_t pieces = ((int64_t)V + n - 1) / n;
#define SDP_LOSS_ROW(WAVES, PIECES) \
    if (pieces <= WAVES * 64 * PIECES) return launch(b, std::integral_constant<int, WAVES>{}, std::integral_constant<int, PIECES>{})
        SDP_LOSS_ROW(1, 1);
        SDP_LOSS_ROW(2, 1);
        SDP_LOSS_ROW(4, 1);
        SDP_LOSS_ROW(4, 2);
        SDP_LOSS_ROW(4, 4);
        SDP_LOSS_ROW(8, 3);
        SDP_LOSS_ROW(8, 4);
        SDP_LOSS_ROW(8, 6);
        SDP_LOSS_ROW(16, 4);
        if constexpr (LEAN) {
            SDP_LOSS_ROW(16, 5);
            SDP_LOSS_ROW(16, 6);
            SDP_LOSS_ROW(16, 7);
        }
        SDP_LOSS_ROW(8, 16);
        SDP_LOSS_ROW(16, 12);
        SDP_LOSS_ROW(16, 16);
#undef SDP_LOSS_ROW
        launch(b, std::integral_constant<int, 16>{}, std::integral_constant<int, 0>{});
    };
    if (bf16) with(std::integral_constant<int, 1>{});
    else with(std::integral_constant<int, 0>{});
}

} // namespace sdp
