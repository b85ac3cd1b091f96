// Rotary positions of Q and K (gfx950); not a step of the paper.
//
// Every pair of channels (a, b) becomes (a cos - b sin, b cos + a sin) * magnitude.  Each element is read and written once, so memory
// is the bound, if the angles do not cost more: a thread takes the same 8 pairs of up to `steps` heads of a token and computes its
// 8 sines and cosines once for all of them.  Measured in a graph (a copy of the card runs at 4.87 TB/s): 16384 tokens x 40 heads x 128, half
// of the channels turning, 68 us = 4.9 TB/s; 4099 x 48 x 64 11.3 us = 4.5 TB/s; 64 tokens x 40 heads 4.3 us, a launch.
#include "sage_paged.h"

#include <algorithm>

namespace sage {
namespace {

struct RopeArgs {
    const uint16_t *q, *k;
    uint16_t *qo, *ko;
    TokenStrides q_st, qo_st, k_st, ko_st;
    const int32_t *positions;
    int T, Hq, H;  // H = Hq + Hkv
    int steps;     // rows of H * T that a thread takes, 512 / D apart
    int skip_rest; // in place: channels that do not turn stay where they are
    float sign;
};

// A row is one head of one token, row = token * H + head; a wavefront takes `steps` times 64 / (D/16) neighbouring rows.  Lane: 16 channels
// of a row, the 8 pairs 8 i .. 8 i + 7 (half layout: two runs of 8 channels rot/2 apart), or 16 channels that do not turn.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void rope_kernel(const RopeArgs a, const sage_rope_plan plan) {
    constexpr int ITEMS = D / 16, ROWS = 64 / ITEMS;
    const int lane = threadIdx.x & 63, item = lane % ITEMS;
    const int64_t wave = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int64_t row0 = wave * ROWS * a.steps + lane / ITEMS;
    int t = (int)(row0 / a.H), h = (int)(row0 - (int64_t)t * a.H);
    const int half = plan.rot / 2;
    const bool turns = 16 * item < plan.rot;
    if (!turns && a.skip_rest) return;
    const bool halves = turns && plan.layout == SAGE_ROPE_HALF;
    const int c0 = halves ? 8 * item : 16 * item, c1 = halves ? half + 8 * item : 16 * item + 8;
    float cs[8], sn[8];
    int have = -1;
    for (int s = 0; s < a.steps && t < a.T; ++s) {
        const bool is_k = h >= a.Hq;
        const int hh = is_k ? h - a.Hq : h;
        const uint16_t *p = is_k ? a.k + t * a.k_st.t + hh * a.k_st.h : a.q + t * a.q_st.t + hh * a.q_st.h;
        uint16_t *o = is_k ? a.ko + t * a.ko_st.t + hh * a.ko_st.h : a.qo + t * a.qo_st.t + hh * a.qo_st.h;
        uint4 x = *reinterpret_cast<const uint4 *>(p + c0), y = *reinterpret_cast<const uint4 *>(p + c1);
        if (turns) {
            if (t != have) {
                const int pos = a.positions[t];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    rope_angle(pos, plan.turns[8 * item + i], cs[i], sn[i]);
                    cs[i] *= plan.magnitude;
                    sn[i] *= plan.magnitude * a.sign;
                }
                have = t;
            }
            rope_turn<BF16>(halves, cs, sn, x, y);
        }
        *reinterpret_cast<uint4 *>(o + c0) = x;
        *reinterpret_cast<uint4 *>(o + c1) = y;
        for (h += ROWS; h >= a.H; h -= a.H) ++t;
    }
}

}  // namespace

hipError_t launch_rope(const void *q, TokenStrides q_st, void *q_out, TokenStrides qo_st, const void *k, TokenStrides k_st, void *k_out,
                       TokenStrides ko_st, const int32_t *positions, int T, int Hq, int Hkv, int d, const sage_rope_plan &plan,
                       bool transposed, bool bf16, hipStream_t stream) {
    const bool in_place = q == q_out && (!k || k == k_out);
    RopeArgs a{static_cast<const uint16_t *>(q), static_cast<const uint16_t *>(k), static_cast<uint16_t *>(q_out), static_cast<uint16_t *>(k_out),
               q_st, qo_st, k_st, ko_st, positions, T, Hq, Hq + Hkv, 1, in_place, transposed ? -1.0f : 1.0f};
    const int rows = 1024 / d;  // per wavefront and step
    const int64_t all = (int64_t)T * a.H, waves = (all + rows - 1) / rows;
    // a wavefront per token (its heads share the angles) as long as that leaves eight wavefronts to a SIMD
    a.steps = (int)std::min<int64_t>(std::max(1, cdiv(a.H, rows)), std::max<int64_t>(1, waves / (8 * 4 * kCUs)));
    const int64_t groups = (all + 4 * rows * a.steps - 1) / (4 * rows * a.steps);
    const dim3 grid((unsigned)groups), block(256);
    if (d == 128)
        (bf16 ? rope_kernel<128, true> : rope_kernel<128, false>)<<<grid, block, 0, stream>>>(a, plan);
    else
        (bf16 ? rope_kernel<64, true> : rope_kernel<64, false>)<<<grid, block, 0, stream>>>(a, plan);
    return hipGetLastError();
}

}  // namespace sage
