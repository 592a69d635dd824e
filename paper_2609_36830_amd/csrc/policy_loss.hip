// The clipped policy loss of a packed batch with its gradient, for gfx950.
// Per response token (tag != -1) of a trajectory with advantage A, with
// d = lp_new - lp_behavior in binary32, r = e^d and k = scale weight A:
//   A > 0:  loss = -k min(r, 1 + eh),            gradient -k r while d <= log(1 + eh)
//   A < 0:  loss = -k min(max(r, 1 - el), c),    gradient -k r while log(1 - el) <= d <= log c
// and the divergence estimate e^d - 1 - d. The bounds are compared in d, which
// the definition rounds once, so that both sides of a bound are exact. Within
// a trajectory every loss has one sign: the sums by trajectory do not cancel.
//
// HBM-bound: 8 bytes read a token (12 with tags), 4 written. One wave takes one
// span of consecutive tokens and walks the trajectories in it, 64 of their
// ends, advantages and weights at a time. A trajectory inside a span is summed
// and written there; one that crosses a span's end leaves its parts in the
// spans' head and tail slots, which a second kernel adds in span order, one
// wave a trajectory. Sums are binary64, so results repeat bit for bit and do
// not depend on the span by more than its rounding.
#include "elem.hpp"
#include "kernels.hpp"

#pragma clang fp contract(off)

namespace pace {

namespace {

constexpr int kLossWaves = 4;          // waves of a workgroup
constexpr int kLossPer = 4;            // consecutive tokens of a lane

struct LossSum {
    double loss, kl;
    int64_t clipped;
};

__device__ __forceinline__ LossSum wave_total(LossSum v) {
#pragma unroll
    for (int off = kWave / 2; off >= 1; off >>= 1) {
        v.loss += __shfl_xor(v.loss, off, kWave);
        v.kl += __shfl_xor(v.kl, off, kWave);
        v.clipped += __shfl_xor((long long)v.clipped, off, kWave);
    }
    return v;
}

// e^d - 1 - d. By its series for small d, where the difference would cancel
// (at 0.7 the terms left out are below 2^-28 of the sum).
__device__ __forceinline__ float exp_rest(float d, float r) {
    if (!(__builtin_fabsf(d) < 0.7f)) return (r - 1.0f) - d;
    float s = 1.0f;
#pragma unroll
    for (int k = 11; k >= 3; --k) s = __builtin_fmaf(d * (1.0f / (float)k), s, 1.0f);
    return 0.5f * d * d * s;
}

struct TokenLoss {
    float grad, loss, kl;
    bool cut;
};
__device__ __forceinline__ TokenLoss token_loss(float lp_new, float lp_beh, float k, const LossBounds &b) {
    const float d = lp_new - lp_beh;
    const float r = expf(d);
    TokenLoss t;
    const bool up = k > 0.0f && d > b.log_high, down = k < 0.0f && d < b.log_low, far = k < 0.0f && d > b.log_dual;
    t.cut = up || down || far;
    const float rc = up ? b.high : (down ? b.low : (far ? b.dual : r));
    // No advantage, no gradient, whatever the ratio.
    t.loss = k == 0.0f ? 0.0f : -k * rc;
    t.grad = t.cut || k == 0.0f ? 0.0f : -k * r;
    t.kl = exp_rest(d, r);
    return t;
}

template <bool kTags>
__global__ __launch_bounds__(kLossWaves * kWave) void policy_loss_kernel(
    const float *__restrict__ lp_new, const float *__restrict__ lp_beh, const int32_t *__restrict__ tags,
    const int64_t *__restrict__ off, int64_t n, int64_t nt, const float *__restrict__ adv,
    const float *__restrict__ weight, double scale, LossBounds bounds, int64_t span, float *__restrict__ grad,
    float *__restrict__ loss, float *__restrict__ kl, int32_t *__restrict__ clipped, LossSum *__restrict__ slots) {
    const int64_t wave = (int64_t)blockIdx.x * kLossWaves + threadIdx.x / kWave;
    const int64_t p0 = wave * span;
    if (p0 >= nt) return;                            // whole waves; no barrier below
    const int64_t p1 = p0 + span < nt ? p0 + span : nt;
    const int lane = lane_id();
    auto zero = [&](int64_t from, int64_t to) {       // tokens of no trajectory
        for (int64_t q = from + lane; q < to; q += kWave) grad[q] = 0.0f;
    };
    int64_t i = wave_last_le(off, n, p0);
    int64_t pos = p0;
    if (i < 0) {
        i = 0;
        const int64_t first = readlane_i64(clamp64(off[0], p0, p1), 0);
        zero(p0, first);
        pos = first;
    }
    bool inside = i < n && readlane_i64(off[i], 0) >= p0;      // trajectory i starts in this span
    while (pos < p1 && i < n) {
        // the next 64 trajectories, one a lane
        const int64_t mine = i + lane;
        const int64_t my_end = mine < n ? clamp64(off[mine + 1], 0, nt) : nt;
        float my_k = 0.0f;
        if (mine < n) my_k = (float)(scale * (weight ? (double)weight[mine] : 1.0) * (double)adv[mine]);
        const int64_t left = n - i;
        const int most = left < kWave ? (int)left : kWave;
        int j = 0;
        for (; j < most && pos < p1; ++j) {
            const int64_t end_all = readlane_i64(my_end, j);
            const int64_t end = end_all < p1 ? end_all : p1;
            if (end > pos) {
                const float k = __builtin_bit_cast(float, readlane_i32(__builtin_bit_cast(int32_t, my_k), j));
                LossSum sum = {0.0, 0.0, 0};
                for (int64_t base = pos; base < end; base += kWave * kLossPer) {
                    const int64_t q = base + (int64_t)lane * kLossPer;
                    float a[kLossPer], b[kLossPer], g[kLossPer];
                    bool live[kLossPer];
                    const bool whole = q + kLossPer <= end;
                    if (whole) {
                        const uint4 x = load_a4(lp_new + q), y = load_a4(lp_beh + q);
                        unpack16<float>(x, a);
                        unpack16<float>(y, b);
                        if (kTags) {
                            const uint4 w = load_a4(tags + q);
                            live[0] = (int32_t)w.x != -1, live[1] = (int32_t)w.y != -1;
                            live[2] = (int32_t)w.z != -1, live[3] = (int32_t)w.w != -1;
                        } else {
#pragma unroll
                            for (int e = 0; e < kLossPer; ++e) live[e] = true;
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < kLossPer; ++e) {
                            const bool in = q + e < end;
                            a[e] = in ? lp_new[q + e] : 0.0f;
                            b[e] = in ? lp_beh[q + e] : 0.0f;
                            live[e] = in && (!kTags || tags[q + e] != -1);
                        }
                    }
#pragma unroll
                    for (int e = 0; e < kLossPer; ++e) {
                        const TokenLoss t = token_loss(a[e], b[e], k, bounds);
                        g[e] = live[e] ? t.grad : 0.0f;
                        sum.loss += live[e] ? (double)t.loss : 0.0;
                        sum.kl += live[e] ? (double)t.kl : 0.0;
                        sum.clipped += live[e] && t.cut ? 1 : 0;
                    }
                    if (whole) {
                        *reinterpret_cast<pace_v4u_a4 *>(grad + q) =
                            pace_v4u_a4{__builtin_bit_cast(uint32_t, g[0]), __builtin_bit_cast(uint32_t, g[1]),
                                        __builtin_bit_cast(uint32_t, g[2]), __builtin_bit_cast(uint32_t, g[3])};
                    } else {
#pragma unroll
                        for (int e = 0; e < kLossPer; ++e)
                            if (q + e < end) grad[q + e] = g[e];
                    }
                }
                sum = wave_total(sum);
                if (lane == 0) {
                    if (inside && end_all <= p1) {
                        loss[i + j] = (float)sum.loss;
                        if (kl) kl[i + j] = (float)sum.kl;
                        if (clipped) clipped[i + j] = (int32_t)sum.clipped;
                    } else {
                        slots[2 * wave + (inside ? 1 : 0)] = sum;      // head slot for what began before
                    }
                }
                pos = end;
            }
            if (pos < p1) inside = true;             // the next trajectory starts here
        }
        i += j;
    }
    zero(pos, p1);
}

// One wave a trajectory: zeros for an empty one, the slots' sum for one that
// crosses spans.
__global__ __launch_bounds__(kLossWaves * kWave) void policy_loss_join_kernel(
    const int64_t *__restrict__ off, int64_t n, int64_t nt, int64_t span, const LossSum *__restrict__ slots,
    float *__restrict__ loss, float *__restrict__ kl, int32_t *__restrict__ clipped) {
    const int64_t i = (int64_t)blockIdx.x * kLossWaves + threadIdx.x / kWave;
    if (i >= n) return;
    const int lane = lane_id();
    const int64_t lo = clamp64(off[i], 0, nt), hi = clamp64(off[i + 1], 0, nt);
    LossSum sum = {0.0, 0.0, 0};
    if (hi > lo) {
        const int64_t s0 = lo / span, s1 = (hi - 1) / span;
        if (s0 == s1) return;                        // written by its span
        for (int64_t s = s0 + lane; s <= s1; s += kWave) {
            const LossSum part = slots[2 * s + (s == s0 ? 1 : 0)];
            sum.loss += part.loss;
            sum.kl += part.kl;
            sum.clipped += part.clipped;
        }
        sum = wave_total(sum);
    }
    if (lane == 0) {
        loss[i] = (float)sum.loss;
        if (kl) kl[i] = (float)sum.kl;
        if (clipped) clipped[i] = (int32_t)sum.clipped;
    }
}

}  // namespace

size_t policy_loss_ws_bytes(int64_t n_tokens) {
    const int64_t span = policy_loss_span(n_tokens), spans = (n_tokens + span - 1) / span;
    return align256((size_t)spans * 2 * sizeof(LossSum)) + 256;
}

hipError_t launch_policy_loss(const float *lp_new, const float *lp_beh, const int32_t *tags, const int64_t *offsets,
                              int64_t n, int64_t n_tokens, const float *adv, const float *weight, double scale,
                              const LossBounds &bounds, float *grad, float *loss, float *kl, int32_t *clipped, void *ws,
                              hipStream_t stream) {
    const int64_t span = policy_loss_span(n_tokens), spans = (n_tokens + span - 1) / span;
    LossSum *slots = (LossSum *)ws;
    hipError_t e = hipSuccess;
    if (spans > 0) {
        const dim3 grid((unsigned)((spans + kLossWaves - 1) / kLossWaves)), block(kLossWaves * kWave);
        e = tags ? launch(kPhaseAux, policy_loss_kernel<true>, grid, block, stream, lp_new, lp_beh, tags, offsets, n, n_tokens,
                          adv, weight, scale, bounds, span, grad, loss, kl, clipped, slots)
                 : launch(kPhaseAux, policy_loss_kernel<false>, grid, block, stream, lp_new, lp_beh, tags, offsets, n, n_tokens,
                          adv, weight, scale, bounds, span, grad, loss, kl, clipped, slots);
    }
    if (e == hipSuccess && n > 0)
        e = launch(-1, policy_loss_join_kernel, dim3((unsigned)((n + kLossWaves - 1) / kLossWaves)),
                   dim3(kLossWaves * kWave), stream, offsets, n, n_tokens, span, (const LossSum *)slots, loss, kl, clipped);
    return e;
}

}  // namespace pace
