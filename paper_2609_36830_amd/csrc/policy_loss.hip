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
// span of consecutive tokens, 256 a round, four consecutive ones a lane; a
// round's bytes are on their way while the trajectories of the one before are
// summed. The trajectories' ends and factors are taken 64 at a time, one a lane;
// a round that several trajectories meet in is summed once for each. A
// trajectory inside a span is written there; one that crosses a span's end
// leaves its parts in the spans' head and tail slots, which a second kernel adds
// in span order, one wave a trajectory. Sums are binary64, in a fixed order.
// 16.8M tokens with tags take 64.8 us (4.2 TB/s, 50 of them the first kernel's
// where nothing else holds the caches; a device copy 4.8 TB/s), 2.5M without 14.6:
// there two launches and one round's dependent chain (bytes, exponentials, sums,
// slots) are 8 us.
#include "elem.hpp"
#include "kernels.hpp"

#pragma clang fp contract(off)

namespace pace {

namespace {

constexpr int kLossWaves = 4;          // waves of a workgroup
constexpr int kLossPer = 4;            // consecutive tokens of a lane
constexpr int kLossRound = kWave * kLossPer;

struct LossSum {
    double loss, kl;
    int64_t clipped;
};

// Sums in lane order's tree (row shifts and row broadcasts), in every lane.
__device__ __forceinline__ double wave_total_f64(double v) {
    auto step = [&](uint64_t got) { v += __builtin_bit_cast(double, got); };
    step(dpp_u64<0x111, 0xf>(0ull, __builtin_bit_cast(uint64_t, v)));
    step(dpp_u64<0x112, 0xf>(0ull, __builtin_bit_cast(uint64_t, v)));
    step(dpp_u64<0x114, 0xf>(0ull, __builtin_bit_cast(uint64_t, v)));
    step(dpp_u64<0x118, 0xf>(0ull, __builtin_bit_cast(uint64_t, v)));
    step(dpp_u64<0x142, 0xa>(0ull, __builtin_bit_cast(uint64_t, v)));
    step(dpp_u64<0x143, 0xc>(0ull, __builtin_bit_cast(uint64_t, v)));
    return __builtin_bit_cast(double, readlane_i64(__builtin_bit_cast(int64_t, v), kWave - 1));
}
__device__ __forceinline__ LossSum wave_total(const LossSum &v) {
    return {wave_total_f64(v.loss), wave_total_f64(v.kl), wave_sum_i64(v.clipped)};
}

// e^d within four units of 2^-24 up to the largest number, zero below 2^-126, by
// 2^(d log2 e) with what the product leaves: a third of the library function's
// instructions, which bound the small batches.
__device__ __forceinline__ float exp_of(float d) {
    constexpr float hi = 1.44269502162933349609375f, lo = 1.92596299112661746887e-8f;      // log2 e
    const float t = d * hi;
    float rest = __builtin_fmaf(d, lo, __builtin_fmaf(d, hi, -t));
    rest = __builtin_fabsf(t) < 192.0f ? rest : 0.0f;      // no number for infinities, too much far beyond the range
    return __builtin_amdgcn_exp2f(t) * __builtin_fmaf(rest, 0.693147180559945309f, 1.0f);
}
// e^d - 1 - d. By its series for small d, where the difference would cancel
// (at 0.7 the terms left out are below 2^-28 of the sum).
__device__ __forceinline__ float exp_rest(float d, float r) {
    float s = 1.0f / 39916800.0f;
    s = __builtin_fmaf(s, d, 1.0f / 3628800.0f);
    s = __builtin_fmaf(s, d, 1.0f / 362880.0f);
    s = __builtin_fmaf(s, d, 1.0f / 40320.0f);
    s = __builtin_fmaf(s, d, 1.0f / 5040.0f);
    s = __builtin_fmaf(s, d, 1.0f / 720.0f);
    s = __builtin_fmaf(s, d, 1.0f / 120.0f);
    s = __builtin_fmaf(s, d, 1.0f / 24.0f);
    s = __builtin_fmaf(s, d, 1.0f / 6.0f);
    s = __builtin_fmaf(s, d, 0.5f);
    return __builtin_fabsf(d) < 0.7f ? d * d * s : (r - 1.0f) - d;
}

struct TokenLoss {
    float grad, loss;
    bool cut;
};
// r = e^d.
__device__ __forceinline__ TokenLoss token_loss(float d, float r, float k, const LossBounds &b) {
    TokenLoss t;
    const bool up = k > 0.0f && d > b.log_high, down = k < 0.0f && d < b.log_low, far = k < 0.0f && d > b.log_dual;
    t.cut = up || down || far;
    const float rc = up ? b.high : (down ? b.low : (far ? b.dual : r));
    // No advantage, no gradient, whatever the ratio.
    t.loss = k == 0.0f ? 0.0f : -k * rc;
    t.grad = t.cut || k == 0.0f ? 0.0f : -k * r;
    return t;
}

// Four consecutive tokens from q on, those at or past `end` as zeros.
__device__ __forceinline__ uint4 load_four(const void *a, int64_t q, int64_t end) {
    const uint32_t *p = reinterpret_cast<const uint32_t *>(a) + q;
    if (q + kLossPer <= end) return load_a4(p);
    uint4 v = make_uint4(0, 0, 0, 0);
    if (q < end) v.x = p[0];
    if (q + 1 < end) v.y = p[1];
    if (q + 2 < end) v.z = p[2];
    return v;
}

template <bool kTags>
__global__ __launch_bounds__(kLossWaves * kWave) void policy_loss_kernel(
    const float *__restrict__ lp_new, const float *__restrict__ lp_beh, const int32_t *__restrict__ tags,
    const int64_t *__restrict__ off, int64_t n, int64_t nt, const float *__restrict__ adv,
    const float *__restrict__ weight, double scale, LossBounds bounds, int64_t span, float *__restrict__ grad,
    float *__restrict__ loss, float *__restrict__ kl, int32_t *__restrict__ clipped, LossSum *__restrict__ slots) {
    const int64_t wave = (int64_t)blockIdx.x * kLossWaves + readlane_i32((int)threadIdx.x / kWave, 0);
    const int64_t p0 = wave * span;
    if (p0 >= nt) return;                            // whole waves; no barrier below
    const int64_t p1 = p0 + span < nt ? p0 + span : nt;
    const int lane = lane_id();
    const int64_t batch = readlane_i64(clamp64(off[n], 0, nt), 0), live1 = batch < p1 ? batch : p1;      // tokens behind it are not read
    uint4 a, b, w = make_uint4(0, 0, 0, 0);
    auto load = [&](int64_t base) {
        const int64_t q = base + (int64_t)lane * kLossPer;
        if (base + kLossRound <= live1) {            // the whole wave: no load behind a branch of its own
            a = load_a4(lp_new + q);
            b = load_a4(lp_beh + q);
            if (kTags) w = load_a4(tags + q);
        } else {
            a = load_four(lp_new, q, live1);
            b = load_four(lp_beh, q, live1);
            if (kTags) w = load_four(tags, q, live1);
        }
    };
    load(p0);

    int64_t i = wave_last_le(off, n, p0);            // the trajectory at pos, or the first behind it
    int64_t pos = p0;
    if (i < 0) {
        i = 0;
        pos = readlane_i64(clamp64(off[0], p0, p1), 0);      // tokens before the first trajectory
    }
    bool inside = i < n && readlane_i64(off[i < n ? i : n], 0) >= p0;      // trajectory i starts in this span
    // The next 64 trajectories from i on, one a lane, and where i is among them.
    int64_t my_end = 0;
    float my_k = 0.0f;
    int at = 0;
    auto take = [&]() {
        const int64_t mine = i + lane;
        my_end = mine < n ? clamp64(off[mine + 1], 0, nt) : nt;
        my_k = mine < n ? (float)(scale * (weight ? (double)weight[mine] : 1.0) * (double)adv[mine]) : 0.0f;
        at = 0;
    };
    int64_t end = nt;
    float k = 0.0f;
    // Trajectory i's end and factor, passing those that end at or before pos; behind the last, the span's end.
    auto at_pos = [&]() {
        for (;;) {
            if (i >= n) {
                end = p1;
                return;
            }
            if (at == kWave) take();
            end = readlane_i64(my_end, at);
            k = __builtin_bit_cast(float, readlane_i32(__builtin_bit_cast(int32_t, my_k), at));
            if (end > pos) return;
            ++i;
            ++at;
            inside = true;
        }
    };
    take();
    at_pos();
    LossSum sum = {0.0, 0.0, 0};
    for (int64_t base = p0; base < p1; base += kLossRound) {
        const int64_t q = base + (int64_t)lane * kLossPer, next = base + kLossRound;
        float x[kLossPer], y[kLossPer], d[kLossPer], r[kLossPer], g[kLossPer];
        bool live[kLossPer];
        unpack16<float>(a, x);
        unpack16<float>(b, y);
        const uint32_t tag[kLossPer] = {w.x, w.y, w.z, w.w};
        if (next < p1) load(next);
#pragma unroll
        for (int e = 0; e < kLossPer; ++e) {
            live[e] = !kTags || (int32_t)tag[e] != -1;
            d[e] = x[e] - y[e];
            r[e] = exp_of(d[e]);
            y[e] = exp_rest(d[e], r[e]);
            g[e] = 0.0f;
        }
        const int64_t stop = next < p1 ? next : p1;
        while (pos < stop) {
            const int64_t to = end < stop ? end : stop;
            if (i < n) {
                const int from = (int)(pos - base) - lane * kLossPer, until = (int)(to - base) - lane * kLossPer;
#pragma unroll
                for (int e = 0; e < kLossPer; ++e) {
                    const bool in = live[e] && e >= from && e < until;
                    const TokenLoss t = token_loss(d[e], r[e], k, bounds);
                    g[e] = in ? t.grad : g[e];
                    sum.loss += (double)(in ? t.loss : 0.0f);
                    sum.kl += (double)(in ? y[e] : 0.0f);
                    sum.clipped += in && t.cut ? 1 : 0;
                }
            }
            pos = to;
            if (i < n && (end <= pos || pos == p1)) {      // ends here, or the span does
                const LossSum all = wave_total(sum);
                if (lane == 0) {
                    if (inside && end <= pos) {
                        loss[i] = (float)all.loss;
                        if (kl) kl[i] = (float)all.kl;
                        if (clipped) clipped[i] = (int32_t)all.clipped;
                    } else {
                        slots[2 * wave + (inside ? 1 : 0)] = all;      // head slot for what began before
                    }
                }
                sum = {0.0, 0.0, 0};
            }
            if (pos < p1 && end <= pos) at_pos();
        }
        if (next <= p1 || q + kLossPer <= p1) {
            *reinterpret_cast<pace_v4u_a4 *>(grad + q) =
                pace_v4u_a4{__builtin_bit_cast(uint32_t, g[0]), __builtin_bit_cast(uint32_t, g[1]), __builtin_bit_cast(uint32_t, g[2]),
                            __builtin_bit_cast(uint32_t, g[3])};
        } else {
#pragma unroll
            for (int e = 0; e < kLossPer; ++e)
                if (q + e < p1) grad[q + e] = g[e];
        }
    }
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

static size_t loss_ws_of(int64_t spans) { return align256((size_t)spans * 2 * sizeof(LossSum)) + 256; }
size_t policy_loss_ws_bytes(int64_t n_tokens) {
    const int64_t span = policy_loss_span(n_tokens);
    return loss_ws_of((n_tokens + span - 1) / span);
}
size_t policy_loss_ws_most(int64_t n_tokens) { return loss_ws_of(policy_loss_spans_most(n_tokens)); }

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
        e = in_launches((n + kLossWaves - 1) / kLossWaves, kLossWaves * kWave, [&](int64_t b, int64_t blocks) {
            const int64_t i = b * kLossWaves;
            return launch(-1, policy_loss_join_kernel, dim3((unsigned)blocks), dim3(kLossWaves * kWave), stream, offsets + i, n - i, n_tokens,
                          span, (const LossSum *)slots, loss + i, kl ? kl + i : nullptr, clipped ? clipped + i : nullptr);
        });
    return e;
}

}  // namespace pace
