// The rules on sizes by which the host takes one path or another. Plain C++
// without HIP, so that the tests compile them and choose their pools by them.
#pragma once

#include <stdint.h>

namespace pace {

// Pools up to this size are selected by the multi-workgroup rank-by-counting
// kernel; larger pools by the single-workgroup radix select.
constexpr int64_t kRankMaxN = 8192;

// ---- scores by trajectory (score_traj.hip) ----------------------------------
constexpr int64_t kTrajCap = 65536;                // tokens one workgroup of four or eight waves sums, at least
constexpr int64_t kTrajOverMax = 4096;             // piece workgroups, at most (the cap grows instead)
constexpr int64_t kTrajFillWaves = 4096;           // waves that few trajectories are spread over

// Waves that take a trajectory, from the mean length: enough bytes for each
// that its start and end (about 3 us) hide under the others' streams, and
// enough waves for the chip when there are few trajectories. Whole steps, 1 / 2
// / 4 / 8 waves: 8192 trajectories of 1464 tokens 38.9 / 39.4 / 41.4 / 53.0 us,
// of 1953 42.0 / 42.2 / 43.4 / 54.5, 8000 of 3500 54.3 / 54.0 / 53.8 / 63.0,
// 4096 of 6103 42.0 / 41.0 / 39.4 / 41.4, of 12,207 75.7 / 75.0 / 70.6 / 67.1.
inline int traj_waves(int64_t n, int64_t n_tokens) {
    const int64_t mean = n_tokens / n;
    const int want = mean >= 8192 ? 8 : (mean >= 2560 ? 4 : (mean >= 1536 ? 2 : 1));
    int fill = 1;
    while (fill < 8 && fill * 2 * n <= kTrajFillWaves) fill *= 2;
    return want > fill ? want : fill;
}

// Whether the score is formed by trajectory rather than over equal chunks of
// tokens. Chunks remain for many short trajectories, where a trajectory does
// not fill a wave's loads: 16,384 trajectories of 2500 tokens take 75 us a step
// by chunks and 78 by trajectory, of 3200 90.4 and 89.2, 8200 of 5000 69 and 65.
inline bool score_by_traj(int64_t n, int64_t n_tokens) { return n <= kRankMaxN || n_tokens / n >= 3072; }

// The most tokens that one workgroup then sums.
inline int64_t score_traj_cap(int64_t n, int64_t n_tokens) {
    if (n == 0) return kTrajCap;
    const int kw = traj_waves(n, n_tokens);
    const int64_t least = kw >= 4 ? kTrajCap : kTrajCap / 4 * kw;
    const int64_t per = n_tokens / kTrajOverMax;
    return per <= least ? least : (per + least - 1) / least * least;
}

// Whether a thread's sum of tags + 1 stays below 2^32: tags are at most V (a
// precondition), and a thread sums at most cap / (64 waves) of them.
inline bool score_traj_narrow(int64_t n, int64_t n_tokens, int32_t V) {
    return (int64_t)V + 1 <= ((((int64_t)1 << 32) - 1) / (score_traj_cap(n, n_tokens) / (64 * traj_waves(n, n_tokens))));
}

// ---- scores over chunks of tokens (score.hip) -------------------------------
// Arithmetic of the reduction; tags are at most V, so tag + 1 <= V + 1.
//   kPacked  every tag + 1 < 2^15: sum and count in one 32-bit number
//   kNarrow  every tag + 1 < 2^24: 32-bit sums of a window, counts apart
//   kWideTags  64-bit sums
enum ReduceMode : int { kPacked = 0, kNarrow = 1, kWideTags = 2 };
inline ReduceMode reduce_mode(int32_t V) {
    return (int64_t)V < (1 << 15) - 1 ? kPacked : ((int64_t)V < (1 << 24) - 1 ? kNarrow : kWideTags);
}

// ---- prompt groups (group.hip) -----------------------------------------------
// Group means formed inside the rank over groups (at most kRankMaxN groups):
// every rank workgroup (one per kRankQ groups) reads all member scores, so the
// group step does that while ceil(ng / kRankQ) * n stays within kGroupRankLoads,
// and makes a separate pass of group means before the rank beyond.
constexpr int kRankQ = 16;              // targets per rank workgroup
constexpr int64_t kGroupRankLoads = (int64_t)1 << 21;
inline bool group_means_in_rank(int64_t n, int64_t ng) { return (ng + kRankQ - 1) / kRankQ * n <= kGroupRankLoads; }

// ---- small filter steps (compact.hip) ----------------------------------------
inline int64_t expected_kept(int64_t n, int64_t n_tokens, int64_t kept) {
    return n > 0 ? (int64_t)((double)n_tokens * ((double)kept / (double)n)) : 0;
}

// Whether the selection and compaction of a filter step go in one launch. Every
// workgroup repeats the ranking, so it is for batches that a few hundred
// workgroups copy: expected kept tokens times columns up to kSmallMaxCopy, twice
// that for at most half as many trajectories. Three launches / two, us a step:
// 64 trajectories, 70K tokens 16.4 / 13.4; 64, 1.5M 16.0 / 14.3; 256, 1M 16.1 /
// 14.1; 256, 2M 16.0 / 18.2; 256, 1M in three columns 17.0 / 21.3.
constexpr int64_t kSmallMaxN = 256;
constexpr int64_t kSmallMaxCopy = (int64_t)1 << 19;
inline bool small_step_ok(int64_t n, int64_t n_tokens, int n_cols, int64_t budget) {
    const int64_t most = kSmallMaxCopy * (n <= kSmallMaxN / 2 ? 2 : 1) / (n_cols > 0 ? n_cols : 1);
    return n <= kSmallMaxN && expected_kept(n, n_tokens, n - budget) <= most;
}

// ---- launches of the operators' kernels -----------------------------------------------
// A dimension of a grid holds fewer than 2^32 threads.
constexpr int64_t kGridThreads = ((int64_t)1 << 32) - 1;
// n workgroups in as many launches as that takes: f(first, count) returns 0, or an
// error that ends it.
template <typename F>
inline auto in_launches(int64_t n, int64_t threads, F f) {
    const int64_t most = kGridThreads / threads;
    for (int64_t first = 0;;) {
        const int64_t count = n - first < most ? n - first : most;
        const auto e = f(first, count);
        first += count;
        if ((int)e != 0 || first >= n) return e;
    }
}

// ---- tiles of matrix products (mfma_tile.hpp) --------------------------------------
// The side of a product's square tiles, by the time that each would take, in
// microseconds: a launch, and for every round of workgroups a beginning and an
// end and its steps of 128 bytes. A step costs by what is in flight: the larger
// tiles read less from memory and LDS a multiplication, the smaller ones fill the
// chip and waste less at the edges. Of 64 two workgroups share a CU from a tile
// a CU on, which then cost more each. Measured in binary16: X X^T of 4096 x
// 16384 342 / 281 / 406 / 484 us (256 / 192 / 128 / 64), of 2500 x 2600 56 / 42 /
// 25 / 37, of 1000 x 3001 62 / 44 / 26 / 14; C X of 4096 x 16384 470 / 614 / 664 / 993.
// In 8 bits, where a step has the same bytes and products, it takes the fastest of the
// four in 20 of 21 products of 40 to 4096 tokens, 2048 to 150000 channels and 512 to 5120
// bytes (4096 x 16384 x 4096 224 / 292 / 335 / 439, 512 x 16384 x 2048 28 / 39 / 27 / 34, 64
// x 16384 x 4096 44 / 32 / 20 / 13), and 2000 x 9000 x 2944 in 79 us for 75.
template <typename Tiles>
inline int product_tile(int64_t steps, int64_t cus, Tiles tiles) {
    constexpr int side[4] = {256, 192, 128, 64};
    constexpr double ends[4] = {5.0, 4.0, 3.0, 1.5}, step[4] = {1.65, 1.1, 0.55, 0.19};
    int best = 64;
    double least = 1e300;
    for (int k = 0; k < 4; ++k) {
        const int64_t n = tiles((int64_t)side[k]);
        const bool two = side[k] == 64 && n > cus;
        const int64_t rounds = two ? (n + 2 * cus - 1) / (2 * cus) : (n + cus - 1) / cus;
        const double t = (double)rounds * (ends[k] + (double)steps * (two ? 0.43 : step[k]));
        if (t < least) least = t, best = side[k];
    }
    return best;
}

// The runs that a product's steps are split into where there are few tiles of 64
// and many steps: a second launch, which adds the parts, costs 3 to 5 us, a step
// 0.19. At least 8 steps a part, and three parts that the chip holds at once (two
// of 24 to 64 steps gave nothing: 200.8 us for 199.7). Five steps on an update of
// 256 x 8192 take 138 us in 16 parts (237 whole), of 64 x 4096 92 in 8 (131), of
// 900 x 8000 283 in 4 (336), of 3001 x 1000 193 in 3 (200), of 512 x 2048 121 in 4
// (129); but of 300 x 1000, with 16 steps, 103 in 2 (97).
constexpr int64_t kPartSteps = 8, kPartsMost = 16, kPartJobs = 512;
inline int product_parts(int64_t steps, int64_t tiles) {
    int64_t parts = steps / kPartSteps;
    if (parts > kPartsMost) parts = kPartsMost;
    if (parts * tiles > kPartJobs) parts = kPartJobs / tiles;
    if (parts < 3) return 1;
    const int64_t run = (steps + parts - 1) / parts;
    return (int)((steps + run - 1) / run);           // no part without a step
}
// No fewer parts times tiles than any product of at most these steps and tiles has.
inline int64_t product_jobs_most(int64_t steps, int64_t tiles) {
    int64_t parts = steps / kPartSteps;
    if (parts < 3) return 0;
    if (parts > kPartsMost) parts = kPartsMost;
    return tiles > kPartJobs / parts ? kPartJobs : parts * tiles;
}
// The parts of an 8-bit product's steps: of rows of whole steps that go straight to LDS
// (direct), 48 or more, and not where the kernel for few tokens takes them (matmul_i8.hip).
inline bool i8_few(int64_t m, int64_t n, bool direct, int64_t cus) { return m <= 4 || (m <= 8 && (!direct || (n + 63) / 64 < cus)); }
constexpr int64_t kI8PartSteps = 48;
inline int i8_parts(int64_t m, int64_t n, int64_t k, bool direct, int64_t cus) {
    if (!direct || k < kI8PartSteps * 128 || i8_few(m, n, direct, cus)) return 1;
    return product_parts(k / 128, ((m + 63) / 64) * ((n + 63) / 64));
}
// As many as any product of at most this size has, times its tiles.
inline int64_t i8_jobs_most(int64_t m, int64_t n, int64_t k, int64_t cus) {
    if (k < kI8PartSteps * 128 || i8_few(m, n, true, cus)) return 0;
    return product_jobs_most(k / 128, ((m + 63) / 64) * ((n + 63) / 64));
}

// Columns of X that a workgroup takes where C and C X go in one launch, 0 where they
// do not. A launch and C's round trip through memory cost 4 to 5 us, but each
// workgroup forms its 64 rows of C again: with one strip (mp = 64) that is as much as
// the product, with two it pays while the chip holds most workgroups, with three and
// four, whose operands fill a CU's LDS, while it holds them all. Five steps in us,
// one launch / two: 1 update of 64 x 4096 69 / 87, 256 of 64 x 512 107 / 143, 24 of
// 128 x 512 65 / 78, 128 of them 143 / 149, 256 of 128 x 1024 485 / 441, 4 of 256 x
// 1000 87 / 94 (64 columns), 24 of 256 x 256 78 / 85 (128; with 64 103), 24 of 256 x 512
// 125 / 102. Of 25 batches of 1 to 80 updates of 192 and 256 rows and up to 4096 columns it
// takes the fastest of the three forms in 23: 8 of 192 x 1000 104 (two launches) / 102 (64
// columns) / 85 (128), 16 of 192 x 192 86 / 67 / 70, 48 of 256 x 256 116 / 149 / 127; but 40 of
// 192 x 400 116 / 148 / 109 and 64 of 192 x 192 111 / 125 / 107.
inline int ortho_step_cols(int64_t mp, int64_t n, int64_t batch, int64_t cus) {
    auto jobs = [&](int64_t cols) { return mp / 64 * ((n + cols - 1) / cols) * batch; };
    if (mp == 64) return 64;
    if (mp == 128) return jobs(64) <= 8 * cus ? 64 : 0;
    if (mp > 256) return 0;
    return jobs(64) <= cus ? 64 : jobs(128) <= cus ? 128 : 0;
}

// Updates that a workgroup of 512 threads takes whole, in one launch: X twice and A in
// LDS, 64 elements a thread on the way in. As far as that fits it is faster than the
// launches on the whole chip, alone and in batches; five steps in us: 1 of 64 x 64
// 12 (38), 1 of 64 x 512 34 (48), 1 of 128 x 256 44 (52), 24 of 64 x 64 12 (40),
// 256 of 64 x 512 38 (109), 2000 of 128 x 256 375 (1159).
inline bool ortho_whole(int64_t mp, int64_t np) { return (mp == 64 && np <= 512) || (mp == 128 && np <= 256); }

// Updates of a batch that one launch of a product's 64 x 64 tiles takes (512 threads
// each): all but of the longest and lowest, of which 256 of 1 x 2^21 are too many.
inline int64_t ortho_batch_most(int64_t m, int64_t n) {
    const int64_t most = kGridThreads / 512 / (((m + 63) / 64) * ((n + 63) / 64));
    return most < 1 ? 1 : most;
}

// ---- policy loss (policy_loss.hip) ------------------------------------------------
// Tokens a wave takes: 256 are one load a lane; at least that, at most
// what leaves 8192 waves, which the chip holds at once.
constexpr int64_t kLossSpanMin = 256;
inline int64_t policy_loss_span(int64_t n_tokens) {
    const int64_t per = (n_tokens / 8192 + 255) / 256 * 256;
    return per > kLossSpanMin ? per : kLossSpanMin;
}
// No fewer spans than any batch of at most n_tokens has: a span is at least
// n_tokens / 8192, rounded down, and that at least 256 where it is not the least.
inline int64_t policy_loss_spans_most(int64_t n_tokens) {
    const int64_t spans = (n_tokens + kLossSpanMin - 1) / kLossSpanMin;
    return spans < 8192 + 32 ? spans : 8192 + 32;
}

// ---- log-probabilities (logprob.hip) --------------------------------------------
// A row of logits is taken by `parts` waves (waves = 1) or workgroups of eight
// waves (8): enough of them for the chip, at most 64, one a lane of the joining
// wave. A wave takes parts up to kLogprobWave logits, of at least
// kLogprobWaveMin; a part's beginning and end cost a workgroup more than its
// logits where these are few. A wave's 64 threads bound up to 32 alternatives
// well; more are left to the workgroup's 512.
struct LogprobPlan {
    int waves;
    int64_t parts;
};
constexpr int64_t kLogprobWaves = 4096, kLogprobWaveMin = 4096, kLogprobWave = 16384;
constexpr int64_t kLogprobGroups = 2048, kLogprobGroupMin = 8192;
inline LogprobPlan logprob_plan(int64_t rows, int64_t vocab, int top_k) {
    auto parts = [&](int64_t fill, int64_t least) {
        const int64_t want = rows > 0 ? (fill + rows - 1) / rows : 1, most = vocab / least;
        const int64_t p = want < most ? want : most;
        return p < 1 ? (int64_t)1 : (p > 64 ? (int64_t)64 : p);
    };
    const int64_t w = parts(kLogprobWaves, kLogprobWaveMin);
    if (top_k <= 32 && vocab / w <= kLogprobWave) return {1, w};
    return {8, parts(kLogprobGroups, kLogprobGroupMin)};
}
// The backward pass has nothing to join: parts of 16,384 logits, as far as one
// launch of workgroups of kLpbThreads holds them.
constexpr int kLpbThreads = 256;
inline int64_t logprob_backward_parts(int64_t rows, int64_t vocab) {
    const int64_t parts = (vocab + 16383) / 16384, most = rows > 0 ? kGridThreads / kLpbThreads / rows : 1;
    return most < 1 ? 1 : (parts < most ? parts : most);
}

}  // namespace pace
