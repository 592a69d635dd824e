// C ABI of the PACE filter step (declared in include/pace.h): host-side
// argument checks, workspace carving and kernel launches. All device work is
// enqueued on the caller's stream; nothing here allocates or synchronises.
#include <math.h>
#include <atomic>
#include <stdint.h>
#include <string.h>

#include <hip/hip_runtime_api.h>

#include "../../include/pace.h"
#include "elem.hpp"
#include "kernels.hpp"

#pragma clang fp contract(off)

using namespace pace;

namespace {

bool aligned(const void *p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

pace_params params_or_default(const pace_params *p) {
    pace_params d;
    pace_default_params(&d);
    return p ? *p : d;
}

int64_t ipow_checked(int64_t x, int g, bool *overflow) {
    // x^g for the 2^53 check of the prefix window; saturates on overflow
    int64_t r = 1;
    for (int k = 0; k < g; ++k) {
        if (x != 0 && r > INT64_MAX / x) {
            *overflow = true;
            return INT64_MAX;
        }
        r *= x;
    }
    return r;
}

int hip_status(hipError_t e) { return e == hipSuccess ? PACE_OK : PACE_ERR_HIP; }

}  // namespace

namespace pace {

int64_t resident_waves() {
    // CU count per device, queried once per device (the attribute is constant).
    static std::atomic<int> cache[64];
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 256 * 16;
    int cu = cache[dev].load(std::memory_order_relaxed);
    if (cu <= 0) {
        if (hipDeviceGetAttribute(&cu, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cu <= 0)
            cu = 256;
        cache[dev].store(cu, std::memory_order_relaxed);
    }
    return (int64_t)cu * 16;
}

namespace {
// Armed timers, per host thread: [phase][start, stop].
thread_local hipEvent_t g_phase_timer[kPhaseCount][2];
}  // namespace

bool take_phase_timer(int phase, hipEvent_t *start, hipEvent_t *stop) {
    if (phase < 0 || phase >= kPhaseCount || g_phase_timer[phase][0] == nullptr) return false;
    *start = g_phase_timer[phase][0];
    *stop = g_phase_timer[phase][1];
    g_phase_timer[phase][0] = g_phase_timer[phase][1] = nullptr;
    return true;
}

namespace {
// Every entry point that enqueues device work holds one of these: when the
// call returns, the thread's armed timers are dropped, used or not, so a
// timer never reaches a later call.
struct TimerScope {
    TimerScope() = default;
    TimerScope(const TimerScope &) = delete;
    TimerScope &operator=(const TimerScope &) = delete;
    ~TimerScope() {
        for (int k = 0; k < kPhaseCount; ++k) g_phase_timer[k][0] = g_phase_timer[k][1] = nullptr;
    }
};
}  // namespace

}  // namespace pace

extern "C" {

void pace_default_params(pace_params *p) {
    if (!p) return;
    p->w_wait = 1.0;
    p->gamma = 4;
    p->window_min = 32;
    p->beta = 0.0;
    p->r_max = 0.9;
}

const char *pace_strerror(int code) {
    switch (code) {
        case PACE_OK: return "ok";
        case PACE_ERR_INVALID_ARG: return "invalid argument";
        case PACE_ERR_WORKSPACE: return "workspace missing, misaligned or too small";
        case PACE_ERR_PRECONDITION: return "data precondition violated";
        case PACE_ERR_HIP: return "HIP launch failure";
        case PACE_ERR_SCRATCH_LIMIT: return "pool too large for the fixed device scratch";
        default: return "unknown error code";
    }
}

int pace_workspace_bytes(int which, int64_t n_traj, int64_t n_tokens, size_t *bytes_out) {
    if (!bytes_out || n_traj < 0 || n_tokens < 0) return PACE_ERR_INVALID_ARG;
    switch (which) {
        case PACE_WS_SCORE: *bytes_out = score_ws_bytes(n_traj, n_tokens); return PACE_OK;
        case PACE_WS_SELECT: *bytes_out = select_ws_bytes(n_traj); return PACE_OK;
        case PACE_WS_COMPACT: *bytes_out = compact_ws_bytes(n_traj, n_tokens); return PACE_OK;
        case PACE_WS_FILTER_STEP: *bytes_out = filter_step_ws_bytes(n_traj, n_tokens); return PACE_OK;
        default: return PACE_ERR_INVALID_ARG;
    }
}

static int check_score_args(const int32_t *tags, const int64_t *offsets, int64_t n_traj,
                            int64_t n_tokens, const int32_t *completion, int32_t current_version,
                            const double *prefix_score, const double *window_sorted,
                            int64_t window_n, const pace_params &p, const double *score_out,
                            const int64_t *gen_sum_out, const int64_t *gen_count_out) {
    if (n_traj < 0 || n_traj >= INT32_MAX || n_tokens < 0 || window_n < 0) return PACE_ERR_INVALID_ARG;
    if (!offsets || (n_traj > 0 && (!completion || !score_out)) || (n_tokens > 0 && !tags))
        return PACE_ERR_INVALID_ARG;
    if (!aligned(tags, 4) || !aligned(offsets, 8) || !aligned(completion, 4) ||
        !aligned(score_out, 8) || !aligned(gen_sum_out, 8) || !aligned(gen_count_out, 8) ||
        !aligned(prefix_score, 8) || !aligned(window_sorted, 8))
        return PACE_ERR_INVALID_ARG;
    if (current_version < 0 || current_version == INT32_MAX) return PACE_ERR_INVALID_ARG;
    if (!(p.w_wait >= 0.0) || isinf(p.w_wait) || p.gamma < 1 || p.gamma > 4 || p.window_min < 0)
        return PACE_ERR_INVALID_ARG;
    if (window_n > 0 && !window_sorted) return PACE_ERR_INVALID_ARG;
    bool of = false;
    if (window_n > 0 && (ipow_checked(window_n, p.gamma, &of) >= ((int64_t)1 << 53) || of))
        return PACE_ERR_INVALID_ARG;
    return PACE_OK;
}

static int check_compact_args(const int64_t *offsets, int64_t n_traj, int64_t n_tokens,
                              const uint8_t *keep, int n_cols, const void *const *cols_in,
                              const int32_t *elem_bytes, void *const *cols_out,
                              const int64_t *offsets_out, const int32_t *kept_ids_out,
                              const int64_t *n_kept_tokens_out, CompactCols *cols) {
    if (n_traj < 0 || n_traj >= INT32_MAX || n_tokens < 0 || n_cols < 0 || n_cols > kMaxCols)
        return PACE_ERR_INVALID_ARG;
    if (!offsets || !offsets_out || !n_kept_tokens_out || (n_traj > 0 && (!keep || !kept_ids_out)))
        return PACE_ERR_INVALID_ARG;
    if (!aligned(offsets, 8) || !aligned(offsets_out, 8) || !aligned(n_kept_tokens_out, 8) ||
        !aligned(kept_ids_out, 4))
        return PACE_ERR_INVALID_ARG;
    if (n_cols > 0 && (!cols_in || !cols_out || !elem_bytes)) return PACE_ERR_INVALID_ARG;
    memset(cols, 0, sizeof(*cols));
    for (int c = 0; c < n_cols; ++c) {
        const int32_t e = elem_bytes[c];
        if (!(e == 1 || e == 2 || e == 4 || e == 8)) return PACE_ERR_INVALID_ARG;
        if (n_tokens > 0 && (!cols_in[c] || !cols_out[c])) return PACE_ERR_INVALID_ARG;
        if (!aligned(cols_in[c], (uintptr_t)e) || !aligned(cols_out[c], (uintptr_t)e))
            return PACE_ERR_INVALID_ARG;
        if (n_tokens > INT64_MAX / 8) return PACE_ERR_INVALID_ARG;
        cols->in[c] = cols_in[c];
        cols->out[c] = cols_out[c];
        cols->elem[c] = e;
        cols->vec[c] = (aligned(cols_in[c], 16) && aligned(cols_out[c], 16)) ? 1 : 0;
    }
    return PACE_OK;
}

int pace_score(const int32_t *tags, const int64_t *offsets, int64_t n_traj, int64_t n_tokens,
               const int32_t *completion, int32_t current_version, const double *prefix_score,
               const double *window_sorted, int64_t window_n, const pace_params *params,
               double *score_out, int64_t *gen_sum_out, int64_t *gen_count_out, void *workspace,
               size_t workspace_bytes, void *stream) {
    const TimerScope timers;
    const pace_params p = params_or_default(params);
    int rc = check_score_args(tags, offsets, n_traj, n_tokens, completion, current_version,
                              prefix_score, window_sorted, window_n, p, score_out, gen_sum_out,
                              gen_count_out);
    if (rc != PACE_OK) return rc;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < score_ws_bytes(n_traj, n_tokens))
        return PACE_ERR_WORKSPACE;
    const int64_t wmin = p.window_min > 1 ? p.window_min : 1;
    const bool use_prefix = prefix_score != nullptr && window_n >= wmin;
    const ScoreWorkspace ws = score_ws_carve(workspace, n_traj, n_tokens);
    return hip_status(launch_score(tags, ScoreArgs{offsets, n_traj, n_tokens, completion, current_version,
                                                   use_prefix ? 1 : 0, p.gamma, prefix_score, window_sorted, window_n,
                                                   p.w_wait, score_out, gen_sum_out, gen_count_out},
                                   ws, (hipStream_t)stream));
}

static int budget_impl(int64_t occupancy, int64_t capacity, const pace_params *params,
                       double *r_hat_inout, int64_t *budget_out) {
    const pace_params p = params_or_default(params);
    if (!r_hat_inout || !budget_out || occupancy < 0 || capacity < 0) return PACE_ERR_INVALID_ARG;
    if (!(p.beta >= 0.0 && p.beta < 1.0) || !(p.r_max >= 0.0 && p.r_max <= 1.0))
        return PACE_ERR_INVALID_ARG;
    const double prev = *r_hat_inout;
    if (!(prev >= 0.0) || isinf(prev)) return PACE_ERR_INVALID_ARG;
    // Eq. (3): fraction of the pool above the target occupancy, clipped.
    const double surplus_frac = (double)(occupancy - capacity) / (double)(occupancy > 1 ? occupancy : 1);
    const double r = surplus_frac < 0.0 ? 0.0 : (surplus_frac > 1.0 ? 1.0 : surplus_frac);
    // Eq. (4): exponential smoothing (two products then one sum, never fused).
    const double kept_part = p.beta * prev;
    const double new_part = (1.0 - p.beta) * r;
    const double r_hat = kept_part + new_part;
    int64_t b = 0;
    if (occupancy > capacity) {
        const double capped = r_hat < p.r_max ? r_hat : p.r_max;
        b = (int64_t)nearbyint(capped * (double)occupancy);   // ties to even
        const int64_t surplus = occupancy - capacity;
        if (b > surplus) b = surplus;
        if (b < 0) b = 0;
    }
    *r_hat_inout = r_hat;
    *budget_out = b;
    return PACE_OK;
}

int pace_budget(int64_t occupancy, int64_t capacity, const pace_params *params,
                double *r_hat_inout, int64_t *budget_out) {
    return budget_impl(occupancy, capacity, params, r_hat_inout, budget_out);
}

int pace_select(const double *score, int64_t n_traj, int64_t budget, uint8_t *keep_out,
                int32_t *reject_ids_out, void *workspace, size_t workspace_bytes, void *stream) {
    const TimerScope timers;
    if (n_traj < 0 || n_traj >= INT32_MAX || budget < 0 || budget > n_traj) return PACE_ERR_INVALID_ARG;
    if (n_traj > 0 && (!score || !keep_out)) return PACE_ERR_INVALID_ARG;
    if (budget > 0 && !reject_ids_out) return PACE_ERR_INVALID_ARG;
    if (!aligned(score, 8) || !aligned(reject_ids_out, 4)) return PACE_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < select_ws_bytes(n_traj))
        return PACE_ERR_WORKSPACE;
    return hip_status(launch_select(score, n_traj, budget, keep_out, reject_ids_out, workspace,
                                    (hipStream_t)stream));
}

int pace_compact(const int64_t *offsets, int64_t n_traj, int64_t n_tokens, const uint8_t *keep,
                 int n_cols, const void *const *cols_in, const int32_t *elem_bytes,
                 void *const *cols_out, int64_t *offsets_out, int32_t *kept_ids_out,
                 int64_t *n_kept_tokens_out, void *workspace, size_t workspace_bytes,
                 void *stream) {
    const TimerScope timers;
    CompactCols cols;
    int rc = check_compact_args(offsets, n_traj, n_tokens, keep, n_cols, cols_in, elem_bytes, cols_out,
                                offsets_out, kept_ids_out, n_kept_tokens_out, &cols);
    if (rc != PACE_OK) return rc;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < compact_ws_bytes(n_traj, n_tokens))
        return PACE_ERR_WORKSPACE;
    return hip_status(launch_compact(offsets, n_traj, n_tokens, keep, cols, n_cols, offsets_out,
                                     kept_ids_out, n_kept_tokens_out, workspace, (hipStream_t)stream));
}

// pace_filter_step's checks and launches. With scratch_limit set, the
// workspace is the fixed device scratch: a pool whose workspace exceeds it is
// refused with PACE_ERR_SCRATCH_LIMIT after the argument checks, and
// `workspace` is looked up only then.
static int filter_step_impl(const int32_t *tags, const int64_t *offsets, int64_t n_traj, int64_t n_tokens,
                            const int32_t *completion, int32_t current_version,
                            const double *prefix_score, const double *window_sorted, int64_t window_n,
                            int64_t occupancy, int64_t capacity, const pace_params *params,
                            double *r_hat_inout, int64_t *budget_out, double *score_out,
                            int64_t *gen_sum_out, int64_t *gen_count_out, uint8_t *keep_out,
                            int32_t *reject_ids_out, int n_cols, const void *const *cols_in,
                            const int32_t *elem_bytes, void *const *cols_out, int64_t *offsets_out,
                            int32_t *kept_ids_out, int64_t *n_kept_tokens_out, void *workspace,
                            size_t workspace_bytes, bool scratch_limit, void *stream) {
    const pace_params p = params_or_default(params);
    int rc = check_score_args(tags, offsets, n_traj, n_tokens, completion, current_version,
                              prefix_score, window_sorted, window_n, p, score_out, gen_sum_out,
                              gen_count_out);
    if (rc != PACE_OK) return rc;
    CompactCols cols;
    rc = check_compact_args(offsets, n_traj, n_tokens, keep_out, n_cols, cols_in, elem_bytes,
                            cols_out, offsets_out, kept_ids_out, n_kept_tokens_out, &cols);
    if (rc != PACE_OK) return rc;
    if (n_traj > 0 && !keep_out) return PACE_ERR_INVALID_ARG;
    if (!r_hat_inout || !budget_out || !aligned(reject_ids_out, 4)) return PACE_ERR_INVALID_ARG;
    if (scratch_limit) {
        if (filter_step_ws_bytes(n_traj, n_tokens) > (size_t)PACE_NOALLOC_SCRATCH_BYTES)
            return PACE_ERR_SCRATCH_LIMIT;
        if (noalloc_scratch(&workspace) != hipSuccess) return PACE_ERR_HIP;
        workspace_bytes = PACE_NOALLOC_SCRATCH_BYTES;
    }
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < filter_step_ws_bytes(n_traj, n_tokens))
        return PACE_ERR_WORKSPACE;
    double r_hat = *r_hat_inout;
    int64_t budget = 0;
    rc = budget_impl(occupancy, capacity, &p, &r_hat, &budget);
    if (rc != PACE_OK) return rc;
    if (budget > n_traj || (budget > 0 && !reject_ids_out)) return PACE_ERR_INVALID_ARG;
    const int64_t wmin = p.window_min > 1 ? p.window_min : 1;
    const bool use_prefix = prefix_score != nullptr && window_n >= wmin;
    rc = hip_status(launch_filter_step(tags, offsets, n_traj, n_tokens, completion, current_version,
                                       prefix_score, window_sorted, window_n, use_prefix, p.w_wait,
                                       p.gamma, budget, score_out, gen_sum_out, gen_count_out,
                                       keep_out, reject_ids_out, cols, n_cols, offsets_out,
                                       kept_ids_out, n_kept_tokens_out, workspace,
                                       (hipStream_t)stream));
    if (rc != PACE_OK) return rc;
    *r_hat_inout = r_hat;
    *budget_out = budget;
    return PACE_OK;
}

int pace_filter_step(const int32_t *tags, const int64_t *offsets, int64_t n_traj, int64_t n_tokens,
                     const int32_t *completion, int32_t current_version,
                     const double *prefix_score, const double *window_sorted, int64_t window_n,
                     int64_t occupancy, int64_t capacity, const pace_params *params,
                     double *r_hat_inout, int64_t *budget_out, double *score_out,
                     int64_t *gen_sum_out, int64_t *gen_count_out, uint8_t *keep_out,
                     int32_t *reject_ids_out, int n_cols, const void *const *cols_in,
                     const int32_t *elem_bytes, void *const *cols_out, int64_t *offsets_out,
                     int32_t *kept_ids_out, int64_t *n_kept_tokens_out, void *workspace,
                     size_t workspace_bytes, void *stream) {
    const TimerScope timers;
    return filter_step_impl(tags, offsets, n_traj, n_tokens, completion, current_version, prefix_score,
                            window_sorted, window_n, occupancy, capacity, params, r_hat_inout, budget_out,
                            score_out, gen_sum_out, gen_count_out, keep_out, reject_ids_out, n_cols, cols_in,
                            elem_bytes, cols_out, offsets_out, kept_ids_out, n_kept_tokens_out, workspace,
                            workspace_bytes, false, stream);
}

int pace_filter_step_noalloc(const int32_t *tags, const int64_t *offsets, int64_t n_traj, int64_t n_tokens,
                             const int32_t *completion, int32_t current_version,
                             const double *prefix_score, const double *window_sorted, int64_t window_n,
                             int64_t occupancy, int64_t capacity, const pace_params *params,
                             double *r_hat_inout, int64_t *budget_out, double *score_out,
                             int64_t *gen_sum_out, int64_t *gen_count_out, uint8_t *keep_out,
                             int32_t *reject_ids_out, int n_cols, const void *const *cols_in,
                             const int32_t *elem_bytes, void *const *cols_out, int64_t *offsets_out,
                             int32_t *kept_ids_out, int64_t *n_kept_tokens_out, void *stream) {
    const TimerScope timers;
    return filter_step_impl(tags, offsets, n_traj, n_tokens, completion, current_version, prefix_score,
                            window_sorted, window_n, occupancy, capacity, params, r_hat_inout, budget_out,
                            score_out, gen_sum_out, gen_count_out, keep_out, reject_ids_out, n_cols, cols_in,
                            elem_bytes, cols_out, offsets_out, kept_ids_out, n_kept_tokens_out, nullptr, 0,
                            true, stream);
}

static int check_groups_arg(const int64_t *group_offsets, int64_t n_groups) {
    if (n_groups < 0 || n_groups >= INT32_MAX || !group_offsets || !aligned(group_offsets, 8))
        return PACE_ERR_INVALID_ARG;
    return PACE_OK;
}

int pace_group_score(const double *score, int64_t n_traj, const int64_t *group_offsets, int64_t n_groups,
                     double *group_score_out, void *stream) {
    const TimerScope timers;
    if (n_traj < 0 || n_traj >= INT32_MAX || check_groups_arg(group_offsets, n_groups) != PACE_OK)
        return PACE_ERR_INVALID_ARG;
    if ((n_traj > 0 && !score) || (n_groups > 0 && !group_score_out) || !aligned(score, 8) ||
        !aligned(group_score_out, 8))
        return PACE_ERR_INVALID_ARG;
    return hip_status(launch_group_score(score, n_traj, group_offsets, n_groups, group_score_out,
                                         (hipStream_t)stream));
}

int pace_group_expand(const int64_t *group_offsets, int64_t n_groups, int64_t n_traj,
                      const uint8_t *group_keep, uint8_t *keep_out, void *stream) {
    const TimerScope timers;
    if (n_traj < 0 || n_traj >= INT32_MAX || check_groups_arg(group_offsets, n_groups) != PACE_OK)
        return PACE_ERR_INVALID_ARG;
    if ((n_groups > 0 && !group_keep) || (n_traj > 0 && !keep_out)) return PACE_ERR_INVALID_ARG;
    return hip_status(launch_group_expand(group_offsets, n_groups, n_traj, group_keep, keep_out,
                                          (hipStream_t)stream));
}

int pace_validate_groups(const int64_t *group_offsets, int64_t n_groups, int64_t n_traj,
                         int32_t *err_word_out, void *stream) {
    const TimerScope timers;
    if (n_traj < 0 || n_traj >= INT32_MAX || check_groups_arg(group_offsets, n_groups) != PACE_OK)
        return PACE_ERR_INVALID_ARG;
    if (!err_word_out || !aligned(err_word_out, 4)) return PACE_ERR_INVALID_ARG;
    return hip_status(launch_group_validate(group_offsets, n_groups, n_traj, err_word_out,
                                            (hipStream_t)stream));
}

int pace_group_filter_step(const int32_t *tags, const int64_t *offsets, int64_t n_traj, int64_t n_tokens,
                           const int32_t *completion, int32_t current_version,
                           const double *prefix_score, const double *window_sorted, int64_t window_n,
                           const int64_t *group_offsets, int64_t n_groups, int64_t occupancy,
                           int64_t capacity, const pace_params *params, double *r_hat_inout,
                           int64_t *budget_out, double *score_out, int64_t *gen_sum_out,
                           int64_t *gen_count_out, double *group_score_out, uint8_t *group_keep_out,
                           int32_t *reject_group_ids_out, uint8_t *keep_out, int n_cols,
                           const void *const *cols_in, const int32_t *elem_bytes, void *const *cols_out,
                           int64_t *offsets_out, int32_t *kept_ids_out, int64_t *n_kept_tokens_out,
                           void *workspace, size_t workspace_bytes, void *stream) {
    const TimerScope timers;
    const pace_params p = params_or_default(params);
    int rc = check_score_args(tags, offsets, n_traj, n_tokens, completion, current_version,
                              prefix_score, window_sorted, window_n, p, score_out, gen_sum_out,
                              gen_count_out);
    if (rc != PACE_OK) return rc;
    if (check_groups_arg(group_offsets, n_groups) != PACE_OK) return PACE_ERR_INVALID_ARG;
    if (n_groups > 0 && (!group_score_out || !group_keep_out)) return PACE_ERR_INVALID_ARG;
    if (!aligned(group_score_out, 8) || !aligned(reject_group_ids_out, 4)) return PACE_ERR_INVALID_ARG;
    CompactCols cols;
    rc = check_compact_args(offsets, n_traj, n_tokens, keep_out, n_cols, cols_in, elem_bytes,
                            cols_out, offsets_out, kept_ids_out, n_kept_tokens_out, &cols);
    if (rc != PACE_OK) return rc;
    if (!r_hat_inout || !budget_out) return PACE_ERR_INVALID_ARG;
    const int64_t N = n_traj > n_groups ? n_traj : n_groups;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < filter_step_ws_bytes(N, n_tokens))
        return PACE_ERR_WORKSPACE;
    double r_hat = *r_hat_inout;
    int64_t budget = 0;
    rc = budget_impl(occupancy, capacity, &p, &r_hat, &budget);
    if (rc != PACE_OK) return rc;
    if (budget > n_groups || (budget > 0 && !reject_group_ids_out)) return PACE_ERR_INVALID_ARG;
    const int64_t wmin = p.window_min > 1 ? p.window_min : 1;
    const bool use_prefix = prefix_score != nullptr && window_n >= wmin;
    rc = hip_status(launch_group_filter_step(
        tags, offsets, n_traj, n_tokens, completion, current_version, prefix_score, window_sorted, window_n,
        use_prefix, p.w_wait, p.gamma, group_offsets, n_groups, budget, score_out, gen_sum_out, gen_count_out,
        group_score_out, group_keep_out, reject_group_ids_out, keep_out, cols, n_cols, offsets_out, kept_ids_out,
        n_kept_tokens_out, workspace, (hipStream_t)stream));
    if (rc != PACE_OK) return rc;
    *r_hat_inout = r_hat;
    *budget_out = budget;
    return PACE_OK;
}

int pace_stream_admit(const double *score, int64_t n_traj, double r_hat, const pace_params *params,
                      int64_t batch_size, double *window_ring, int64_t window_cap, int64_t *window_state,
                      uint8_t *status_out, uint8_t *keep_out, int32_t *reject_ids_out, double *kappa_out,
                      int64_t *counts_out, void *stream) {
    const TimerScope timers;
    const pace_params p = params_or_default(params);
    if (n_traj < 0 || n_traj >= INT32_MAX || batch_size < 0) return PACE_ERR_INVALID_ARG;
    if (!(r_hat >= 0.0) || isinf(r_hat) || !(p.r_max >= 0.0 && p.r_max <= 1.0) || p.window_min < 0)
        return PACE_ERR_INVALID_ARG;
    if (window_cap < 1 || window_cap > kStreamWindowMax || !window_ring || !window_state || !kappa_out ||
        !counts_out)
        return PACE_ERR_INVALID_ARG;
    if (n_traj > 0 && (!score || !status_out || !keep_out || !reject_ids_out)) return PACE_ERR_INVALID_ARG;
    if (!aligned(score, 8) || !aligned(window_ring, 8) || !aligned(window_state, 8) || !aligned(kappa_out, 8) ||
        !aligned(counts_out, 8) || !aligned(reject_ids_out, 4))
        return PACE_ERR_INVALID_ARG;
    const double rate = r_hat < p.r_max ? r_hat : p.r_max;
    return hip_status(launch_stream_admit(score, n_traj, rate, p.window_min, batch_size, window_ring,
                                          window_cap, window_state, status_out, keep_out, reject_ids_out,
                                          kappa_out, counts_out, nullptr, 0, PieceParts{}, (hipStream_t)stream));
}

int pace_stream_step(const int32_t *tags, const int64_t *offsets, int64_t n_traj, int64_t n_tokens,
                     const int32_t *completion, int32_t current_version, const double *prefix_score,
                     const double *window_sorted, int64_t window_n, int64_t occupancy, int64_t capacity,
                     const pace_params *params, double *r_hat_inout, int64_t batch_size,
                     double *window_ring, int64_t window_cap, int64_t *window_state, double *score_out,
                     int64_t *gen_sum_out, int64_t *gen_count_out, uint8_t *status_out, uint8_t *keep_out,
                     int32_t *reject_ids_out, double *kappa_out, int64_t *counts_out, int n_cols,
                     const void *const *cols_in, const int32_t *elem_bytes, void *const *cols_out,
                     int64_t *offsets_out, int32_t *kept_ids_out, int64_t *n_kept_tokens_out,
                     void *workspace, size_t workspace_bytes, void *stream) {
    const TimerScope timers;
    const pace_params p = params_or_default(params);
    int rc = check_score_args(tags, offsets, n_traj, n_tokens, completion, current_version,
                              prefix_score, window_sorted, window_n, p, score_out, gen_sum_out,
                              gen_count_out);
    if (rc != PACE_OK) return rc;
    CompactCols cols;
    rc = check_compact_args(offsets, n_traj, n_tokens, keep_out, n_cols, cols_in, elem_bytes,
                            cols_out, offsets_out, kept_ids_out, n_kept_tokens_out, &cols);
    if (rc != PACE_OK) return rc;
    if (!r_hat_inout || batch_size < 0 || window_cap < 1 || window_cap > kStreamWindowMax || !window_ring ||
        !window_state || !kappa_out || !counts_out)
        return PACE_ERR_INVALID_ARG;
    if (n_traj > 0 && (!status_out || !keep_out || !reject_ids_out)) return PACE_ERR_INVALID_ARG;
    if (!aligned(window_ring, 8) || !aligned(window_state, 8) || !aligned(kappa_out, 8) ||
        !aligned(counts_out, 8) || !aligned(reject_ids_out, 4))
        return PACE_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < filter_step_ws_bytes(n_traj, n_tokens))
        return PACE_ERR_WORKSPACE;
    double r_hat = *r_hat_inout;
    int64_t budget = 0;
    rc = budget_impl(occupancy, capacity, &p, &r_hat, &budget);
    if (rc != PACE_OK) return rc;
    const int64_t wmin = p.window_min > 1 ? p.window_min : 1;
    const bool use_prefix = prefix_score != nullptr && window_n >= wmin;
    char *w = (char *)workspace;
    const ScoreWorkspace sws = score_ws_carve(w, n_traj, n_tokens);
    void *cws = w + align256(score_ws_bytes(n_traj, n_tokens));
    hipStream_t st = (hipStream_t)stream;
    ScoreJoin join;
    hipError_t e = launch_score_unjoined(tags, ScoreArgs{offsets, n_traj, n_tokens, completion, current_version,
                                                         use_prefix ? 1 : 0, p.gamma, prefix_score, window_sorted,
                                                         window_n, p.w_wait, score_out, gen_sum_out, gen_count_out},
                                         sws, st, &join);
    // Pools the piece compaction takes get their block partials from the
    // draw itself; the kept trajectories are at most min(batch_size, n).
    const bool pieces = compact_piece_ok(n_traj, n_tokens);
    const CompactWs cw = compact_ws_carve(cws, n_traj, n_tokens);
    if (e == hipSuccess) {
        const double rate = r_hat < p.r_max ? r_hat : p.r_max;
        e = launch_stream_admit(score_out, n_traj, rate, p.window_min, batch_size, window_ring, window_cap,
                                window_state, status_out, keep_out, reject_ids_out, kappa_out, counts_out,
                                pieces ? offsets : nullptr, n_tokens, pieces ? cw.parts : PieceParts{}, st, join);
    }
    if (e == hipSuccess) {
        if (pieces)
            e = launch_compact_pieces(offsets, n_traj, n_tokens, keep_out, cw.parts, cols, n_cols, offsets_out,
                                      kept_ids_out, n_kept_tokens_out, nullptr, 0,
                                      batch_size < n_traj ? batch_size : n_traj, st);
        else
            e = launch_compact(offsets, n_traj, n_tokens, keep_out, cols, n_cols, offsets_out, kept_ids_out,
                               n_kept_tokens_out, cws, st);
    }
    rc = hip_status(e);
    if (rc != PACE_OK) return rc;
    *r_hat_inout = r_hat;
    return PACE_OK;
}

int pace_prefix_score(const float *lp_new, const float *lp_behavior, const int32_t *tags,
                      const int64_t *prefix_offsets, int64_t n, int64_t n_tokens, int64_t cap,
                      int64_t min_tokens, double *s_pre_out, void *stream) {
    const TimerScope timers;
    if (n < 0 || n >= INT32_MAX || n_tokens < 0 || cap < 0 || min_tokens < 0 || !prefix_offsets)
        return PACE_ERR_INVALID_ARG;
    if ((n > 0 && !s_pre_out) || (n_tokens > 0 && (!lp_new || !lp_behavior))) return PACE_ERR_INVALID_ARG;
    if (!aligned(lp_new, 4) || !aligned(lp_behavior, 4) || !aligned(tags, 4) || !aligned(prefix_offsets, 8) ||
        !aligned(s_pre_out, 8))
        return PACE_ERR_INVALID_ARG;
    return hip_status(launch_prefix_score(lp_new, lp_behavior, tags, prefix_offsets, n, n_tokens, cap, min_tokens,
                                          s_pre_out, (hipStream_t)stream));
}

int pace_stale_k(const int64_t *gen_sum, const int64_t *gen_count, const int32_t *completion,
                 int32_t current_version, int64_t n_traj, int64_t k, uint8_t *keep_out, double *lag_out,
                 void *stream) {
    const TimerScope timers;
    if (n_traj < 0 || n_traj >= INT32_MAX || k < 0 || k >= INT32_MAX || current_version < 0)
        return PACE_ERR_INVALID_ARG;
    if (n_traj > 0 && (!gen_sum || !gen_count || !completion || !keep_out)) return PACE_ERR_INVALID_ARG;
    if (!aligned(gen_sum, 8) || !aligned(gen_count, 8) || !aligned(completion, 4) || !aligned(lag_out, 8))
        return PACE_ERR_INVALID_ARG;
    return hip_status(launch_stale_k(gen_sum, gen_count, completion, current_version, n_traj, k, keep_out, lag_out,
                                     (hipStream_t)stream));
}

int pace_diagnostics(const double *score, const int64_t *gen_sum, const int64_t *gen_count,
                     const int32_t *completion, int32_t current_version, const uint8_t *keep, int64_t n_traj,
                     const double *edges, int nbins, int64_t *hist_out, int64_t *totals_out, void *stream) {
    const TimerScope timers;
    if (n_traj < 0 || n_traj >= INT32_MAX || nbins < 1 || nbins > kDiagBinsMax || current_version < 0)
        return PACE_ERR_INVALID_ARG;
    if (!edges || !hist_out || !totals_out) return PACE_ERR_INVALID_ARG;
    if (n_traj > 0 && (!score || !gen_sum || !gen_count || !completion || !keep)) return PACE_ERR_INVALID_ARG;
    if (!aligned(score, 8) || !aligned(gen_sum, 8) || !aligned(gen_count, 8) || !aligned(completion, 4) ||
        !aligned(edges, 8) || !aligned(hist_out, 8) || !aligned(totals_out, 8))
        return PACE_ERR_INVALID_ARG;
    return hip_status(launch_diagnostics(score, gen_sum, gen_count, completion, current_version, keep, n_traj,
                                         edges, nbins, hist_out, totals_out, (hipStream_t)stream));
}

static_assert(PACE_F32 == kF32 && PACE_BF16 == kBf16 && PACE_F16 == kF16, "element types");
static_assert(PACE_TOP_MAX == kTopMax, "alternatives");

// 128 * 128 * k stays below 2^31: the integer sums are exact.
constexpr int64_t kMatmulI8MaxK = 131072;

// Tiles of 64 of both sides are numbered in a grid's 16-bit axis, and a tile's rows by 32-bit byte offsets.
constexpr int64_t kOrthoSideMax = (int64_t)1 << 21;

// Spans and their workgroups stay 32-bit numbers.
constexpr int64_t kLossTokensMax = (int64_t)1 << 40;

// Rows of `cols` elements `stride` apart, as the operators on matrices take them.
static bool rows_ok(const void *p, int dtype, int64_t rows, int64_t cols, int64_t stride) {
    if (dtype < 0 || dtype >= kElemTypes || rows < 0 || rows >= INT32_MAX || cols < 1 || cols >= INT32_MAX) return false;
    if (stride < cols || (rows > 0 && stride > INT64_MAX / 4 / rows)) return false;
    return rows == 0 || (p != nullptr && aligned(p, elem_bytes_of(dtype)));
}

// c = log2(e) / temperature and its inverse stay normal binary32 numbers.
static bool temperature_ok(double t) { return t >= 1e-6 && t <= 1e6; }

int pace_token_logprob_workspace_bytes(int64_t n_rows, int64_t vocab, int top_k, size_t *bytes_out) {
    if (!bytes_out || n_rows < 0 || n_rows >= INT32_MAX || vocab < 1 || vocab >= INT32_MAX || top_k < 0 || top_k > kTopMax)
        return PACE_ERR_INVALID_ARG;
    *bytes_out = logprob_ws_bytes(n_rows, vocab, top_k);
    return PACE_OK;
}

int pace_token_logprob(const void *logits, int dtype, int64_t n_rows, int64_t vocab, int64_t row_stride,
                       const int32_t *token_ids, double temperature, int top_k, float *logp_out, float *entropy_out,
                       float *stats_out, int32_t *top_ids_out, float *top_logp_out, void *workspace,
                       size_t workspace_bytes, void *stream) {
    const TimerScope timers;
    if (!rows_ok(logits, dtype, n_rows, vocab, row_stride) || !temperature_ok(temperature)) return PACE_ERR_INVALID_ARG;
    if (top_k < 0 || top_k > kTopMax || top_k > vocab) return PACE_ERR_INVALID_ARG;
    if (n_rows > 0 && (!token_ids || !logp_out || (top_k > 0 && (!top_ids_out || !top_logp_out)))) return PACE_ERR_INVALID_ARG;
    if (!aligned(token_ids, 4) || !aligned(logp_out, 4) || !aligned(entropy_out, 4) || !aligned(stats_out, 4) ||
        !aligned(top_ids_out, 4) || !aligned(top_logp_out, 4))
        return PACE_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < logprob_ws_bytes(n_rows, vocab, top_k))
        return PACE_ERR_WORKSPACE;
    return hip_status(launch_token_logprob(logits, dtype, n_rows, vocab, row_stride, token_ids, temperature, top_k,
                                           LogprobOut{logp_out, entropy_out, stats_out, top_ids_out, top_logp_out},
                                           workspace, (hipStream_t)stream));
}

int pace_token_logprob_backward(const void *logits, int dtype, int64_t n_rows, int64_t vocab, int64_t row_stride,
                                const int32_t *token_ids, double temperature, const float *stats, const float *entropy,
                                const float *grad_logp, const float *grad_entropy, void *grad_logits_out,
                                int64_t grad_row_stride, void *stream) {
    const TimerScope timers;
    if (!rows_ok(logits, dtype, n_rows, vocab, row_stride) || !rows_ok(grad_logits_out, dtype, n_rows, vocab, grad_row_stride) ||
        !temperature_ok(temperature))
        return PACE_ERR_INVALID_ARG;
    if (n_rows > 0 && (!token_ids || !stats || !grad_logp || (grad_entropy && !entropy))) return PACE_ERR_INVALID_ARG;
    // In place only element for element.
    if (grad_logits_out == logits && grad_row_stride != row_stride) return PACE_ERR_INVALID_ARG;
    if (!aligned(token_ids, 4) || !aligned(stats, 4) || !aligned(entropy, 4) || !aligned(grad_logp, 4) ||
        !aligned(grad_entropy, 4))
        return PACE_ERR_INVALID_ARG;
    return hip_status(launch_token_logprob_backward(logits, dtype, n_rows, vocab, row_stride, token_ids, temperature, stats,
                                                    entropy, grad_logp, grad_entropy, grad_logits_out, grad_row_stride,
                                                    (hipStream_t)stream));
}

int pace_policy_loss_workspace_bytes(int64_t n_traj, int64_t n_tokens, size_t *bytes_out) {
    if (!bytes_out || n_traj < 0 || n_traj >= INT32_MAX || n_tokens < 0 || n_tokens >= kLossTokensMax)
        return PACE_ERR_INVALID_ARG;
    *bytes_out = policy_loss_ws_most(n_tokens);
    return PACE_OK;
}

int pace_policy_loss(const float *lp_new, const float *lp_behavior, const int32_t *tags, const int64_t *offsets,
                     int64_t n_traj, int64_t n_tokens, const float *advantage, const float *weight, double scale,
                     double clip_low, double clip_high, double dual_clip, float *grad_out, float *loss_out, float *kl_out,
                     int32_t *clipped_out, void *workspace, size_t workspace_bytes, void *stream) {
    const TimerScope timers;
    if (n_traj < 0 || n_traj >= INT32_MAX || n_tokens < 0 || n_tokens >= kLossTokensMax || !offsets)
        return PACE_ERR_INVALID_ARG;
    if ((n_tokens > 0 && (!lp_new || !lp_behavior || !grad_out)) || (n_traj > 0 && (!advantage || !loss_out)))
        return PACE_ERR_INVALID_ARG;
    if (!aligned(lp_new, 4) || !aligned(lp_behavior, 4) || !aligned(tags, 4) || !aligned(offsets, 8) ||
        !aligned(advantage, 4) || !aligned(weight, 4) || !aligned(grad_out, 4) || !aligned(loss_out, 4) ||
        !aligned(kl_out, 4) || !aligned(clipped_out, 4))
        return PACE_ERR_INVALID_ARG;
    if (!isfinite(scale) || !(clip_low >= 0.0 && clip_low < 1.0) || !(clip_high >= 0.0) || !(dual_clip > 1.0))
        return PACE_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < policy_loss_ws_bytes(n_tokens))
        return PACE_ERR_WORKSPACE;
    const LossBounds b{(float)(1.0 - clip_low), (float)(1.0 + clip_high), (float)dual_clip,
                       (float)log1p(-clip_low), (float)log1p(clip_high), (float)log(dual_clip)};
    return hip_status(launch_policy_loss(lp_new, lp_behavior, tags, offsets, n_traj, n_tokens, advantage, weight, scale, b,
                                         grad_out, loss_out, kl_out, clipped_out, workspace, (hipStream_t)stream));
}

int pace_quantize_rows(const void *x, int dtype, int64_t n_rows, int64_t n_cols, int64_t row_stride, int8_t *q_out,
                       float *scale_out, void *stream) {
    const TimerScope timers;
    if (!rows_ok(x, dtype, n_rows, n_cols, row_stride)) return PACE_ERR_INVALID_ARG;
    if (n_rows > 0 && (!q_out || !scale_out || !aligned(scale_out, 4))) return PACE_ERR_INVALID_ARG;
    return hip_status(launch_quantize_rows(x, dtype, n_rows, n_cols, row_stride, q_out, scale_out, (hipStream_t)stream));
}

int pace_matmul_i8_workspace_bytes(int64_t m, int64_t n, int64_t k, size_t *bytes_out) {
    if (!bytes_out || m < 0 || m >= INT32_MAX || n < 0 || n >= INT32_MAX || k < 1 || k >= kMatmulI8MaxK)
        return PACE_ERR_INVALID_ARG;
    *bytes_out = matmul_i8_ws_most(m, n, k);
    return PACE_OK;
}

int pace_matmul_i8(const int8_t *a, int64_t a_stride, const float *a_scale, const int8_t *b, int64_t b_stride,
                   const float *b_scale, int64_t m, int64_t n, int64_t k, void *out, int out_dtype, int64_t out_stride,
                   void *workspace, size_t workspace_bytes, void *stream) {
    const TimerScope timers;
    if (m < 0 || m >= INT32_MAX || n < 0 || n >= INT32_MAX || k < 1 || k >= kMatmulI8MaxK) return PACE_ERR_INVALID_ARG;
    if (a_stride < k || b_stride < k || (m > 0 && a_stride > INT64_MAX / 4 / m) || (n > 0 && b_stride > INT64_MAX / 4 / n))
        return PACE_ERR_INVALID_ARG;
    if (n > 0 && !rows_ok(out, out_dtype, m, n, out_stride)) return PACE_ERR_INVALID_ARG;
    // tiles are numbered in 32 bits
    if (((m + 63) / 64) * ((n + 63) / 64) >= INT32_MAX) return PACE_ERR_INVALID_ARG;
    if (m > 0 && n > 0 && (!a || !a_scale || !b || !b_scale)) return PACE_ERR_INVALID_ARG;
    if (!aligned(a_scale, 4) || !aligned(b_scale, 4)) return PACE_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < matmul_i8_ws_bytes(a, a_stride, b, b_stride, m, n, k))
        return PACE_ERR_WORKSPACE;
    return hip_status(launch_matmul_i8(a, a_stride, a_scale, b, b_stride, b_scale, m, n, k, out, out_dtype, out_stride,
                                       workspace, (hipStream_t)stream));
}

static bool ortho_sizes_ok(int64_t batch, int64_t rows, int64_t cols) {
    return batch >= 0 && batch < 65536 && rows >= 1 && rows <= kOrthoSideMax && cols >= 1 && cols <= kOrthoSideMax &&
           rows * cols <= INT64_MAX / 64 / (batch > 0 ? batch : 1);
}

int pace_orthogonalize_workspace_bytes(int64_t batch, int64_t rows, int64_t cols, size_t *bytes_out) {
    if (!bytes_out || !ortho_sizes_ok(batch, rows, cols)) return PACE_ERR_INVALID_ARG;
    *bytes_out = ortho_ws_most(batch, rows, cols);
    return PACE_OK;
}

int pace_orthogonalize(const void *update, int dtype, int64_t batch, int64_t rows, int64_t cols, int64_t row_stride,
                       int64_t batch_stride, int steps, const double *coefs, double eps, void *out, void *workspace,
                       size_t workspace_bytes, void *stream) {
    const TimerScope timers;
    if (!ortho_sizes_ok(batch, rows, cols) || steps < 0 || steps > 100 || !coefs) return PACE_ERR_INVALID_ARG;
    if (!rows_ok(update ? update : out, dtype, batch > 0 ? rows : 0, cols, row_stride)) return PACE_ERR_INVALID_ARG;
    if (batch > 1 && (batch_stride < 0 || batch_stride > INT64_MAX / 4 / batch || batch_stride < (rows - 1) * row_stride + cols))
        return PACE_ERR_INVALID_ARG;
    if (batch > 0 && (!update || !out || !aligned(out, 2))) return PACE_ERR_INVALID_ARG;
    if (!isfinite(coefs[0]) || !isfinite(coefs[1]) || !isfinite(coefs[2]) || !(eps > 0.0) || isinf(eps)) return PACE_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < ortho_ws_bytes(batch, rows, cols)) return PACE_ERR_WORKSPACE;
    return hip_status(launch_orthogonalize(update, dtype, batch, rows, cols, row_stride, batch_stride, steps, coefs, eps, out,
                                           workspace, (hipStream_t)stream));
}

// Whole numbers up to kLnColsMax are binary32 numbers, and a grid's workgroups of columns fit.
static bool layer_norm_ok(const void *x, int dtype, int64_t rows, int64_t cols, int64_t stride, int weight_dtype) {
    return rows_ok(x, dtype, rows, cols, stride) && cols <= kLnColsMax && (weight_dtype == dtype || weight_dtype == kF32);
}

int pace_layer_norm(const void *x, int dtype, int64_t n_rows, int64_t n_cols, int64_t row_stride, const void *weight,
                    const void *bias, int weight_dtype, double eps, void *out, int64_t out_stride, float *stats_out,
                    void *stream) {
    const TimerScope timers;
    if (!layer_norm_ok(x, dtype, n_rows, n_cols, row_stride, weight_dtype) || !rows_ok(out, dtype, n_rows, n_cols, out_stride))
        return PACE_ERR_INVALID_ARG;
    if (!aligned(weight, elem_bytes_of(weight_dtype)) || !aligned(bias, elem_bytes_of(weight_dtype)) || !aligned(stats_out, 4))
        return PACE_ERR_INVALID_ARG;
    if (!(eps >= 1e-30 && eps <= 1e30) || (n_rows > 0 && out == x)) return PACE_ERR_INVALID_ARG;
    return hip_status(launch_layer_norm(x, dtype, n_rows, n_cols, row_stride, weight, bias, weight_dtype, eps, out, out_stride,
                                        stats_out, (hipStream_t)stream));
}

int pace_layer_norm_backward_workspace_bytes(int64_t n_rows, int64_t n_cols, size_t *bytes_out) {
    if (!bytes_out || n_rows < 0 || n_rows >= INT32_MAX || n_cols < 1 || n_cols > kLnColsMax) return PACE_ERR_INVALID_ARG;
    *bytes_out = layer_norm_backward_ws_most(n_rows, n_cols);
    return PACE_OK;
}

int pace_layer_norm_backward(const void *x, int dtype, int64_t n_rows, int64_t n_cols, int64_t row_stride, const void *weight,
                             int weight_dtype, const float *stats, const void *grad_out, int64_t grad_out_stride,
                             void *grad_x_out, int64_t grad_x_stride, float *grad_weight_out, float *grad_bias_out,
                             void *workspace, size_t workspace_bytes, void *stream) {
    const TimerScope timers;
    if (!layer_norm_ok(x, dtype, n_rows, n_cols, row_stride, weight_dtype) ||
        !rows_ok(grad_out, dtype, n_rows, n_cols, grad_out_stride) || !rows_ok(grad_x_out, dtype, n_rows, n_cols, grad_x_stride))
        return PACE_ERR_INVALID_ARG;
    if (n_rows > 0 && !stats) return PACE_ERR_INVALID_ARG;
    // In place only element for element.
    if (n_rows > 0 && (grad_x_out == x || (grad_x_out == grad_out && grad_x_stride != grad_out_stride))) return PACE_ERR_INVALID_ARG;
    if (!aligned(weight, elem_bytes_of(weight_dtype)) || !aligned(stats, 4) || !aligned(grad_weight_out, 4) || !aligned(grad_bias_out, 4))
        return PACE_ERR_INVALID_ARG;
    if ((grad_weight_out || grad_bias_out) &&
        (!workspace || !aligned(workspace, 256) || workspace_bytes < layer_norm_backward_ws_bytes(n_rows, n_cols)))
        return PACE_ERR_WORKSPACE;
    return hip_status(launch_layer_norm_backward(x, dtype, n_rows, n_cols, row_stride, weight, weight_dtype, stats, grad_out,
                                                 grad_out_stride, grad_x_out, grad_x_stride, grad_weight_out, grad_bias_out,
                                                 workspace, (hipStream_t)stream));
}

// Sizes within the limit, together too, and a pointer aligned to its element for each tensor that is not empty.
static bool sizes_ok(int64_t n, const int64_t *sizes) {
    if (n < 0 || n >= INT32_MAX || (n > 0 && !sizes)) return false;
    int64_t total = 0;
    for (int64_t i = 0; i < n; ++i) {
        if (sizes[i] < 0 || sizes[i] > kAdamElementsMax || total > INT64_MAX / 4) return false;
        total += sizes[i];
    }
    return true;
}
static bool each_ok(int64_t n, const int64_t *sizes, const void *const *p, const int32_t *dtypes, uintptr_t bytes) {
    if (n > 0 && !p) return false;
    for (int64_t i = 0; i < n; ++i) {
        if (dtypes && (dtypes[i] < 0 || dtypes[i] >= kElemTypes)) return false;
        if (sizes[i] > 0 && (!p[i] || !aligned(p[i], dtypes ? (uintptr_t)elem_bytes_of(dtypes[i]) : bytes))) return false;
    }
    return true;
}

int pace_grad_norm_workspace_bytes(int64_t n_tensors, int64_t n_elements, size_t *bytes_out) {
    if (!bytes_out || n_tensors < 0 || n_tensors >= INT32_MAX || n_elements < 0 || n_elements > INT64_MAX / 4)
        return PACE_ERR_INVALID_ARG;
    *bytes_out = grad_norm_ws_most(n_tensors, n_elements);
    return PACE_OK;
}

int pace_grad_norm(int64_t n_tensors, const void *const *grads, const int32_t *grad_dtypes, const int64_t *sizes, double max_norm,
                   float *norm_out, float *factor_out, void *workspace, size_t workspace_bytes, void *stream) {
    const TimerScope timers;
    if (!sizes_ok(n_tensors, sizes) || (n_tensors > 0 && !grad_dtypes) || !each_ok(n_tensors, sizes, grads, grad_dtypes, 0))
        return PACE_ERR_INVALID_ARG;
    if (!(max_norm >= 0.0) || (!norm_out && !factor_out) || !aligned(norm_out, 4) || !aligned(factor_out, 4)) return PACE_ERR_INVALID_ARG;
    Tensors t = {};
    t.n = n_tensors, t.sizes = sizes, t.grads = grads, t.grad_dtypes = grad_dtypes;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < grad_norm_ws_bytes(t)) return PACE_ERR_WORKSPACE;
    return hip_status(launch_grad_norm(t, max_norm, norm_out, factor_out, workspace, (hipStream_t)stream));
}

int pace_adamw(int64_t n_tensors, const int64_t *sizes, void *const *params, const int32_t *param_dtypes, const void *const *grads,
               const int32_t *grad_dtypes, int state_bits, void *const *exp_avg, void *const *exp_avg_sq, float *const *scales,
               void *const *copies, const int32_t *copy_dtypes, const float *weight_decay, const pace_adamw_params *hyper,
               const float *grad_scale, const double *schedule, void *stream) {
    const TimerScope timers;
    if (!hyper || (state_bits != 32 && state_bits != 8) || !sizes_ok(n_tensors, sizes)) return PACE_ERR_INVALID_ARG;
    if (n_tensors > 0 && (!param_dtypes || !grad_dtypes)) return PACE_ERR_INVALID_ARG;
    const uintptr_t moment = state_bits == 32 ? 4 : 1;
    if (!each_ok(n_tensors, sizes, params, param_dtypes, 0) || !each_ok(n_tensors, sizes, grads, grad_dtypes, 0) ||
        !each_ok(n_tensors, sizes, exp_avg, nullptr, moment) || !each_ok(n_tensors, sizes, exp_avg_sq, nullptr, moment))
        return PACE_ERR_INVALID_ARG;
    if (state_bits == 8 && !each_ok(n_tensors, sizes, (const void *const *)scales, nullptr, 4)) return PACE_ERR_INVALID_ARG;
    for (int64_t i = 0; i < n_tensors; ++i) {
        if (copies && copies[i] && (!copy_dtypes || (copy_dtypes[i] != kBf16 && copy_dtypes[i] != kF16) || !aligned(copies[i], 2)))
            return PACE_ERR_INVALID_ARG;
        if (weight_decay && !(weight_decay[i] >= 0.0f && weight_decay[i] <= 1e30f)) return PACE_ERR_INVALID_ARG;
    }
    const double b1 = hyper->beta1, b2 = hyper->beta2;
    if (!(b1 >= 0.0 && b1 < 1.0) || !(b2 >= 0.0 && b2 < 1.0) || !(hyper->eps >= 1e-30 && hyper->eps <= 1e30)) return PACE_ERR_INVALID_ARG;
    // What a block loses where its V counts as zero is below eps / 256 then (adamw.hip).
    if (state_bits == 8 && !(hyper->eps * sqrt(1.0 - b2) >= 0x1p-55)) return PACE_ERR_INVALID_ARG;
    if (!aligned(grad_scale, 4) || !aligned(schedule, 8)) return PACE_ERR_INVALID_ARG;
    AdamHyper h = {0.0, b1, b2, hyper->eps, 1.0, 1.0, grad_scale, schedule};
    if (!schedule) {
        if (!isfinite(hyper->lr) || hyper->step < 1) return PACE_ERR_INVALID_ARG;
        h.lr = hyper->lr;
        h.keep1 = 1.0 - pow(b1, (double)hyper->step);
        h.keep2 = 1.0 - pow(b2, (double)hyper->step);
    }
    const Tensors t = {n_tensors, sizes, params, param_dtypes, grads, grad_dtypes, exp_avg, exp_avg_sq, scales, copies, copy_dtypes, weight_decay};
    return hip_status(launch_adamw(t, state_bits, h, (hipStream_t)stream));
}

int pace_adamw_unpack(int64_t n_tensors, const int64_t *sizes, const int8_t *const *exp_avg, const uint8_t *const *exp_avg_sq,
                      const float *const *scales, float *const *exp_avg_out, float *const *exp_avg_sq_out, void *stream) {
    const TimerScope timers;
    if (!sizes_ok(n_tensors, sizes) || (!exp_avg_out && !exp_avg_sq_out && n_tensors > 0)) return PACE_ERR_INVALID_ARG;
    if (!each_ok(n_tensors, sizes, (const void *const *)exp_avg, nullptr, 1) || !each_ok(n_tensors, sizes, (const void *const *)exp_avg_sq, nullptr, 1) ||
        !each_ok(n_tensors, sizes, (const void *const *)scales, nullptr, 4))
        return PACE_ERR_INVALID_ARG;
    if ((exp_avg_out && !each_ok(n_tensors, sizes, (const void *const *)exp_avg_out, nullptr, 4)) ||
        (exp_avg_sq_out && !each_ok(n_tensors, sizes, (const void *const *)exp_avg_sq_out, nullptr, 4)))
        return PACE_ERR_INVALID_ARG;
    Tensors t = {};
    t.n = n_tensors, t.sizes = sizes;
    t.m = (void *const *)exp_avg, t.v = (void *const *)exp_avg_sq, t.scales = (float *const *)scales;
    return hip_status(launch_adamw_unpack(t, exp_avg_out, exp_avg_sq_out, (hipStream_t)stream));
}

static_assert(PACE_ADAMW_BLOCK == kAdamBlock, "elements of a scale");
static_assert(PACE_PHASE_COUNT == kPhaseCount, "phase count");

int pace_time_next_kernel(int phase, void *start_event, void *stop_event) {
    if (phase < 0 || phase >= PACE_PHASE_COUNT) return PACE_ERR_INVALID_ARG;
    if ((start_event == nullptr) != (stop_event == nullptr)) return PACE_ERR_INVALID_ARG;
    g_phase_timer[phase][0] = (hipEvent_t)start_event;
    g_phase_timer[phase][1] = (hipEvent_t)stop_event;
    return PACE_OK;
}

int pace_validate(const int32_t *tags, const int64_t *offsets, int64_t n_traj, int64_t n_tokens,
                  const int32_t *completion, int32_t current_version, const double *window_sorted,
                  int64_t window_n, int32_t *err_word_out, void *stream) {
    const TimerScope timers;
    if (n_traj < 0 || n_traj >= INT32_MAX || n_tokens < 0 || window_n < 0) return PACE_ERR_INVALID_ARG;
    if (!offsets || !err_word_out || (n_traj > 0 && !completion) || (n_tokens > 0 && !tags) ||
        (window_n > 0 && !window_sorted))
        return PACE_ERR_INVALID_ARG;
    if (!aligned(tags, 4) || !aligned(offsets, 8) || !aligned(completion, 4) ||
        !aligned(err_word_out, 4) || !aligned(window_sorted, 8))
        return PACE_ERR_INVALID_ARG;
    return hip_status(launch_validate(tags, offsets, n_traj, n_tokens, completion, current_version,
                                      window_sorted, window_n, err_word_out, (hipStream_t)stream));
}

}  // extern "C"
