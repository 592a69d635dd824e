// Log-probabilities of given tokens for gfx950, with the entropy and the best
// alternatives of each row of logits, and their backward pass.
//
//   m = max z,  e_i = exp((z_i - m) / tau),  S = sum e,  logp = (z_t - m)/tau - log S
//   H = log S - (sum e_i (z_i - m)/tau) / S
//   dz_i = (g ([i = t] - p_i) - g_H p_i (log p_i + H)) / tau,   p = e / S
//
// Forward: one pass over the logits with the running maximum, sum and weighted
// sum of each thread, joined over the workgroup and, where a row is split over
// several workgroups, by a second small kernel. Everything is held in binary32
// in units of log2: u = z c - m c with c = log2(e)/tau, one fused step and one
// exp2 an element. The rounding of m c is the same for every u of a row, so it
// leaves S and u_t by the same factor and cancels in logp.
//
// Best alternatives: keys (logit in order, ~index), all different, so the set
// and its order do not depend on the order of arrival. After its first chunk a
// workgroup takes a bound that at least top_k of its threads' maxima reach; an
// element that reaches it is put into a list in LDS. A list that overflows
// (rows of many equal logits, rising rows) is given up and the part is read
// again, selecting by digits of the key.
#include "elem.hpp"
#include "kernels.hpp"

#pragma clang fp contract(off)

namespace pace {

namespace {

constexpr int kLpThreads = 512;
constexpr int kLpWaves = kLpThreads / kWave;
constexpr int kLpUnroll = 4;                       // 16-byte vectors a thread takes of a chunk
constexpr int kLpList = 1024;                      // candidates a workgroup keeps
constexpr float kLowest = -3.402823466e+38f;       // below no finite logit
constexpr float kFarLog2 = -1e30f;                 // stands for the logarithm of nothing, finite
constexpr float kLn2 = 0.693147180559945309f;

// log2 of the factor that brings sums against the maximum `from` to `to`; finite.
__device__ __forceinline__ float log2_shift(float from, float to, float c) {
    const float d = (from - to) * c;
    return d > kFarLog2 ? d : kFarLog2;
}
// log p of a logit z, with ls = log S: in natural units, where a mask of the
// type's lowest value stays a number.
__device__ __forceinline__ float log_prob(float z, float m, float ls, float inv_t) { return (z - m) * inv_t - ls; }

struct RowSum {
    float m, s, w;      // maximum; sum of 2^u; sum of 2^u u
};
// b's sums joined to a's. Both maxima are numbers (kLowest for nothing).
__device__ __forceinline__ RowSum joined(const RowSum &a, const RowSum &b, float c) {
    RowSum r;
    r.m = a.m > b.m ? a.m : b.m;
    const float da = log2_shift(a.m, r.m, c), db = log2_shift(b.m, r.m, c);
    const float fa = __builtin_amdgcn_exp2f(da), fb = __builtin_amdgcn_exp2f(db);
    r.s = a.s * fa + b.s * fb;
    r.w = (a.w + a.s * da) * fa + (b.w + b.s * db) * fb;
    return r;
}
__device__ __forceinline__ RowSum wave_joined(RowSum v, float c) {
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
        RowSum o;
        o.m = __shfl_xor(v.m, off, kWave);
        o.s = __shfl_xor(v.s, off, kWave);
        o.w = __shfl_xor(v.w, off, kWave);
        // the lower lane's sums first on both sides, so that every lane forms the same number
        v = (lane_id() & off) ? joined(o, v, c) : joined(v, o, c);
    }
    return v;
}

// An order-preserving key of a finite logit (-0 as +0).
__device__ __forceinline__ uint32_t logit_key(float z) {
    const uint32_t b = __builtin_bit_cast(uint32_t, z + 0.0f);
    return (b >> 31) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float key_logit(uint32_t k) {
    return __builtin_bit_cast(float, (k >> 31) ? (k & 0x7fffffffu) : ~k);
}
__device__ __forceinline__ uint64_t token_key(float z, int32_t i) {
    return ((uint64_t)logit_key(z) << 32) | (uint32_t)~i;
}
__device__ __forceinline__ int32_t key_token(uint64_t k) { return (int32_t)~(uint32_t)k; }

template <typename T>
__device__ __forceinline__ uint4 load_vec(const T *row, int64_t v) {
    return load_a1(row + v * kVecOf<T>);
}

// The row's outputs from its whole sums.
__device__ __forceinline__ void write_row(const LogprobOut &o, int64_t row, const RowSum &r, float zt, bool known,
                                          float inv_t) {
    const float ls = logf(r.s);
    // A row whose mask leaves nothing: no token has a probability.
    const bool none = r.s == 0.0f;
    const float nan = __builtin_nanf("");
    float lp = log_prob(zt, r.m, ls, inv_t);
    if (none) lp = -__builtin_inff();
    o.logp[row] = known ? lp : nan;
    if (o.entropy) o.entropy[row] = none ? 0.0f : ls - kLn2 * (r.w / r.s);
    if (o.stats) {
        o.stats[2 * row] = r.m;
        o.stats[2 * row + 1] = r.s;
    }
}
__device__ __forceinline__ void write_skipped(const LogprobOut &o, int64_t row, int top_k, int t) {
    if (t == 0) {
        o.logp[row] = 0.0f;
        if (o.entropy) o.entropy[row] = 0.0f;
        if (o.stats) o.stats[2 * row] = o.stats[2 * row + 1] = 0.0f;
    }
    if (t < top_k) {
        o.top_ids[row * top_k + t] = -1;
        o.top_logp[row * top_k + t] = -__builtin_inff();
    }
}
__device__ __forceinline__ void write_top(const LogprobOut &o, int64_t row, int top_k, int rank, uint64_t key,
                                          const RowSum &r, float inv_t) {
    o.top_ids[row * top_k + rank] = key ? key_token(key) : -1;
    const float lp = log_prob(key_logit((uint32_t)(key >> 32)), r.m, logf(r.s), inv_t);
    o.top_logp[row * top_k + rank] = key ? lp : -__builtin_inff();
}

struct TopLds {
    uint32_t most[kLpThreads];     // keys of the threads' maxima over their first chunk
    uint64_t list[kLpList];
    uint32_t hist[256];
    uint32_t n;
};

// The largest t of 16 high bits with at least k of the workgroup's maxima at or
// above it, as a logit. Every wave counts all maxima by itself.
__device__ __forceinline__ float top_bound(const TopLds &lds, int k) {
    uint32_t key[kLpWaves];
#pragma unroll
    for (int j = 0; j < kLpWaves; ++j) key[j] = lds.most[j * kWave + lane_id()];
    uint32_t t = 0;
#pragma unroll 1
    for (int bit = 31; bit >= 16; --bit) {
        const uint32_t at = t | (1u << bit);
        int n = 0;
#pragma unroll
        for (int j = 0; j < kLpWaves; ++j) n += __popcll(ballot(key[j] >= at));
        if (n >= k) t = at;
    }
    return key_logit(t);
}

// Elements [0, len) of a part, each with its index, to f, all threads alike.
template <typename T, typename F>
__device__ __forceinline__ void each_of_part(const T *row, int64_t v0, int64_t v1, int64_t tail0, int64_t tail1, F f) {
    constexpr int V = kVecOf<T>;
    for (int64_t v = v0 + threadIdx.x; v < v1; v += kLpThreads) {
        float z[V];
        unpack16<T>(load_vec(row, v), z);
#pragma unroll
        for (int e = 0; e < V; ++e) f(z[e], (int32_t)(v * V + e));
    }
    const int64_t i = tail0 + threadIdx.x;
    if (i < tail1) f(to_f32(row[i]), (int32_t)i);
}

// The top_k largest keys of a part whose list overflowed: the top_k-th key is
// found by its eight digits, each a count over the part.
template <typename T>
__device__ void select_by_digits(TopLds &lds, const T *row, int64_t v0, int64_t v1, int64_t tail0, int64_t tail1,
                                 int k) {
    uint64_t prefix = 0;
    uint32_t want = (uint32_t)k;
#pragma unroll 1
    for (int shift = 56; shift >= 0; shift -= 8) {
        __syncthreads();
        if (threadIdx.x < 256) lds.hist[threadIdx.x] = 0;
        __syncthreads();
        each_of_part(row, v0, v1, tail0, tail1, [&](float z, int32_t i) {
            const uint64_t key = token_key(z, i);
            const bool in = z >= kLowest && (shift == 56 || (key >> (shift + 8)) == (prefix >> (shift + 8)));
            if (in) {
                const uint32_t digit = (uint32_t)(key >> shift) & 255u;
                // rows of equal logits: one count for lanes with the same digit
                const uint32_t first = (uint32_t)__builtin_amdgcn_readfirstlane((int)digit);
                const uint64_t same = ballot(digit == first);
                if (digit != first) atomicAdd(&lds.hist[digit], 1u);
                else if ((same & lanes_below()) == 0) atomicAdd(&lds.hist[first], (uint32_t)__popcll(same));
            }
        });
        __syncthreads();
        // the digit of the want-th largest key (0 where the part holds fewer)
        uint32_t above = 0;
        int d = 255;
        for (; d > 0; --d) {
            const uint32_t h = lds.hist[d];
            if (above + h >= want) break;
            above += h;
        }
        want -= above;
        prefix |= (uint64_t)d << shift;
    }
    __syncthreads();
    if (threadIdx.x == 0) lds.n = 0;
    __syncthreads();
    each_of_part(row, v0, v1, tail0, tail1, [&](float z, int32_t i) {
        const uint64_t key = token_key(z, i);
        if (z >= kLowest && key >= prefix) {
            const uint32_t at = atomicAdd(&lds.n, 1u);
            if (at < (uint32_t)kLpList) lds.list[at] = key;
        }
    });
    __syncthreads();
}

template <typename T, bool kTop>
__global__ __launch_bounds__(kLpThreads) void logprob_kernel(const T *__restrict__ logits, int64_t vocab,
                                                             int64_t stride, const int32_t *__restrict__ ids, float c, float inv_t,
                                                             int top_k, int parts, LogprobOut out, RowSum *part_sum,
                                                             uint64_t *part_top) {
    constexpr int V = kVecOf<T>, U = kLpUnroll;
    __shared__ RowSum wsum[kLpWaves];
    __shared__ TopLds lds;      // unused, and so not allocated, without alternatives
    const int64_t row_i = blockIdx.x / (unsigned)parts;
    const int part = (int)(blockIdx.x % (unsigned)parts);
    const int t = threadIdx.x;
    const int32_t id = ids[row_i];
    if (id == -1) {                                  // the whole workgroup
        if (part == 0) write_skipped(out, row_i, kTop ? top_k : 0, t);
        return;
    }
    const T *row = logits + row_i * stride;
    const int64_t nv = vocab / V;
    const int64_t v0 = nv * part / parts, v1 = nv * (part + 1) / parts;
    const int64_t tail0 = part == parts - 1 ? nv * V : vocab;      // the last part takes the elements behind the vectors
    if (kTop && t == 0) lds.n = 0;

    RowSum r = {kLowest, 0.0f, 0.0f};
    float bound = -__builtin_inff();
    const float ninf = -__builtin_inff();
    auto take = [&](const float (&z)[U * V], int64_t vbase, bool first) {
        float m = z[0];
#pragma unroll
        for (int e = 1; e < U * V; ++e) m = __builtin_fmaxf(m, z[e]);
        const float mn = __builtin_fmaxf(r.m, m);
        const float d = log2_shift(r.m, mn, c), f = __builtin_amdgcn_exp2f(d);
        float s = r.s * f, w = (r.w + r.s * d) * f;
        r.m = mn;
#pragma unroll
        for (int e = 0; e < U * V; ++e) {
            const float u = (z[e] - mn) * c;
            const float x = __builtin_amdgcn_exp2f(u);
            s += x;
            w = __builtin_fmaf(x, __builtin_fmaxf(u, kFarLog2), w);      // nothing where x is: 0 times a finite number
        }
        r.s = s, r.w = w;
        if constexpr (kTop) {
            if (first) {
                lds.most[t] = logit_key(mn);
                __syncthreads();
                bound = top_bound(lds, top_k);
            }
            if (m >= bound) {
#pragma unroll
                for (int e = 0; e < U * V; ++e) {
                    if (z[e] >= bound) {
                        const uint32_t at = atomicAdd(&lds.n, 1u);
                        if (at < (uint32_t)kLpList)
                            lds.list[at] = token_key(z[e], (int32_t)((vbase + (int64_t)(e / V) * kLpThreads) * V + e % V));
                    }
                }
            }
        }
    };
    // The first chunk is taken by every thread, the elements behind the
    // vectors with it, so that the bound is known from there on.
    uint4 raw[U];
    auto load = [&](int64_t v) {
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int64_t at = v + (int64_t)k * kLpThreads;
            if (at < v1) raw[k] = load_vec(row, at);
        }
    };
    auto values = [&](int64_t v, float (&z)[U * V]) {
#pragma unroll
        for (int k = 0; k < U; ++k) {
            float x[V];
            unpack16<T>(raw[k], x);
            const bool in = v + (int64_t)k * kLpThreads < v1;
#pragma unroll
            for (int e = 0; e < V; ++e) z[k * V + e] = in ? x[e] : ninf;
        }
    };
#pragma unroll
    for (int k = 0; k < U; ++k) raw[k] = make_uint4(0, 0, 0, 0);
    {
        const int64_t v = v0 + t;
        float z[U * V];
        load(v);
        values(v, z);
        take(z, v, true);
    }
    for (int64_t v = v0 + t + (int64_t)U * kLpThreads; v < v1; v += (int64_t)U * kLpThreads) {
        float z[U * V];
        load(v);
        values(v, z);
        take(z, v, false);
    }
    if (tail0 + t < vocab) {
        const float x = to_f32(row[tail0 + t]);
        const RowSum one = {x > kLowest ? x : kLowest, 0.0f, 0.0f};
        r = joined(r, one, c);
        const float u = (x - r.m) * c, y = __builtin_amdgcn_exp2f(u);
        r.s += y;
        r.w = __builtin_fmaf(y, __builtin_fmaxf(u, kFarLog2), r.w);
        if (kTop && x >= bound && x >= kLowest) {
            const uint32_t at = atomicAdd(&lds.n, 1u);
            if (at < (uint32_t)kLpList) lds.list[at] = token_key(x, (int32_t)(tail0 + t));
        }
    }

    r = wave_joined(r, c);
    if (lane_id() == 0) wsum[t / kWave] = r;
    __syncthreads();
    r = wsum[0];
#pragma unroll
    for (int k = 1; k < kLpWaves; ++k) r = joined(r, wsum[k], c);
    if (parts > 1) {
        if (t == 0) part_sum[row_i * parts + part] = r;
    } else if (t == 0) {
        const bool known = id >= 0 && id < vocab;
        write_row(out, row_i, r, known ? to_f32(row[id]) : 0.0f, known, inv_t);
    }
    if constexpr (kTop) {
        if (lds.n > (uint32_t)kLpList) select_by_digits(lds, row, v0, v1, tail0, vocab, top_k);     // uniform
        const int n = (int)(lds.n < (uint32_t)kLpList ? lds.n : (uint32_t)kLpList);
        for (int i = t; i < n; i += kLpThreads) {
            const uint64_t key = lds.list[i];
            int rank = 0;
            for (int j = 0; j < n; ++j) rank += lds.list[j] > key ? 1 : 0;
            if (rank < top_k) {
                if (parts > 1) part_top[(row_i * parts + part) * top_k + rank] = key;
                else write_top(out, row_i, top_k, rank, key, r, inv_t);
            }
        }
        if (t >= n && t < top_k) {                   // fewer candidates than alternatives
            if (parts > 1) part_top[(row_i * parts + part) * top_k + t] = 0;
            else write_top(out, row_i, top_k, t, 0, r, inv_t);
        }
    }
}

// One wave a row: the parts' sums, and the alternatives from the heads of the
// parts' lists, each in order.
template <typename T>
__global__ __launch_bounds__(kWave) void logprob_join_kernel(const T *__restrict__ logits, int64_t vocab,
                                                             int64_t stride, const int32_t *__restrict__ ids, float c, float inv_t,
                                                             int top_k, int parts, LogprobOut out,
                                                             const RowSum *__restrict__ part_sum,
                                                             const uint64_t *__restrict__ part_top) {
    const int64_t row_i = blockIdx.x;
    const int lane = lane_id();
    const int32_t id = ids[row_i];
    if (id == -1) return;                            // written by the first kernel
    RowSum r = {kLowest, 0.0f, 0.0f};
    if (lane < parts) r = part_sum[row_i * parts + lane];
    r = wave_joined(r, c);
    if (lane == 0) {
        const bool known = id >= 0 && id < vocab;
        write_row(out, row_i, r, known ? to_f32(logits[row_i * stride + id]) : 0.0f, known, inv_t);
    }
    if (top_k > 0) {
        const uint64_t *mine = part_top + (row_i * parts + lane) * top_k;
        int at = 0;
        uint64_t head = lane < parts ? mine[0] : 0;
        uint64_t key = 0;
        for (int k = 0; k < top_k; ++k) {
            const uint64_t best = wave_max_u64(head);
            if (lane == k) key = best;
            if (best != 0 && head == best) {         // keys are all different: one lane
                ++at;
                head = at < top_k ? mine[at] : 0;
            }
        }
        if (lane < top_k) write_top(out, row_i, top_k, lane, key, r, inv_t);
    }
}

constexpr int kLpbThreads = 256;

template <typename T, bool kEntropy>
__global__ __launch_bounds__(kLpbThreads) void logprob_backward_kernel(
    const T *logits, int64_t vocab, int64_t stride, const int32_t *__restrict__ ids, float c, double inv_t,
    const float *__restrict__ stats, const float *__restrict__ entropy, const float *__restrict__ g_logp,
    const float *__restrict__ g_entropy, T *grad, int64_t grad_stride, int parts) {
    constexpr int V = kVecOf<T>;
    const int64_t row_i = blockIdx.x / (unsigned)parts;
    const int part = (int)(blockIdx.x % (unsigned)parts);
    const int64_t nv = vocab / V;
    const int64_t v0 = nv * part / parts, v1 = nv * (part + 1) / parts;
    const T *row = logits + row_i * stride;
    T *to = grad + row_i * grad_stride;
    const int32_t id = ids[row_i];
    const float m = stats[2 * row_i], s = stats[2 * row_i + 1];
    if (id == -1 || s == 0.0f) {                     // skipped, or nothing left of the row
        for (int64_t v = v0 + threadIdx.x; v < v1; v += kLpbThreads) store_a1(to + v * V, make_uint4(0, 0, 0, 0));
        if (part == parts - 1 && nv * V + threadIdx.x < vocab) to[nv * V + threadIdx.x] = from_f32<T>(0.0f);
        return;
    }
    // The row's factors are rounded once.
    const float g = (float)((double)g_logp[row_i] * inv_t);
    const float k0 = -g / s;
    float kh = 0.0f, hh = 0.0f;                       // with entropy: p (g + gH (log p + H))
    if (kEntropy) {
        kh = (float)(-(double)g_entropy[row_i] * inv_t / s * 0.69314718055994530942);
        hh = entropy[row_i] / kLn2 - log2f(s);        // log p + H = ln2 (u + hh)
    }
    auto of = [&](float z) {
        const float u = (z - m) * c;
        const float x = __builtin_amdgcn_exp2f(u);
        if (!kEntropy) return x * k0;
        return x * __builtin_fmaf(__builtin_fmaxf(u, kFarLog2) + hh, kh, k0);
    };
    for (int64_t v = v0 + threadIdx.x; v < v1; v += kLpbThreads) {
        float z[V];
        unpack16<T>(load_vec(row, v), z);
        const int64_t own = (int64_t)id - v * V;
#pragma unroll
        for (int e = 0; e < V; ++e) z[e] = of(z[e]);
        if (own >= 0 && own < V) {
#pragma unroll
            for (int e = 0; e < V; ++e) z[e] += e == (int)own ? g : 0.0f;
        }
        store_a1(to + v * V, pack16<T>(z));
    }
    if (part == parts - 1 && nv * V + threadIdx.x < vocab) {
        const int64_t i = nv * V + threadIdx.x;
        to[i] = from_f32<T>(of(to_f32(row[i])) + (i == id ? g : 0.0f));
    }
}

}  // namespace

size_t logprob_ws_bytes(int64_t rows, int64_t vocab, int top_k) {
    const int64_t parts = logprob_parts(rows, vocab);
    if (parts <= 1) return 256;
    return align256((size_t)(rows * parts) * sizeof(RowSum)) + align256((size_t)(rows * parts) * top_k * 8) + 256;
}

hipError_t launch_token_logprob(const void *logits, int dtype, int64_t rows, int64_t vocab, int64_t stride,
                                const int32_t *ids, double temperature, int top_k, const LogprobOut &out, void *ws,
                                hipStream_t stream) {
    if (rows == 0) return hipSuccess;
    const int parts = (int)logprob_parts(rows, vocab);
    RowSum *sum = (RowSum *)ws;
    uint64_t *top = (uint64_t *)((char *)ws + align256((size_t)(rows * parts) * sizeof(RowSum)));
    const float c = (float)(1.44269504088896340736 / temperature), inv_t = (float)(1.0 / temperature);
    return with_elem(dtype, [&](auto tag) {
        using T = decltype(tag);
        const dim3 grid((unsigned)(rows * parts));
        hipError_t e = top_k > 0 ? launch(kPhaseAux, logprob_kernel<T, true>, grid, dim3(kLpThreads), stream, (const T *)logits,
                                          vocab, stride, ids, c, inv_t, top_k, parts, out, sum, top)
                                 : launch(kPhaseAux, logprob_kernel<T, false>, grid, dim3(kLpThreads), stream, (const T *)logits,
                                          vocab, stride, ids, c, inv_t, 0, parts, out, sum, top);
        if (e == hipSuccess && parts > 1)
            e = launch(-1, logprob_join_kernel<T>, dim3((unsigned)rows), dim3(kWave), stream, (const T *)logits, vocab, stride,
                       ids, c, inv_t, top_k, parts, out, (const RowSum *)sum, (const uint64_t *)top);
        return e;
    });
}

hipError_t launch_token_logprob_backward(const void *logits, int dtype, int64_t rows, int64_t vocab, int64_t stride,
                                         const int32_t *ids, double temperature, const float *stats,
                                         const float *entropy, const float *g_logp, const float *g_entropy, void *grad,
                                         int64_t grad_stride, hipStream_t stream) {
    if (rows == 0) return hipSuccess;
    const int parts = (int)logprob_backward_parts(rows, vocab);
    const float c = (float)(1.44269504088896340736 / temperature);
    const double inv_t = 1.0 / temperature;
    return with_elem(dtype, [&](auto tag) {
        using T = decltype(tag);
        const dim3 grid((unsigned)(rows * parts));
        return g_entropy ? launch(kPhaseAux, logprob_backward_kernel<T, true>, grid, dim3(kLpbThreads), stream,
                                  (const T *)logits, vocab, stride, ids, c, inv_t, stats, entropy, g_logp, g_entropy,
                                  (T *)grad, grad_stride, parts)
                         : launch(kPhaseAux, logprob_backward_kernel<T, false>, grid, dim3(kLpbThreads), stream,
                                  (const T *)logits, vocab, stride, ids, c, inv_t, stats, entropy, g_logp, g_entropy,
                                  (T *)grad, grad_stride, parts);
    });
}

}  // namespace pace
