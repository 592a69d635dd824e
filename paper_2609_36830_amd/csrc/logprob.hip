// Log-probabilities of given tokens for gfx950, with the entropy and the best
// alternatives of each row of logits, and their backward pass.
//
//   m = max z,  e_i = exp((z_i - m) / tau),  S = sum e,  logp = (z_t - m)/tau - log S
//   H = log S - (sum e_i (z_i - m)/tau) / S
//   dz_i = (g ([i = t] - p_i) - g_H p_i (log p_i + H)) / tau,   p = e / S
//
// Forward: one pass over the logits with the running maximum, sum and weighted
// sum of each thread, joined over the workgroup and, where a row is split over
// several waves or workgroups, by a second small kernel. Everything is held in
// binary32 in units of log2: u = (z - m) c with c = log2(e)/tau and one exp2 an
// element. The difference is taken first: z c - m c would be one step less, but
// its rounding grows with |m c|, and logits of the type's lowest value leave the
// range. The exponents are rounded by 2^-24 of |u|, where p is at most 2^u.
//
// A part of a row (all of it where there are rows enough) is taken by one wave
// or by a workgroup of eight, by its length; the parts are as many as fill the
// chip. Bound by HBM, with 12 vector instructions an element close behind: 3074
// scored rows of 150000 bfloat16 take 171 us (5.4 TB/s; a device copy 4.8), 4096
// with the backward pass 250 + 445 (4.9 and 5.5 TB/s: the logits, 1.2 GB, are read
// again from HBM), 1023 of 50021 in binary32 with an entropy
// gradient 49 + 71. 48 rows with 20 alternatives take 15.8 us, of which two
// launches' beginnings and the dependent reads of the second (bound, holders,
// list, rank) are all but 3. Many short rows with alternatives are bound by vector
// instructions, issued in 82% of the cycles: 8000 of 5000 with 20 take 30 us, without 19.
//
// Best alternatives: keys (logit in order, ~index), all different, so the set
// and its order do not depend on the order of arrival. The pass over the logits
// is the same as without them: it ends with the largest logit of every thread,
// and a bound that at least top_k of these reach. Only the threads that reach
// it hold candidates; their logits are read once more, by all threads together,
// and what reaches the bound is listed in LDS and ranked. A list that overflows
// (rows of many equal logits) is given up and the part is read again, selecting
// by digits of the key.
#include "elem.hpp"
#include "kernels.hpp"

#pragma clang fp contract(off)

namespace pace {

namespace {

constexpr int kLpThreads = 512;                    // of a workgroup: eight waves for a part, or a wave for each of eight
constexpr int kLpAgain = 4;                        // vectors a thread reads again at a time
constexpr int kLpUnroll = 4;                       // 16-byte vectors a thread takes of a chunk
constexpr float kLowest = -3.402823466e+38f;       // below no finite logit
constexpr float kFarLog2 = -256.0f;                // stands for the logarithm of what 2^u has as 0; its products with factors stay finite
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
// v against the maximum m.
__device__ __forceinline__ RowSum against(const RowSum &v, float m, float c) {
    const float d = log2_shift(v.m, m, c), f = __builtin_amdgcn_exp2f(d);
    return {m, v.s * f, (v.w + v.s * d) * f};
}
// Reductions in lane order's tree (row shifts and row broadcasts), in every lane.
__device__ __forceinline__ float wave_max_f32(float v) {
    const uint32_t low = __builtin_bit_cast(uint32_t, kLowest);
    auto step = [&](uint32_t got) { v = __builtin_fmaxf(v, __builtin_bit_cast(float, got)); };
    step(dpp_u32<0x111, 0xf>(low, __builtin_bit_cast(uint32_t, v)));
    step(dpp_u32<0x112, 0xf>(low, __builtin_bit_cast(uint32_t, v)));
    step(dpp_u32<0x114, 0xf>(low, __builtin_bit_cast(uint32_t, v)));
    step(dpp_u32<0x118, 0xf>(low, __builtin_bit_cast(uint32_t, v)));
    step(dpp_u32<0x142, 0xa>(low, __builtin_bit_cast(uint32_t, v)));
    step(dpp_u32<0x143, 0xc>(low, __builtin_bit_cast(uint32_t, v)));
    return __builtin_bit_cast(float, readlane_i32(__builtin_bit_cast(int32_t, v), kWave - 1));
}
__device__ __forceinline__ float wave_sum_f32(float v) {
    auto step = [&](uint32_t got) { v += __builtin_bit_cast(float, got); };
    step(dpp_u32<0x111, 0xf>(0u, __builtin_bit_cast(uint32_t, v)));
    step(dpp_u32<0x112, 0xf>(0u, __builtin_bit_cast(uint32_t, v)));
    step(dpp_u32<0x114, 0xf>(0u, __builtin_bit_cast(uint32_t, v)));
    step(dpp_u32<0x118, 0xf>(0u, __builtin_bit_cast(uint32_t, v)));
    step(dpp_u32<0x142, 0xa>(0u, __builtin_bit_cast(uint32_t, v)));
    step(dpp_u32<0x143, 0xc>(0u, __builtin_bit_cast(uint32_t, v)));
    return __builtin_bit_cast(float, readlane_i32(__builtin_bit_cast(int32_t, v), kWave - 1));
}
__device__ __forceinline__ RowSum wave_joined(RowSum v, float c) {
    v = against(v, wave_max_f32(v.m), c);
    return {v.m, wave_sum_f32(v.s), wave_sum_f32(v.w)};
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

// What the kWaves waves that take a part share.
template <int kWaves>
struct Part {
    static constexpr int kThreads = kWaves * kWave, kGroups = kLpThreads / kThreads;
    static constexpr int kList = kWaves == 1 ? 512 : 1024;      // candidates
    struct Sums {
        RowSum wave[kWaves];
    };
    struct Top {
        uint64_t list[kList];
        uint32_t most[kThreads];                     // keys of the threads' maxima
        uint32_t holds[kThreads];                    // threads that hold candidates
        uint32_t hist[256];
        uint32_t n, n_holds;
    };
    // Orders the LDS accesses of the part's waves.
    static __device__ __forceinline__ void sync() {
        if constexpr (kWaves == 1) {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        } else {
            __syncthreads();
        }
    }
};

// The largest t of 16 high bits with at least k of the part's maxima at or
// above it, as a logit. Every wave counts all maxima by itself.
template <int kWaves>
__device__ __forceinline__ float top_bound(const uint32_t *most, int k) {
    uint32_t key[kWaves];
#pragma unroll
    for (int j = 0; j < kWaves; ++j) key[j] = most[j * kWave + lane_id()];
    uint32_t t = 0;
#pragma unroll 1
    for (int bit = 31; bit >= 16; --bit) {
        const uint32_t at = t | (1u << bit);
        int n = 0;
#pragma unroll
        for (int j = 0; j < kWaves; ++j) n += __popcll(ballot(key[j] >= at));
        if (n >= k) t = at;
    }
    return key_logit(t);
}

// A part of a row: vectors [v0, v1) and the elements [tail0, tail1) behind the row's vectors.
template <typename T>
struct Span {
    const T *row;
    int64_t v0, v1, tail0, tail1;
};

// Every element of a part with its index to f, the part's threads alike.
template <int kThreads, typename T, typename F>
__device__ __forceinline__ void each_of_part(const Span<T> &p, int t, F f) {
    constexpr int V = kVecOf<T>;
    for (int64_t v = p.v0 + t; v < p.v1; v += kThreads) {
        float z[V];
        unpack16<T>(load_vec(p.row, v), z);
#pragma unroll
        for (int e = 0; e < V; ++e) f(z[e], (int32_t)(v * V + e));
    }
    if (p.tail0 + t < p.tail1) f(to_f32(p.row[p.tail0 + t]), (int32_t)(p.tail0 + t));
}

// The k largest keys of a part whose list overflowed: the k-th key is found by
// its eight digits, each a count over the part.
template <int kWaves, typename T>
__device__ void select_by_digits(typename Part<kWaves>::Top &lds, const Span<T> &p, int t, int k) {
    using G = Part<kWaves>;
    uint64_t prefix = 0;
    uint32_t want = (uint32_t)k;
#pragma unroll 1
    for (int shift = 56; shift >= 0; shift -= 8) {
        G::sync();
        for (int i = t; i < 256; i += G::kThreads) lds.hist[i] = 0;
        G::sync();
        each_of_part<G::kThreads>(p, t, [&](float z, int32_t i) {
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
        G::sync();
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
    G::sync();
    if (t == 0) lds.n = 0;
    G::sync();
    each_of_part<G::kThreads>(p, t, [&](float z, int32_t i) {
        const uint64_t key = token_key(z, i);
        if (z >= kLowest && key >= prefix) {
            const uint32_t at = atomicAdd(&lds.n, 1u);
            if (at < (uint32_t)G::kList) lds.list[at] = key;
        }
    });
    G::sync();
}

// The k largest keys of a part, in no order, in lds.list; their number. `most`:
// the largest logit of this thread's share, which is vec_of(t, i) for i < each
// (a vector's number, p.v1 for none) and, behind the vectors, the element t.
template <int kWaves, typename T, typename VecOf>
__device__ __forceinline__ int part_top(typename Part<kWaves>::Top &lds, const Span<T> &p, int t, float most, int k, uint32_t each,
                                        VecOf vec_of) {
    using G = Part<kWaves>;
    constexpr int V = kVecOf<T>;
    if (t == 0) lds.n = lds.n_holds = 0;
    lds.most[t] = logit_key(most);
    G::sync();
    const float bound = top_bound<kWaves>(lds.most, k);
    if (most >= bound) lds.holds[atomicAdd(&lds.n_holds, 1u)] = (uint32_t)t;
    G::sync();
    // A lane's `count` candidates take places behind those of the lanes before
    // it: one addition to the list's length by a wave.
    auto place = [&](uint32_t count) -> uint32_t {
        const uint32_t incl = wave_incl_scan_u32(count), total = (uint32_t)readlane_i32((int32_t)incl, kWave - 1);
        if (total == 0) return 0;
        uint32_t base = 0;
        if (lane_id() == 0) base = atomicAdd(&lds.n, total);
        return (uint32_t)readlane_i32((int32_t)base, 0) + incl - count;
    };
    const uint32_t all = (uint32_t)readlane_i32((int32_t)(lds.n_holds * each), 0);
    for (uint32_t q0 = 0; q0 < all; q0 += kLpAgain * G::kThreads) {
        uint4 raw[kLpAgain];                         // on their way together
        int64_t v[kLpAgain];
#pragma unroll
        for (int k = 0; k < kLpAgain; ++k) {
            const uint32_t q = q0 + (uint32_t)k * G::kThreads + t, h = q / each;
            v[k] = q < all ? vec_of(lds.holds[h], q - h * each) : p.v1;
            if (v[k] < p.v1) raw[k] = load_vec(p.row, v[k]);
        }
#pragma unroll
        for (int k = 0; k < kLpAgain; ++k) {
            float z[V];
            uint32_t count = 0;
            if (v[k] < p.v1) {
                unpack16<T>(raw[k], z);
#pragma unroll
                for (int e = 0; e < V; ++e) count += z[e] >= bound ? 1u : 0u;
            }
            uint32_t at = place(count);
            if (count) {
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (z[e] >= bound) {
                        if (at < (uint32_t)G::kList) lds.list[at] = token_key(z[e], (int32_t)(v[k] * V + e));
                        ++at;
                    }
            }
        }
    }
    const float last = p.tail0 + t < p.tail1 ? to_f32(p.row[p.tail0 + t]) : __builtin_nanf("");
    const uint32_t at = place(last >= bound ? 1u : 0u);
    if (last >= bound && at < (uint32_t)G::kList) lds.list[at] = token_key(last, (int32_t)(p.tail0 + t));
    G::sync();
    if (lds.n > (uint32_t)G::kList) select_by_digits<kWaves>(lds, p, t, k);      // the same for all
    return (int)(lds.n < (uint32_t)G::kList ? lds.n : (uint32_t)G::kList);
}

// The n listed keys' ranks, and the top_k first.
template <int kThreads>
__device__ __forceinline__ void write_tops(const uint64_t *list, int n, const LogprobOut &out, int64_t row_i, int top_k, int t,
                                           const RowSum &r, float inv_t) {
    for (int i = t; i < n; i += kThreads) {
        const uint64_t key = list[i];
        int rank = 0;
#pragma unroll 8
        for (int j = 0; j < n; ++j) rank += list[j] > key ? 1 : 0;
        if (rank < top_k) write_top(out, row_i, top_k, rank, key, r, inv_t);
    }
    if (t >= n && t < top_k) write_top(out, row_i, top_k, t, 0, r, inv_t);      // fewer candidates than alternatives
}

template <typename T, bool kTop, int kWaves>
__global__ __launch_bounds__(kLpThreads) void logprob_kernel(const T *__restrict__ logits, int64_t vocab, int64_t rows,
                                                             int64_t stride, const int32_t *__restrict__ ids, float c, float inv_t,
                                                             int top_k, int parts, LogprobOut out, RowSum *part_sum,
                                                             float *part_most) {
    using G = Part<kWaves>;
    constexpr int V = kVecOf<T>, U = kLpUnroll;
    __shared__ typename G::Sums sums;                // of a workgroup that takes one part
    __shared__ __attribute__((aligned(16))) typename G::Top tops[kTop ? G::kGroups : 1];
    const int group = kWaves == 1 ? readlane_i32((int)threadIdx.x / kWave, 0) : 0;
    const int t = kWaves == 1 ? lane_id() : (int)threadIdx.x;
    const int64_t unit = (int64_t)blockIdx.x * G::kGroups + group;
    const int64_t row_i = unit / parts;
    const int part = (int)(unit - row_i * parts);
    if (row_i >= rows) return;                       // waves of their own: no barrier of the workgroup below
    const int32_t id = ids[row_i];
    if (id == -1) {
        if (part == 0) write_skipped(out, row_i, kTop ? top_k : 0, t);
        return;
    }
    const int64_t nv = vocab / V;
    // The last part takes the elements behind the vectors.
    const Span<T> p{logits + row_i * stride, nv * part / parts, nv * (part + 1) / parts, part == parts - 1 ? nv * V : vocab, vocab};

    RowSum r = {kLowest, 0.0f, 0.0f};
    const float ninf = -__builtin_inff();
    for (int64_t v = p.v0 + t; v < p.v1; v += (int64_t)U * G::kThreads) {
        uint4 raw[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int64_t at = v + (int64_t)k * G::kThreads;
            raw[k] = make_uint4(0, 0, 0, 0);
            if (at < p.v1) raw[k] = load_vec(p.row, at);
        }
        float z[U * V];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            float x[V];
            unpack16<T>(raw[k], x);
            const bool in = v + (int64_t)k * G::kThreads < p.v1;
#pragma unroll
            for (int e = 0; e < V; ++e) z[k * V + e] = in ? x[e] : ninf;
        }
        float m = z[0];
#pragma unroll
        for (int e = 1; e < U * V; ++e) m = __builtin_fmaxf(m, z[e]);
        r = against(r, __builtin_fmaxf(r.m, m), c);
#pragma unroll
        for (int e = 0; e < U * V; ++e) {
            const float u = (z[e] - r.m) * c;
            const float x = __builtin_amdgcn_exp2f(u);
            r.s += x;
            r.w = __builtin_fmaf(x, __builtin_fmaxf(u, kFarLog2), r.w);      // nothing where x is: 0 times a finite number
        }
    }
    if (p.tail0 + t < p.tail1) {
        const float x = to_f32(p.row[p.tail0 + t]);
        r = against(r, __builtin_fmaxf(r.m, x), c);
        const float u = (x - r.m) * c, y = __builtin_amdgcn_exp2f(u);
        r.s += y;
        r.w = __builtin_fmaf(y, __builtin_fmaxf(u, kFarLog2), r.w);
    }
    const float most = r.m;
    r = wave_joined(r, c);
    if constexpr (kWaves > 1) {
        if (lane_id() == 0) sums.wave[threadIdx.x / kWave] = r;
        __syncthreads();
        float m = sums.wave[0].m;
#pragma unroll
        for (int k = 1; k < kWaves; ++k) m = __builtin_fmaxf(m, sums.wave[k].m);
        RowSum all = against(sums.wave[0], m, c);
#pragma unroll
        for (int k = 1; k < kWaves; ++k) {
            const RowSum o = against(sums.wave[k], m, c);
            all.s += o.s;
            all.w += o.w;
        }
        r = all;
    }
    if (t == 0) {
        if (parts > 1) {
            part_sum[unit] = r;
        } else {
            const bool known = id >= 0 && id < vocab;
            write_row(out, row_i, r, known ? to_f32(p.row[id]) : 0.0f, known, inv_t);
        }
    }
    if constexpr (kTop) {
        if (parts > 1) {
            part_most[unit * G::kThreads + t] = most;
            return;
        }
        auto &lds = tops[group];
        const int n = part_top<kWaves>(lds, p, t, most, top_k, (uint32_t)((p.v1 + G::kThreads - 1) / G::kThreads),
                                       [&](uint32_t h, uint32_t i) { return (int64_t)h + (int64_t)i * G::kThreads; });
        write_tops<G::kThreads>(lds.list, n, out, row_i, top_k, t, r, inv_t);
    }
}

// Rows in parts: a wave joins the parts' sums; for alternatives a workgroup of
// eight waves, each of whose threads stands for the threads of the first kernel
// of a number up to a multiple of its own.
template <typename T, bool kTop>
__global__ __launch_bounds__(kTop ? kLpThreads : kWave) void logprob_join_kernel(const T *__restrict__ logits, int64_t vocab,
                                                             int64_t stride, const int32_t *__restrict__ ids, float c, float inv_t,
                                                             int top_k, int parts, int part_threads, LogprobOut out,
                                                             const RowSum *__restrict__ part_sum,
                                                             const float *__restrict__ part_most) {
    using G = Part<8>;
    __shared__ __attribute__((aligned(16))) typename G::Top lds[1];      // unused, and so not allocated, without alternatives
    const int64_t row_i = blockIdx.x;
    const int t = threadIdx.x;
    const int32_t id = ids[row_i];
    // on their way before the id is known: a row that is not scored has nothing here
    RowSum r = {kLowest, 0.0f, 0.0f};
    if (lane_id() < parts) r = part_sum[row_i * parts + lane_id()];
    const T *row = logits + row_i * stride;
    float most = kLowest;
    const uint32_t threads = (uint32_t)(parts * part_threads);
    if constexpr (kTop) {
#pragma unroll 4
        for (uint32_t u = t; u < threads; u += kLpThreads) most = __builtin_fmaxf(most, part_most[row_i * threads + u]);
    }
    if (id == -1) return;                            // written by the first kernel
    r = wave_joined(r, c);                           // every wave
    if (t == 0) {
        const bool known = id >= 0 && id < vocab;
        write_row(out, row_i, r, known ? to_f32(row[id]) : 0.0f, known, inv_t);
    }
    if constexpr (kTop) {
        constexpr int V = kVecOf<T>;
        const int64_t nv = vocab / V;
        const Span<T> p{row, 0, nv, nv * V, vocab};
        const uint32_t shares = (threads + kLpThreads - 1) / kLpThreads;
        const uint32_t vecs = (uint32_t)((nv / parts + 1 + part_threads - 1) / part_threads);      // of a thread, at most
        const int n = part_top<8>(lds[0], p, t, most, top_k, shares * vecs, [&](uint32_t h, uint32_t i) {
            const uint32_t u = h + i / vecs * kLpThreads;
            if (u >= threads) return nv;
            const int64_t part = u / (uint32_t)part_threads, at = u % (uint32_t)part_threads;
            const int64_t v = nv * part / parts + at + (int64_t)(i % vecs) * part_threads;
            return v < nv * (part + 1) / parts ? v : nv;
        });
        write_tops<kLpThreads>(lds[0].list, n, out, row_i, top_k, t, r, inv_t);
    }
}

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
    const LogprobPlan plan = logprob_plan(rows, vocab, top_k);
    if (plan.parts <= 1) return 256;
    const size_t units = (size_t)(rows * plan.parts);
    return align256(units * sizeof(RowSum)) + (top_k > 0 ? align256(units * plan.waves * kWave * sizeof(float)) : 0) + 256;
}

hipError_t launch_token_logprob(const void *logits, int dtype, int64_t rows, int64_t vocab, int64_t stride,
                                const int32_t *ids, double temperature, int top_k, const LogprobOut &out, void *ws,
                                hipStream_t stream) {
    if (rows == 0) return hipSuccess;
    const LogprobPlan plan = logprob_plan(rows, vocab, top_k);
    const int parts = (int)plan.parts;
    RowSum *sum = (RowSum *)ws;
    float *most = (float *)((char *)ws + align256((size_t)(rows * parts) * sizeof(RowSum)));
    const float c = (float)(1.44269504088896340736 / temperature), inv_t = (float)(1.0 / temperature);
    return with_elem(dtype, [&](auto tag) {
        using T = decltype(tag);
        // Rows in parts are few, and go in one launch.
        auto first = [&](auto kernel, int64_t groups) {
            return in_launches((rows * parts + groups - 1) / groups, kLpThreads, [&](int64_t b, int64_t blocks) {
                const int64_t r = b * groups / parts;
                const LogprobOut o{out.logp + r, out.entropy ? out.entropy + r : nullptr, out.stats ? out.stats + 2 * r : nullptr,
                                   out.top_ids ? out.top_ids + r * top_k : nullptr, out.top_logp ? out.top_logp + r * top_k : nullptr};
                return launch(kPhaseAux, kernel, dim3((unsigned)blocks), dim3(kLpThreads), stream, (const T *)logits + r * stride, vocab,
                              rows - r, stride, ids + r, c, inv_t, top_k, parts, o, sum, most);
            });
        };
        auto join = [&](auto kernel, int threads) {
            return launch(-1, kernel, dim3((unsigned)rows), dim3(threads), stream, (const T *)logits, vocab, stride, ids, c, inv_t, top_k, parts,
                          plan.waves * kWave, out, (const RowSum *)sum, (const float *)most);
        };
        hipError_t e;
        if (plan.waves == 1) e = top_k > 0 ? first(logprob_kernel<T, true, 1>, 8) : first(logprob_kernel<T, false, 1>, 8);
        else e = top_k > 0 ? first(logprob_kernel<T, true, 8>, 1) : first(logprob_kernel<T, false, 8>, 1);
        if (e == hipSuccess && parts > 1)
            e = top_k > 0 ? join(logprob_join_kernel<T, true>, kLpThreads) : join(logprob_join_kernel<T, false>, kWave);
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
        const auto kernel = g_entropy ? logprob_backward_kernel<T, true> : logprob_backward_kernel<T, false>;
        return in_launches(rows * parts, kLpbThreads, [&](int64_t b, int64_t blocks) {      // several only of whole rows
            const int64_t r = b / parts;
            return launch(kPhaseAux, kernel, dim3((unsigned)blocks), dim3(kLpbThreads), stream, (const T *)logits + r * stride, vocab,
                          stride, ids + r, c, inv_t, stats + 2 * r, entropy ? entropy + r : nullptr, g_logp + r,
                          g_entropy ? g_entropy + r : nullptr, (T *)grad + r * grad_stride, grad_stride, parts);
        });
    });
}

}  // namespace pace
