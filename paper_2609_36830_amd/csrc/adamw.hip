// The norm of all gradients and the AdamW step over many tensors, for gfx950.
// With g = gradient x factor, of each element
//   m' = b1 m + (1 - b1) g,   v' = b2 v + (1 - b2) g^2
//   p' = p (1 - lr decay) - lr / (1 - b1^t) m' / (sqrt(v' / (1 - b2^t)) + eps)
//
// Moments are binary32, or codes of 8 bits with two binary32 scales for every
// 256 consecutive elements of a tensor, M = max |m'| and V = max v':
//   code c in -127 .. 127 stands for c |c| M / 127^2,  c in 0 .. 255 for (c / 255)^4 V,
// so that the square root that the step takes of v is held like m. A moment
// goes to the code that is nearest in that root, a positive v' to 1 at least: a
// small v beside large ones is never a zero that rounding made. A block's whole v
// is, where V would be below 2^-126. As long as that goes on (1 - b2) g^2 < 2^-126, so
// the formula's sqrt(v / (1 - b2^t)) stays below 2^-63 / sqrt(1 - b2); an eps of no
// less than 256 times that is demanded, and what is lost changes a step by less than
// half of the way between two codes of v does. Codes change at borders, where a
// last place decides, so they go by the largest moment itself, of which the scale is
// the rounding: m', v' and the largest are binary64, and a root of binary32 that
// comes within its own error of a border is decided by comparing in binary64.
//
// HBM-bound: with a binary32 parameter, a bfloat16 gradient and copy 28 bytes an
// element, 16 with moments in 8 bits. A launch takes up to kTable tensors by a
// table in its arguments: workgroups find their tensor in one
// load and vote of a wave. A wave takes 512 elements at a time, eight a lane in two
// runs of four: two blocks of 256, each by half a wave, so that a block's largest is five
// steps for eight elements of a lane (with a wave a block, six for four, and the library's
// square roots and divisions, the step in 8 bits was bound by its instructions: 787 us for 550).
// 201M elements of that kind take 945 us (6.0 TB/s; a device copy 4.6, an addition in
// place 5.9) and 540 (6.0 TB/s) with moments in 8 bits, their unpacking 354, the
// norm 66 (bfloat16, 6.1 TB/s). Small calls are launches: 96 vectors of 4096 are 2.8 + 1.9
// us for the norm and 3.7 + 3.5 for the step, in two tables.
#include "elem.hpp"
#include "kernels.hpp"

#pragma clang fp contract(off)

namespace pace {

namespace {

constexpr int kAdamThreads = 256;
constexpr int64_t kWaveRun = 2 * kAdamBlock;                     // elements that a wave takes at a time
static_assert(kAdamRound == kAdamThreads / kWave * kWaveRun, "elements of a workgroup at a time");
constexpr int kLaneRuns = 2, kPerRun = 4;                       // of a lane: elements 4 l .. and 128 + 4 l .. of its half's block
// The first element of a lane's run j, in the elements from `at` on.
__device__ __forceinline__ int64_t run_of(int64_t at, int j) {
    return at + (lane_id() / 32) * kAdamBlock + j * (kAdamBlock / kLaneRuns) + lane_id() % 32 * kPerRun;
}

// Four elements at any element's alignment, those at or past n as zeros. A step touches everything once and the next is a
// pass of the model away: non-temporal, so that what the caches hold is not written back for it (201M elements with the
// norm before 1008 us, 1132 without; the norm's own reads stay in the caches for the step).
template <typename T> struct Four { T e[4]; };
template <typename T, bool kFull>
__device__ __forceinline__ Four<T> load_four_of(const T *p, int64_t i, int64_t n) {
    typedef uint8_t bytes_a1 __attribute__((ext_vector_type(sizeof(T) * 4), aligned(1)));
    if constexpr (kFull) return __builtin_bit_cast(Four<T>, __builtin_nontemporal_load(reinterpret_cast<const bytes_a1 *>(p + i)));
    // From the last element where there is none: no branch that would have each load waited for.
    Four<T> v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v.e[e] = p[i + e < n ? i + e : n - 1];
#pragma unroll
    for (int e = 0; e < 4; ++e) v.e[e] = i + e < n ? v.e[e] : T{};
    return v;
}
template <typename T, bool kFull>
__device__ __forceinline__ void store_four_of(T *p, int64_t i, int64_t n, const Four<T> &v) {
    typedef uint8_t bytes_a1 __attribute__((ext_vector_type(sizeof(T) * 4), aligned(1)));
    if (kFull || i + 4 <= n) {
        __builtin_nontemporal_store(__builtin_bit_cast(bytes_a1, v), reinterpret_cast<bytes_a1 *>(p + i));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (i + e < n) p[i + e] = v.e[e];
    }
}

// The tensor that workgroup `b` belongs to: the last whose first is at most b.
template <typename E, int kMost>
__device__ __forceinline__ int tensor_of(const Table<E, kMost> &t, uint32_t b) {
    int k = -1;
#pragma unroll
    for (int from = 0; from < kMost; from += kWave) {
        const int i = from + lane_id();
        k += __popcll(ballot(i < kMost && t.first[i < kMost ? i : 0] <= b));
    }
    return readlane_i32(k, 0);
}
// ---- gradient norm ----------------------------------------------------------------------
struct NormEntry {
    const void *g;
    int64_t n;
    int32_t dtype;
};
constexpr int kNormTable = 128, kNormThreads = 256;

__device__ __forceinline__ double wave_sum_f64(double v) {
    auto step = [&](uint64_t got) { v += __builtin_bit_cast(double, got); };
    step(dpp_u64<0x111, 0xf>(0ull, __builtin_bit_cast(uint64_t, v)));
    step(dpp_u64<0x112, 0xf>(0ull, __builtin_bit_cast(uint64_t, v)));
    step(dpp_u64<0x114, 0xf>(0ull, __builtin_bit_cast(uint64_t, v)));
    step(dpp_u64<0x118, 0xf>(0ull, __builtin_bit_cast(uint64_t, v)));
    step(dpp_u64<0x142, 0xa>(0ull, __builtin_bit_cast(uint64_t, v)));
    step(dpp_u64<0x143, 0xc>(0ull, __builtin_bit_cast(uint64_t, v)));
    return __builtin_bit_cast(double, readlane_i64(__builtin_bit_cast(int64_t, v), kWave - 1));
}

template <int kVec>
__device__ __forceinline__ void add_squares(const float (&v)[kVec], double (&s)[2]) {
#pragma unroll
    for (int e = 0; e < kVec; ++e) s[e % 2] = __builtin_fma((double)v[e], (double)v[e], s[e % 2]);
}
template <typename T>
__device__ __forceinline__ double squares(const T *g, int64_t from, int64_t to) {
    constexpr int kVec = kVecOf<T>, kRound = kNormThreads * kVec, kAtOnce = 4;
    double s[2] = {0.0, 0.0};
    float v[kVec];
    int64_t i = from + (int64_t)threadIdx.x * kVec;
    for (; i + (kAtOnce - 1) * kRound + kVec <= to; i += kAtOnce * kRound) {
        uint4 r[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) r[k] = load_a1(g + i + k * kRound);
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            unpack16<T>(r[k], v);
            add_squares(v, s);
        }
    }
    for (; i < to; i += kRound) {
        if (i + kVec <= to) {
            unpack16<T>(load_a1(g + i), v);
        } else {
#pragma unroll
            for (int e = 0; e < kVec; ++e) v[e] = i + e < to ? to_f32(g[i + e]) : 0.0f;
        }
        add_squares(v, s);
    }
    return s[0] + s[1];
}

__global__ __launch_bounds__(kNormThreads) void grad_norm_kernel(Table<NormEntry, kNormTable> t, int64_t chunk, double *__restrict__ sums) {
    const int k = tensor_of(t, blockIdx.x);
    const NormEntry in = t.entry[k];
    const int64_t from = (int64_t)(blockIdx.x - t.first[k]) * chunk, to = from + chunk < in.n ? from + chunk : in.n;
    double s = in.dtype == kF32 ? squares((const float *)in.g, from, to)
                                : (in.dtype == kBf16 ? squares((const bf16_t *)in.g, from, to) : squares((const f16_t *)in.g, from, to));
    s = wave_sum_f64(s);
    __shared__ double wave[kNormThreads / kWave];
    if (lane_id() == 0) wave[threadIdx.x / kWave] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = 0.0;
#pragma unroll
        for (int w = 0; w < kNormThreads / kWave; ++w) s += wave[w];
        sums[blockIdx.x] = s;
    }
}

constexpr int kNormJoin = 1024;
__global__ __launch_bounds__(kNormJoin) void grad_norm_join_kernel(const double *__restrict__ sums, int64_t n, double max_norm,
                                                                   float *__restrict__ norm_out, float *__restrict__ factor_out) {
    double s = 0.0;
#pragma unroll 8
    for (int64_t i = threadIdx.x; i < n; i += kNormJoin) s += sums[i];
    s = wave_sum_f64(s);
    __shared__ double wave[kNormJoin / kWave];
    if (lane_id() == 0) wave[threadIdx.x / kWave] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = 0.0;
#pragma unroll
        for (int w = 0; w < kNormJoin / kWave; ++w) s += wave[w];
        const double norm = sqrt(s);
        if (norm_out) *norm_out = (float)norm;
        if (factor_out) *factor_out = s < __builtin_inf() ? (norm <= max_norm ? 1.0f : (float)(max_norm / norm)) : __builtin_nanf("");
    }
}

// ---- AdamW ---------------------------------------------------------------------------------
struct AdamEntry {
    void *p;
    const void *g;
    void *m, *v;
    float *scale;
    void *copy;
    int64_t n;
    float decay;
};
constexpr int kTable = 56;           // tables of 3.8 KB: a kernel's arguments are at most 4 KB
typedef Table<AdamEntry, kTable> AdamTable;
constexpr double kRoots2 = 16129.0, kRoots4 = 4228250625.0;      // 127^2, 255^4
constexpr float kScaleMin = 1.17549435e-38f;             // smaller scales (2^-126) count as none

// b^t of a whole t >= 1.
__device__ __forceinline__ double power(double b, double t) {
    uint64_t k = t >= 1.0 ? (uint64_t)(t < 4.6e18 ? t : 4.6e18) : 1;
    double r = 1.0;
    for (; k; k >>= 1, b *= b)
        if (k & 1) r *= b;
    return r;
}

// What all elements of a tensor share.
struct AdamStep {
    float keep, size, unbias, eps;      // p' = p keep - size m' / (sqrt(v') unbias + eps)
    __device__ __forceinline__ AdamStep(const AdamHyper &h, float decay) {
        double lr = h.lr, keep1 = h.keep1, keep2 = h.keep2;
        if (h.schedule) {
            lr = h.schedule[0];
            keep1 = 1.0 - power(h.beta1, h.schedule[1]);
            keep2 = 1.0 - power(h.beta2, h.schedule[1]);
        }
        keep = (float)(1.0 - lr * (double)decay);
        size = (float)(lr / keep1);
        unbias = (float)(1.0 / sqrt(keep2));
        eps = (float)h.eps;
    }
    // root = sqrt(v') and the quotient by the chip's own square root and reciprocal, a unit of 2^-23 each.
    __device__ __forceinline__ float operator()(float p, float m, float root) const {
        const float q = m * __builtin_amdgcn_rcpf(__builtin_fmaf(root, unbias, eps));
        return __builtin_fmaf(-size, q, p * keep);
    }
};

// Square roots of a lane's v, which the chip takes of normal numbers only.
template <int kN>
__device__ __forceinline__ void roots(const float (&v)[kN], float (&root)[kN]) {
    uint32_t least = UINT32_MAX;
#pragma unroll
    for (int e = 0; e < kN; ++e) {
        root[e] = __builtin_amdgcn_sqrtf(v[e]);
        const uint32_t bits = __builtin_bit_cast(uint32_t, v[e]) - 1u;      // 0 comes last
        least = bits < least ? bits : least;
    }
    if (least < 0x7fffffu) {
#pragma unroll
        for (int e = 0; e < kN; ++e) root[e] = sqrtf(v[e]);
    }
}

template <typename P, bool kFull>
__device__ __forceinline__ void store_params(const AdamEntry &t, int copy_dtype, int64_t i, const float *p) {
    Four<P> to;
#pragma unroll
    for (int e = 0; e < 4; ++e) to.e[e] = from_f32<P>(p[e]);
    store_four_of<P, kFull>((P *)t.p, i, t.n, to);
    if (copy_dtype == kBf16) {
        Four<bf16_t> c;
#pragma unroll
        for (int e = 0; e < 4; ++e) c.e[e] = from_f32<bf16_t>(p[e]);
        store_four_of<bf16_t, kFull>((bf16_t *)t.copy, i, t.n, c);
    } else if (copy_dtype == kF16) {
        Four<f16_t> c;
#pragma unroll
        for (int e = 0; e < 4; ++e) c.e[e] = from_f32<f16_t>(p[e]);
        store_four_of<f16_t, kFull>((f16_t *)t.copy, i, t.n, c);
    }
}

template <typename P, typename G>
struct Adam32 {
    Four<P> p[kLaneRuns];
    Four<G> g[kLaneRuns];
    Four<float> m[kLaneRuns], v[kLaneRuns];
    template <bool kFull>
    __device__ __forceinline__ void load(const AdamEntry &t, int64_t at) {
#pragma unroll
        for (int j = 0; j < kLaneRuns; ++j) {
            const int64_t i = run_of(at, j);
            p[j] = load_four_of<P, kFull>((const P *)t.p, i, t.n);
            g[j] = load_four_of<G, kFull>((const G *)t.g, i, t.n);
            m[j] = load_four_of<float, kFull>((const float *)t.m, i, t.n);
            v[j] = load_four_of<float, kFull>((const float *)t.v, i, t.n);
        }
    }
    template <bool kFull>
    __device__ __forceinline__ void step(const AdamEntry &t, const AdamHyper &h, const AdamStep &s, float factor, int copy_dtype, int64_t at) {
        const float b1 = (float)h.beta1, c1 = (float)(1.0 - h.beta1), b2 = (float)h.beta2, c2 = (float)(1.0 - h.beta2);
#pragma unroll
        for (int j = 0; j < kLaneRuns; ++j) {
            const int64_t i = run_of(at, j);
            float to[kPerRun], root[kPerRun];
#pragma unroll
            for (int e = 0; e < kPerRun; ++e) {
                const float d = to_f32(g[j].e[e]) * factor;
                m[j].e[e] = __builtin_fmaf(b1, m[j].e[e], c1 * d);
                v[j].e[e] = __builtin_fmaf(b2, v[j].e[e], c2 * d * d);
            }
            roots(v[j].e, root);
#pragma unroll
            for (int e = 0; e < kPerRun; ++e) to[e] = s(to_f32(p[j].e[e]), m[j].e[e], root[e]);
            store_params<P, kFull>(t, copy_dtype, i, to);
            store_four_of<float, kFull>((float *)t.m, i, t.n, m[j]);
            store_four_of<float, kFull>((float *)t.v, i, t.n, v[j]);
        }
    }
};

// The largest of 32 lanes' numbers (no NaN), in each of them.
__device__ __forceinline__ double half_max_f64(double v) {
    auto step = [&](uint64_t got) {
        const double x = __builtin_bit_cast(double, got);
        v = x > v ? x : v;
    };
    step(dpp_u64<0xb1, 0xf>(0ull, __builtin_bit_cast(uint64_t, v)));
    step(dpp_u64<0x4e, 0xf>(0ull, __builtin_bit_cast(uint64_t, v)));
    step(dpp_u64<0x141, 0xf>(0ull, __builtin_bit_cast(uint64_t, v)));
    step(dpp_u64<0x140, 0xf>(0ull, __builtin_bit_cast(uint64_t, v)));
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_ds_swizzle((int)(uint32_t)b, 0x401f), hi = (uint32_t)__builtin_amdgcn_ds_swizzle((int)(b >> 32), 0x401f);
    step(((uint64_t)hi << 32) | lo);
    return v;
}
// The four bytes of a word as numbers, and four numbers 0 .. 255 as bytes, to the nearest.
__device__ __forceinline__ float byte_of(uint32_t w, int e) { return (float)((w >> (8 * e)) & 0xffu); }
__device__ __forceinline__ uint32_t bytes_from(const float *v) {
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) w = __builtin_amdgcn_cvt_pk_u8_f32(v[e], e, w);
    return w;
}
// Whether x (of a block whose largest is `most`) is at or above what lies halfway between the codes c and c + 1.
__device__ __forceinline__ bool above_m(double x, double c, double most) { return x * kRoots2 >= (c + 0.5) * (c + 0.5) * most; }
__device__ __forceinline__ bool above_v(double x, double c, double most) {
    const double b = (c + 0.5) * (c + 0.5);
    return x * kRoots4 >= b * b * most;
}

template <typename P, typename G>
struct Adam8 {
    Four<P> p[kLaneRuns];
    Four<G> g[kLaneRuns];
    Four<uint8_t> mc[kLaneRuns], vc[kLaneRuns];
    float2 scale;      // M, V
    static __device__ __forceinline__ int64_t block_of(int64_t at) { return at / kAdamBlock + lane_id() / 32; }
    template <bool kFull>
    __device__ __forceinline__ void load(const AdamEntry &t, int64_t at) {
#pragma unroll
        for (int j = 0; j < kLaneRuns; ++j) {
            const int64_t i = run_of(at, j);
            p[j] = load_four_of<P, kFull>((const P *)t.p, i, t.n);
            g[j] = load_four_of<G, kFull>((const G *)t.g, i, t.n);
            mc[j] = load_four_of<uint8_t, kFull>((const uint8_t *)t.m, i, t.n);
            vc[j] = load_four_of<uint8_t, kFull>((const uint8_t *)t.v, i, t.n);
        }
        const int64_t block = block_of(at);
        const int64_t from = kFull || block * kAdamBlock < t.n ? 2 * block : 0;      // behind the last block all are zeros
        scale = make_float2(t.scale[from], t.scale[from + 1]);
    }
    template <bool kFull>
    __device__ __forceinline__ void step(const AdamEntry &t, const AdamHyper &h, const AdamStep &s, float factor, int copy_dtype, int64_t at) {
        const double m_unit = h.beta1 * ((double)scale.x * (1.0 / kRoots2)), v_unit = h.beta2 * ((double)scale.y * (1.0 / kRoots4));
        const double f = (double)factor, c1 = (1.0 - h.beta1) * f, c2 = (1.0 - h.beta2) * f * f;
        constexpr int kN = kLaneRuns * kPerRun;
        double m[kN], v[kN], m_most = 0.0, v_most = 0.0;
        float m32[kN], v32[kN], root[kN];
        uint32_t largest = 0;                          // of v's bits: infinities and NaN are above numbers
        // Elements behind the tensor's last are zeros, codes, gradient and all.
#pragma unroll
        for (int k = 0; k < kN; ++k) {
            const int j = k / kPerRun, e = k % kPerRun;
            const double d = (double)to_f32(g[j].e[e]);
            const float c = byte_of(__builtin_bit_cast(uint32_t, mc[j]) ^ 0x80808080u, e) - 128.0f, q = byte_of(__builtin_bit_cast(uint32_t, vc[j]), e);
            const double qq = (double)(q * q);
            m[k] = __builtin_fma((double)(c * __builtin_fabsf(c)), m_unit, c1 * d);
            v[k] = __builtin_fma(qq * v_unit, qq, c2 * d * d);
            m32[k] = (float)m[k];
            v32[k] = (float)v[k];
            const uint32_t bits = __builtin_bit_cast(uint32_t, v32[k]);
            largest = bits > largest ? bits : largest;
            const double x = __builtin_fabs(m[k]);
            m_most = x > m_most ? x : m_most;
            v_most = v[k] > v_most ? v[k] : v_most;
        }
        roots(v32, root);
#pragma unroll
        for (int j = 0; j < kLaneRuns; ++j) {
            float to[kPerRun];
#pragma unroll
            for (int e = 0; e < kPerRun; ++e) to[e] = s(to_f32(p[j].e[e]), m32[j * kPerRun + e], root[j * kPerRun + e]);
            store_params<P, kFull>(t, copy_dtype, run_of(at, j), to);
        }
        m_most = half_max_f64(m_most);
        v_most = half_max_f64(v_most);
        const uint64_t spoilt = ballot(largest >= 0x7f800000u || !(__builtin_fabsf(scale.x) < __builtin_inff()));
        const bool bad = (uint32_t)(spoilt >> (lane_id() & 32)) != 0;
        const float m_new = new_scale(m_most, bad), v_new = new_scale(v_most, bad);

        // Codes from roots in binary32. 127 sqrt(|m| / M): roundings of m, of M, of 1 / M and of their product, halved, a unit of 2^-23
        // of the root and a rounding of the product with 127, 5 x 2^-24 x 127 = 2^-14.6 in all; 255 sqrt(sqrt(v) / sqrt(V)): the
        // roundings of v and V, halved, a unit of one root and a rounding of the other, of its inverse and of the product, all of
        // that halved, a unit and a rounding, 6 x 2^-24 x 255 = 2^-13.4.
        constexpr float kNearM = 0.5f - 0x1p-14f, kNearV = 0.5f - 0x1p-13f;
        const float m_inv = 1.0f / m_new, v_inv = 1.0f / sqrtf(v_new);
        float cm[kN], cv[kN], far_m = 0.0f, far_v = 0.0f, least = 1.0f;
#pragma unroll
        for (int k = 0; k < kN; ++k) {
            const float tm = 127.0f * __builtin_amdgcn_sqrtf(__builtin_fabsf(m32[k]) * m_inv), tv = 255.0f * __builtin_amdgcn_sqrtf(root[k] * v_inv);
            cm[k] = __builtin_rintf(tm);
            cv[k] = __builtin_rintf(tv);
            far_m = __builtin_fmaxf(far_m, __builtin_fabsf(tm - cm[k]));
            far_v = __builtin_fmaxf(far_v, __builtin_fabsf(tv - cv[k]));
            least = __builtin_fminf(least, cv[k]);
        }
        auto far_out = [](float scale) { return scale > 0.0f && (scale < 0x1p-80f || scale > 0x1p100f); };
        const bool tiny = far_out(m_new) || far_out(v_new);
        if (far_m >= kNearM || far_v >= kNearV || least < 1.0f || tiny) {
#pragma unroll
            for (int k = 0; k < kN; ++k) {
                const double x = __builtin_fabs(m[k]), y = v[k];
                if (tiny) {      // shares that leave binary32's normal numbers
                    cm[k] = (float)__builtin_floor(127.0 * sqrt(x / m_most));
                    cv[k] = (float)__builtin_floor(255.0 * sqrt(sqrt(y / v_most)));
                    cm[k] += above_m(x, cm[k], m_most) ? 1.0f : 0.0f;
                    cv[k] += above_v(y, cv[k], v_most) ? 1.0f : 0.0f;
                } else {
                    const float tm = 127.0f * __builtin_amdgcn_sqrtf(__builtin_fabsf(m32[k]) * m_inv);
                    const float tv = 255.0f * __builtin_amdgcn_sqrtf(root[k] * v_inv);
                    if (__builtin_fabsf(tm - cm[k]) >= kNearM) cm[k] = __builtin_floorf(tm) + (above_m(x, __builtin_floorf(tm), m_most) ? 1.0f : 0.0f);
                    if (__builtin_fabsf(tv - cv[k]) >= kNearV) cv[k] = __builtin_floorf(tv) + (above_v(y, __builtin_floorf(tv), v_most) ? 1.0f : 0.0f);
                }
                cv[k] = y > 0.0 && cv[k] < 1.0f ? 1.0f : cv[k];
            }
        }
#pragma unroll
        for (int k = 0; k < kN; ++k) cm[k] = __builtin_copysignf(cm[k], m32[k]) + 128.0f;
#pragma unroll
        for (int j = 0; j < kLaneRuns; ++j) {
            const int64_t i = run_of(at, j);
            const uint32_t mw = m_new > 0.0f ? bytes_from(cm + j * kPerRun) ^ 0x80808080u : 0u, vw = v_new > 0.0f ? bytes_from(cv + j * kPerRun) : 0u;
            store_four_of<uint8_t, kFull>((uint8_t *)t.m, i, t.n, __builtin_bit_cast(Four<uint8_t>, mw));
            store_four_of<uint8_t, kFull>((uint8_t *)t.v, i, t.n, __builtin_bit_cast(Four<uint8_t>, vw));
        }
        const int64_t block = block_of(at);
        if (lane_id() % 32 == 0 && (kFull || block * kAdamBlock < t.n)) {
            t.scale[2 * block] = m_new;
            t.scale[2 * block + 1] = v_new;
        }
    }
    static __device__ __forceinline__ float new_scale(double most, bool bad) {
        const float v = (float)most;
        return bad || !(v < __builtin_inff()) ? __builtin_nanf("") : (most < (double)kScaleMin ? 0.0f : v);
    }
};

template <typename P, typename G, template <typename, typename> class State>
__global__ __launch_bounds__(kAdamThreads) void adamw_kernel(AdamTable table, AdamHyper h, int copy_dtype, int turns) {
    const float factor = h.factor ? *h.factor : 1.0f;
    const bool skip = !(__builtin_fabsf(factor) < __builtin_inff());      // no number: the step is left out
    const int k = tensor_of(table, blockIdx.x);
    const AdamEntry t = table.entry[k];
    const int wave = readlane_i32((int)threadIdx.x / kWave, 0);
    const int64_t from = (int64_t)(blockIdx.x - table.first[k]) * turns * kAdamRound;
    auto first_of = [&](int turn) { return from + (int64_t)turn * kAdamRound + wave * kWaveRun; };
    // The next run's bytes are on their way while this one is computed. One copy of the code a path: a launch begins with
    // none of it in the caches.
    State<P, G> state;
    if (from + turns * kAdamRound <= t.n) {
        state.template load<true>(t, first_of(0));
        const AdamStep s(h, t.decay);
        if (skip) return;
#pragma unroll 1
        for (int turn = 0; turn < turns; ++turn) {
            State<P, G> next = state;
            if (turn + 1 < turns) next.template load<true>(t, first_of(turn + 1));
            state.template step<true>(t, h, s, factor, copy_dtype, first_of(turn));
            state = next;
        }
    } else {
        const AdamStep s(h, t.decay);
        if (skip) return;
#pragma unroll 1
        for (int turn = 0; turn < turns && first_of(turn) < t.n; ++turn) {
            state.template load<false>(t, first_of(turn));
            state.template step<false>(t, h, s, factor, copy_dtype, first_of(turn));
        }
    }
}

// The values that moments in 8 bits stand for.
struct UnpackEntry {
    const int8_t *m;
    const uint8_t *v;
    const float *scale;
    float *m_out, *v_out;
    int64_t n;
};
constexpr int kUnpackTable = 64;
constexpr int64_t kUnpackChunk = 4096;           // elements of a workgroup

struct Codes {
    Four<uint8_t> m, v;
    float2 scale;
    template <bool kFull>
    __device__ __forceinline__ void load(const UnpackEntry &t, int64_t at) {
        const int64_t i = at + lane_id() * kPerRun, block = (kFull || at < t.n ? at : t.n - 1) / kAdamBlock;
        m = load_four_of<uint8_t, kFull>((const uint8_t *)t.m, i, t.n);
        v = load_four_of<uint8_t, kFull>(t.v, i, t.n);
        scale = make_float2(t.scale[2 * block], t.scale[2 * block + 1]);
    }
    template <bool kFull>
    __device__ __forceinline__ void store(const UnpackEntry &t, int64_t at) const {
        const int64_t i = at + lane_id() * kPerRun;
        const double m_unit = (double)scale.x * (1.0 / kRoots2), v_unit = (double)scale.y * (1.0 / kRoots4);
        Four<float> x, y;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float c = byte_of(__builtin_bit_cast(uint32_t, m) ^ 0x80808080u, e) - 128.0f, q = byte_of(__builtin_bit_cast(uint32_t, v), e);
            const double qq = (double)(q * q);
            x.e[e] = (float)((double)(c * __builtin_fabsf(c)) * m_unit);
            y.e[e] = (float)(qq * v_unit * qq);
        }
        if (t.m_out) store_four_of<float, kFull>(t.m_out, i, t.n, x);
        if (t.v_out) store_four_of<float, kFull>(t.v_out, i, t.n, y);
    }
};

__global__ __launch_bounds__(kAdamThreads) void adamw_unpack_kernel(Table<UnpackEntry, kUnpackTable> table) {
    constexpr int kTurns = (int)(kUnpackChunk / (kAdamThreads / kWave) / kAdamBlock);      // a block a wave
    const int k = tensor_of(table, blockIdx.x);
    const UnpackEntry t = table.entry[k];
    const int wave = readlane_i32((int)threadIdx.x / kWave, 0);
    const int64_t from = (int64_t)(blockIdx.x - table.first[k]) * kUnpackChunk;
    auto first_of = [&](int turn) { return from + (int64_t)(turn * (kAdamThreads / kWave) + wave) * kAdamBlock; };
    auto all = [&](auto full) {      // every load before the first store, also where runs are behind the last element
        constexpr bool kFull = decltype(full)::value;
        Codes c[kTurns];
#pragma unroll
        for (int turn = 0; turn < kTurns; ++turn) c[turn].template load<kFull>(t, first_of(turn));
#pragma unroll
        for (int turn = 0; turn < kTurns; ++turn) c[turn].template store<kFull>(t, first_of(turn));
    };
    if (from + kUnpackChunk <= t.n) all(std::true_type{});
    else all(std::false_type{});
}

constexpr int64_t kAdamBlocksMost = kGridThreads / kAdamThreads;

}  // namespace

size_t grad_norm_ws_bytes(const Tensors &t) {
    int64_t total = 0, slots = 0;
    for (int64_t i = 0; i < t.n; ++i) total += t.sizes[i];
    const int64_t chunk = grad_norm_chunk(total);
    for (int64_t i = 0; i < t.n; ++i) slots += (t.sizes[i] + chunk - 1) / chunk;
    return align256((size_t)slots * sizeof(double)) + 256;
}
size_t grad_norm_ws_most(int64_t n_tensors, int64_t n_elements) {
    return align256((size_t)grad_norm_slots_most(n_tensors, n_elements) * sizeof(double)) + 256;
}

hipError_t launch_grad_norm(const Tensors &t, double max_norm, float *norm, float *factor, void *ws, hipStream_t stream) {
    int64_t total = 0, slots = 0;
    for (int64_t i = 0; i < t.n; ++i) total += t.sizes[i];
    const int64_t chunk = grad_norm_chunk(total);
    double *sums = (double *)ws;
    const hipError_t e = by_tables<hipError_t, NormEntry, kNormTable>(
        t.n, t.sizes, chunk, kGridThreads / kNormThreads,
        [&](int64_t i, NormEntry &to) {
            to = {t.grads[i], t.sizes[i], t.grad_dtypes[i]};
            return true;
        },
        [&](const Table<NormEntry, kNormTable> &table, int64_t blocks) {
            const hipError_t err = launch(kPhaseAux, grad_norm_kernel, dim3((unsigned)blocks), dim3(kNormThreads), stream, table, chunk, sums + slots);
            slots += blocks;
            return err;
        });
    if (e != hipSuccess) return e;
    return launch(-1, grad_norm_join_kernel, dim3(1), dim3(kNormJoin), stream, (const double *)sums, slots, max_norm, norm, factor);
}

hipError_t launch_adamw(const Tensors &t, int bits, const AdamHyper &h, hipStream_t stream) {
    // A launch's tensors have the same types: a pass over the list for each kind that it holds.
    auto copy_of = [&](int64_t i) { return t.copies && t.copies[i] ? t.copy_dtypes[i] : 0; };
    uint64_t kinds = 0;
    auto kind_of = [&](int64_t i) { return (t.param_dtypes[i] * kElemTypes + t.grad_dtypes[i]) * kElemTypes + copy_of(i); };
    for (int64_t i = 0; i < t.n; ++i)
        if (t.sizes[i] > 0) kinds |= (uint64_t)1 << kind_of(i);
    int64_t total = 0;
    for (int64_t i = 0; i < t.n; ++i) total += t.sizes[i];
    const int turns = adamw_turns(total);
    for (int kind = 0; kinds >> kind; ++kind) {
        if (!(kinds >> kind & 1)) continue;
        const int copy = kind % kElemTypes;
        const hipError_t e = by_tables<hipError_t, AdamEntry, kTable>(
            t.n, t.sizes, turns * kAdamRound, kAdamBlocksMost,
            [&](int64_t i, AdamEntry &to) {
                if (kind_of(i) != kind) return false;
                to = {t.params[i], t.grads[i], t.m[i], t.v[i], bits == 8 ? t.scales[i] : nullptr, copy ? t.copies[i] : nullptr, t.sizes[i],
                      t.decay ? t.decay[i] : 0.0f};
                return true;
            },
            [&](const AdamTable &table, int64_t blocks) {
                return with_elem(kind / kElemTypes / kElemTypes, [&](auto p) {
                    return with_elem(kind / kElemTypes % kElemTypes, [&](auto g) {
                        using P = decltype(p);
                        using G = decltype(g);
                        const dim3 grid((unsigned)blocks), block(kAdamThreads);
                        return bits == 8 ? launch(kPhaseAux, adamw_kernel<P, G, Adam8>, grid, block, stream, table, h, copy, turns)
                                         : launch(kPhaseAux, adamw_kernel<P, G, Adam32>, grid, block, stream, table, h, copy, turns);
                    });
                });
            });
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_adamw_unpack(const Tensors &t, float *const *m_out, float *const *v_out, hipStream_t stream) {
    return by_tables<hipError_t, UnpackEntry, kUnpackTable>(
        t.n, t.sizes, kUnpackChunk, kAdamBlocksMost,
        [&](int64_t i, UnpackEntry &to) {
            to = {(const int8_t *)t.m[i], (const uint8_t *)t.v[i], t.scales[i], m_out ? m_out[i] : nullptr, v_out ? v_out[i] : nullptr, t.sizes[i]};
            return true;
        },
        [&](const Table<UnpackEntry, kUnpackTable> &table, int64_t blocks) {
            return launch(kPhaseAux, adamw_unpack_kernel, dim3((unsigned)blocks), dim3(kAdamThreads), stream, table);
        });
}

}  // namespace pace
