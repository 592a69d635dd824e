// The norm of all gradients and the AdamW step over many tensors, for gfx950.
// With g = gradient x factor, of each element
//   m' = b1 m + (1 - b1) g,   v' = b2 v + (1 - b2) g^2
//   p' = p (1 - lr decay) - lr / (1 - b1^t) m' / (sqrt(v' / (1 - b2^t)) + eps)
//
// Moments are binary32, or codes of 8 bits with two binary32 scales for every
// 256 consecutive elements of a tensor, M = max |m'| and V = max v':
//   code c in -127 .. 127 stands for c |c| M / 127^2,  c in 0 .. 255 for (c / 255)^4 V,
// so that the square root that the step takes of v is held like m. A moment
// goes to the code that is nearest in that root, a positive v' to 1 at least: no
// step is divided by a zero that rounding made. Codes change at borders, where a
// last place decides, so they go by the largest moment itself, of which the scale is
// the rounding: m', v' and the largest are binary64, and a root of binary32 that
// comes within its own error of a border is decided by comparing in binary64.
//
// HBM-bound: with a binary32 parameter, a bfloat16 gradient and copy 28 bytes an
// element, 16 with moments in 8 bits. A launch takes up to kTable tensors by a
// table in its arguments: workgroups of 4096 elements find their tensor in one
// load and vote of a wave. A wave takes a block of 256 elements, four a lane.
#include "elem.hpp"
#include "kernels.hpp"

#pragma clang fp contract(off)

namespace pace {

namespace {

constexpr int kAdamThreads = 256;
constexpr int kWaveTurns = (int)(kAdamChunk / (kAdamThreads / kWave) / kAdamBlock);      // blocks that a wave takes
constexpr int kPerLane = (int)kAdamBlock / kWave;

// Four elements at any element's alignment, those at or past n as zeros.
template <typename T> struct Four { T e[4]; };
template <typename T, bool kFull>
__device__ __forceinline__ Four<T> load_four_of(const T *p, int64_t i, int64_t n) {
    typedef uint8_t bytes_a1 __attribute__((ext_vector_type(sizeof(T) * 4), aligned(1)));
    if constexpr (kFull) return __builtin_bit_cast(Four<T>, *reinterpret_cast<const bytes_a1 *>(p + i));
    Four<T> v = {};
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (i + e < n) v.e[e] = p[i + e];
    return v;
}
template <typename T, bool kFull>
__device__ __forceinline__ void store_four_of(T *p, int64_t i, int64_t n, const Four<T> &v) {
    typedef uint8_t bytes_a1 __attribute__((ext_vector_type(sizeof(T) * 4), aligned(1)));
    if constexpr (kFull) {
        *reinterpret_cast<bytes_a1 *>(p + i) = __builtin_bit_cast(bytes_a1, v);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (i + e < n) p[i + e] = v.e[e];
    }
}

// ---- the table of a launch ---------------------------------------------------------
// first: the tensor's first workgroup; entries behind the last hold 2^32 - 1.
template <typename E, int kMost>
struct Table {
    E entry[kMost];
    uint32_t first[kMost];
};
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
// Fills tables with the tensors that `take` makes an entry of, `per` elements a workgroup, and hands each
// to `flush` with its number of workgroups: when it is full, or its workgroups are as many as a grid holds.
template <typename E, int kMost, typename Take, typename Flush>
hipError_t by_tables(const Tensors &t, int64_t per, int64_t blocks_most, Take take, Flush flush) {
    Table<E, kMost> table;
    int n = 0;
    int64_t blocks = 0;
    auto out = [&]() {
        for (int k = n; k < kMost; ++k) table.first[k] = UINT32_MAX;
        const hipError_t e = flush(table, blocks);
        n = 0;
        blocks = 0;
        return e;
    };
    for (int64_t i = 0; i < t.n; ++i) {
        if (t.sizes[i] == 0) continue;
        const int64_t need = (t.sizes[i] + per - 1) / per;
        if (!take(i, table.entry[n])) continue;
        if (n > 0 && blocks + need > blocks_most) {
            const E held = table.entry[n];
            const hipError_t e = out();
            if (e != hipSuccess) return e;
            table.entry[0] = held;
        }
        table.first[n++] = (uint32_t)blocks;
        blocks += need;
        if (n == kMost) {
            const hipError_t e = out();
            if (e != hipSuccess) return e;
        }
    }
    return n > 0 ? out() : hipSuccess;
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

template <typename T>
__device__ __forceinline__ double squares(const T *g, int64_t from, int64_t to) {
    constexpr int kVec = kVecOf<T>;
    double s = 0.0;
#pragma unroll 4
    for (int64_t i = from + (int64_t)threadIdx.x * kVec; i < to; i += kNormThreads * kVec) {
        float v[kVec];
        if (i + kVec <= to) {
            unpack16<T>(load_a1(g + i), v);
        } else {
#pragma unroll
            for (int e = 0; e < kVec; ++e) v[e] = i + e < to ? to_f32(g[i + e]) : 0.0f;
        }
#pragma unroll
        for (int e = 0; e < kVec; ++e) s = __builtin_fma((double)v[e], (double)v[e], s);
    }
    return s;
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
#pragma unroll 4
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
    __device__ __forceinline__ float operator()(float p, float m, float v) const {
        return p * keep - size * (m / (sqrtf(v) * unbias + eps));
    }
};

template <typename P, bool kFull>
__device__ __forceinline__ void store_params(const AdamEntry &t, int copy_dtype, int64_t i, const float (&p)[4]) {
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
    Four<P> p;
    Four<G> g;
    Four<float> m, v;
    template <bool kFull>
    __device__ __forceinline__ void load(const AdamEntry &t, int64_t i, int64_t) {
        p = load_four_of<P, kFull>((const P *)t.p, i, t.n);
        g = load_four_of<G, kFull>((const G *)t.g, i, t.n);
        m = load_four_of<float, kFull>((const float *)t.m, i, t.n);
        v = load_four_of<float, kFull>((const float *)t.v, i, t.n);
    }
    template <bool kFull>
    __device__ __forceinline__ void step(const AdamEntry &t, const AdamHyper &h, const AdamStep &s, float factor, int copy_dtype,
                                         int64_t i, int64_t) {
        const float b1 = (float)h.beta1, c1 = (float)(1.0 - h.beta1), b2 = (float)h.beta2, c2 = (float)(1.0 - h.beta2);
        float to[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float d = to_f32(g.e[e]) * factor;
            m.e[e] = __builtin_fmaf(b1, m.e[e], c1 * d);
            v.e[e] = __builtin_fmaf(b2, v.e[e], c2 * d * d);
            to[e] = s(to_f32(p.e[e]), m.e[e], v.e[e]);
        }
        store_params<P, kFull>(t, copy_dtype, i, to);
        store_four_of<float, kFull>((float *)t.m, i, t.n, m);
        store_four_of<float, kFull>((float *)t.v, i, t.n, v);
    }
};

// The code of x >= 0 against a scale, from its root t in binary32: the nearest whole
// number. `reaches(b)`: whether x is at or above what b stands for, in binary64. t is
// within 2^-13 of the root: a rounding of x over the scale, a unit of 2^-23 of each
// square root and a rounding of the product, (1/4 + 2/2 + 2 + 1) 2^-24 x 255 = 6.5e-5 where
// the root is the fourth.
template <typename F>
__device__ __forceinline__ int code_of(float t, F reaches) {
    const float low = __builtin_floorf(t), rest = t - low;
    int c = (int)low + (rest >= 0.5f ? 1 : 0);
    if (__builtin_fabsf(rest - 0.5f) < 0x1p-13f) c = (int)low + (reaches((double)low + 0.5) ? 1 : 0);
    return c;
}

template <typename P, typename G>
struct Adam8 {
    Four<P> p;
    Four<G> g;
    Four<int8_t> mc;
    Four<uint8_t> vc;
    float m_scale, v_scale;
    template <bool kFull>
    __device__ __forceinline__ void load(const AdamEntry &t, int64_t i, int64_t block) {
        p = load_four_of<P, kFull>((const P *)t.p, i, t.n);
        g = load_four_of<G, kFull>((const G *)t.g, i, t.n);
        mc = load_four_of<int8_t, kFull>((const int8_t *)t.m, i, t.n);
        vc = load_four_of<uint8_t, kFull>((const uint8_t *)t.v, i, t.n);
        m_scale = t.scale[2 * block];
        v_scale = t.scale[2 * block + 1];
    }
    template <bool kFull>
    __device__ __forceinline__ void step(const AdamEntry &t, const AdamHyper &h, const AdamStep &s, float factor, int copy_dtype,
                                         int64_t i, int64_t block) {
        const double m_unit = h.beta1 * ((double)m_scale * (1.0 / kRoots2)), v_unit = h.beta2 * ((double)v_scale * (1.0 / kRoots4));
        const double c1 = 1.0 - h.beta1, c2 = 1.0 - h.beta2, f = (double)factor;
        double m[4], v[4];
        float to[4];
        uint64_t m_most = 0, v_most = 0;      // numbers as bits: in order, NaN above infinity
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const double d = (double)to_f32(g.e[e]) * f;
            const int c = mc.e[e], a = c < 0 ? -c : c;
            const uint32_t q = (uint32_t)vc.e[e] * (uint32_t)vc.e[e];
            m[e] = __builtin_fma((double)(c * a), m_unit, c1 * d);
            v[e] = __builtin_fma((double)(q * q), v_unit, c2 * d * d);
            const float m32 = (float)m[e], v32 = (float)v[e];
            to[e] = s(to_f32(p.e[e]), m32, v32);
            const uint64_t mb = __builtin_bit_cast(uint64_t, __builtin_fabs(m[e])), vb = __builtin_bit_cast(uint64_t, __builtin_fabs(v[e]));
            m_most = mb > m_most ? mb : m_most;
            v_most = vb > v_most ? vb : v_most;
        }
        store_params<P, kFull>(t, copy_dtype, i, to);
        // Elements behind the tensor's last are zeros, codes, gradient and all.
        const double m_in = __builtin_bit_cast(double, wave_max_u64(m_most)), v_in = __builtin_bit_cast(double, wave_max_u64(v_most));
        const float m_new = new_scale(m_in), v_new = new_scale(v_in);
        const double m_inv = 1.0 / m_in, v_inv = 1.0 / v_in;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const double x = __builtin_fabs(m[e]);
            int c = 0;
            if (m_new > 0.0f)
                c = code_of(127.0f * __builtin_amdgcn_sqrtf((float)(x * m_inv)), [&](double b) { return x * kRoots2 >= b * b * m_in; });
            mc.e[e] = (int8_t)(m[e] < 0.0 ? -c : c);
            c = 0;
            if (v_new > 0.0f) {
                const double y = v[e];
                c = code_of(255.0f * __builtin_amdgcn_sqrtf(__builtin_amdgcn_sqrtf((float)(y * v_inv))),
                            [&](double b) { return y * kRoots4 >= (b * b) * (b * b) * v_in; });
                c = y > 0.0 && c == 0 ? 1 : c;
            }
            vc.e[e] = (uint8_t)c;
        }
        store_four_of<int8_t, kFull>((int8_t *)t.m, i, t.n, mc);
        store_four_of<uint8_t, kFull>((uint8_t *)t.v, i, t.n, vc);
        if (lane_id() == 0) {
            t.scale[2 * block] = m_new;
            t.scale[2 * block + 1] = v_new;
        }
    }
    static __device__ __forceinline__ float new_scale(double most) {
        const float v = (float)most;
        return v < __builtin_inff() ? (most < (double)kScaleMin ? 0.0f : v) : __builtin_nanf("");
    }
};

template <typename P, typename G, template <typename, typename> class State>
__global__ __launch_bounds__(kAdamThreads) void adamw_kernel(AdamTable table, AdamHyper h, int copy_dtype) {
    float factor = 1.0f;
    if (h.factor) {
        factor = *h.factor;
        if (!(__builtin_fabsf(factor) < __builtin_inff())) return;      // no number: the step is left out
    }
    const int k = tensor_of(table, blockIdx.x);
    const AdamEntry t = table.entry[k];
    const AdamStep s(h, t.decay);
    const int wave = readlane_i32((int)threadIdx.x / kWave, 0);
    const int64_t from = (int64_t)(blockIdx.x - table.first[k]) * kAdamChunk;
    auto first_of = [&](int turn) { return from + (int64_t)(turn * (kAdamThreads / kWave) + wave) * kAdamBlock; };
    const int lane = lane_id() * kPerLane;
    if (from + kAdamChunk <= t.n) {
        State<P, G> state[kWaveTurns];
#pragma unroll
        for (int turn = 0; turn < kWaveTurns; ++turn) state[turn].template load<true>(t, first_of(turn) + lane, first_of(turn) / kAdamBlock);
#pragma unroll
        for (int turn = 0; turn < kWaveTurns; ++turn)
            state[turn].template step<true>(t, h, s, factor, copy_dtype, first_of(turn) + lane, first_of(turn) / kAdamBlock);
    } else {
        for (int turn = 0; turn < kWaveTurns; ++turn) {
            const int64_t at = first_of(turn);
            if (at >= t.n) break;                      // the whole wave
            State<P, G> state;
            state.template load<false>(t, at + lane, at / kAdamBlock);
            state.template step<false>(t, h, s, factor, copy_dtype, at + lane, at / kAdamBlock);
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

__global__ __launch_bounds__(kAdamThreads) void adamw_unpack_kernel(Table<UnpackEntry, kUnpackTable> table) {
    const int k = tensor_of(table, blockIdx.x);
    const UnpackEntry t = table.entry[k];
    const int wave = readlane_i32((int)threadIdx.x / kWave, 0);
    const int64_t from = (int64_t)(blockIdx.x - table.first[k]) * kAdamChunk;
    auto one = [&](auto full, int64_t at) {
        constexpr bool kFull = decltype(full)::value;
        const int64_t i = at + lane_id() * kPerLane, block = at / kAdamBlock;
        const Four<int8_t> mc = load_four_of<int8_t, kFull>(t.m, i, t.n);
        const Four<uint8_t> vc = load_four_of<uint8_t, kFull>(t.v, i, t.n);
        const double m_unit = (double)t.scale[2 * block] * (1.0 / kRoots2), v_unit = (double)t.scale[2 * block + 1] * (1.0 / kRoots4);
        Four<float> m, v;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int c = mc.e[e], a = c < 0 ? -c : c;
            const uint32_t q = (uint32_t)vc.e[e] * (uint32_t)vc.e[e];
            m.e[e] = (float)((double)(c * a) * m_unit);
            v.e[e] = (float)((double)(q * q) * v_unit);
        }
        if (t.m_out) store_four_of<float, kFull>(t.m_out, i, t.n, m);
        if (t.v_out) store_four_of<float, kFull>(t.v_out, i, t.n, v);
    };
    for (int turn = 0; turn < kWaveTurns; ++turn) {
        const int64_t at = from + (int64_t)(turn * (kAdamThreads / kWave) + wave) * kAdamBlock;
        if (at + kAdamBlock <= t.n) one(std::true_type{}, at);
        else if (at < t.n) one(std::false_type{}, at);
    }
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
    const hipError_t e = by_tables<NormEntry, kNormTable>(
        t, chunk, kGridThreads / kNormThreads,
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
    for (int kind = 0; kinds >> kind; ++kind) {
        if (!(kinds >> kind & 1)) continue;
        const int copy = kind % kElemTypes;
        const hipError_t e = by_tables<AdamEntry, kTable>(
            t, kAdamChunk, kAdamBlocksMost,
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
                        return bits == 8 ? launch(kPhaseAux, adamw_kernel<P, G, Adam8>, grid, block, stream, table, h, copy)
                                         : launch(kPhaseAux, adamw_kernel<P, G, Adam32>, grid, block, stream, table, h, copy);
                    });
                });
            });
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_adamw_unpack(const Tensors &t, float *const *m_out, float *const *v_out, hipStream_t stream) {
    return by_tables<UnpackEntry, kUnpackTable>(
        t, kAdamChunk, kAdamBlocksMost,
        [&](int64_t i, UnpackEntry &to) {
            to = {(const int8_t *)t.m[i], (const uint8_t *)t.v[i], t.scales[i], m_out ? m_out[i] : nullptr, v_out ? v_out[i] : nullptr, t.sizes[i]};
            return true;
        },
        [&](const Table<UnpackEntry, kUnpackTable> &table, int64_t blocks) {
            return launch(kPhaseAux, adamw_unpack_kernel, dim3((unsigned)blocks), dim3(kAdamThreads), stream, table);
        });
}

}  // namespace pace
