// Layer norm and its backward pass for gfx950. For a row x of n elements
//   mu = mean x,  rstd = 1 / sqrt(mean (x - mu)^2 + eps),  h = (x - mu) rstd,  y = h w + b
// and with the gradient dy of y, a = dy w:
//   dx = rstd (a - mean a - h mean(a h)),  dw = sum over rows of dy h,  db = sum over rows of dy.
//
// HBM-bound: the forward pass reads x and writes y, the backward pass reads x
// and dy and writes dx, with 16 and 25 vector instructions an element. A
// row is held in registers, 16 elements a lane, by 8 lanes up to 128 columns
// and twice as many for twice the columns, up to 1024 lanes for 16384; wider rows are
// read again for each step. The weights stay in registers from row to row.
//
// Each wave takes its mean first, then sums (x - mean) and (x - mean)^2: the
// first sum corrects the mean's own rounding, so that rows far from zero keep
// their variance. Waves are joined by their means and sums of squares about them.
//
// The weights' gradients are sums down the columns: a lane adds its columns over
// the rows that its workgroup takes, in binary32, at most kLnChain of them one
// after the other; the workgroups' sums are added by a second kernel, in their order.
//
// By itself, over three inputs in rotation: 16384 rows of 4096 in bfloat16 take 54 us forward
// (5.0 TB/s; a device copy 4.6 to 5.4) and 80 to 83 backward (4.8 to 5.1, with 5 us of the second
// kernel), 4099 of them 13 and 28, 2047 of 16384 in binary16 27 and 53 (the column sums of 256
// workgroups are 34 MB there, written and read), 131077 of 128 12 and 23. One row of 4096 is 2.7 us on
// the card. Wider rows are not worked on yet: 3300 of 20000 in bfloat16 267 and 350.
// Forward, a lane's reductions and its row's root cost as much as its 16 elements: with the
// library's square root and division, and each sum gathered by four lanes' reads, 20
// instructions an element kept the vector units 77% busy (4099 x 4096 14.8 us for 13.2).
// Rows that end inside a vector are a kernel of their own: with both in one, tests and their
// masks took 24 to 67 scalar registers out of the loop (16384 x 4096 forward 71 us for 54).
#include "elem.hpp"
#include "kernels.hpp"

#pragma clang fp contract(off)

namespace pace {

namespace {

constexpr int kLnForward = 256;                    // threads of a workgroup, or a row's lanes where these are more
constexpr int kLnBackward = 512;

// Sum over kLanes consecutive lanes (8, 16, 32 or a wave), in every lane.
template <int kLanes>
__device__ __forceinline__ float lanes_sum(float v) {
    auto step = [&](uint32_t got) { v += __builtin_bit_cast(float, got); };
    step(dpp_u32<0xb1, 0xf>(0u, __builtin_bit_cast(uint32_t, v)));       // quads: lane ^ 1, lane ^ 2
    step(dpp_u32<0x4e, 0xf>(0u, __builtin_bit_cast(uint32_t, v)));
    step(dpp_u32<0x141, 0xf>(0u, __builtin_bit_cast(uint32_t, v)));      // mirrored within 8, then within 16
    if constexpr (kLanes == 8) return v;
    step(dpp_u32<0x140, 0xf>(0u, __builtin_bit_cast(uint32_t, v)));
    if constexpr (kLanes == 16) return v;
    if constexpr (kLanes == 32) return v + __builtin_bit_cast(float, __builtin_amdgcn_ds_swizzle(__builtin_bit_cast(int, v), 0x401f));
    step(dpp_u32<0x142, 0xa>(0u, __builtin_bit_cast(uint32_t, v)));      // rows of 16 into the next, the first two into the last
    step(dpp_u32<0x143, 0xc>(0u, __builtin_bit_cast(uint32_t, v)));
    return __builtin_bit_cast(float, readlane_i32(__builtin_bit_cast(int32_t, v), kWave - 1));
}

// The row of the workgroup's that a thread has; one for the wave where waves have whole rows.
template <int kLanes>
__device__ __forceinline__ int group_of() {
    const int g = (int)threadIdx.x / kLanes;
    return kLanes >= kWave ? readlane_i32(g, 0) : g;
}

// The vectors that a lane holds of a row: lane l has l, l + kLanes, .. Where a row does not end
// with a vector (kWhole false) its last one is the row's last kVec elements: those that the one
// before has too, below low_of, count as none. So all loads are vectors, with no branch that has
// each waited for (backward, with a tail by elements: 4099 x 2049 in binary32 35.3 us for 26.5, in
// bfloat16 29.2 for 24.1, 30000 x 130 17.1 for 14.3). Only in rows shorter than a vector do the
// elements below low_of lie before the row; they are not read.
template <typename T>
struct Slice {
    static constexpr int kVec = kVecOf<T>, kVecs = kLnPer / kVec;
    uint4 raw[kVecs];
};
template <typename T, int kLanes, bool kWhole>
__device__ __forceinline__ int place_of(int lane, int k, int cols) {      // the column of vector k's first element
    constexpr int kVec = Slice<T>::kVec;
    const int c = (lane + k * kLanes) * kVec;
    return kWhole || c + kVec <= cols ? c : cols - kVec;
}
template <typename T, int kLanes, bool kWhole>
__device__ __forceinline__ int low_of(int lane, int k, int cols) {
    return kWhole ? 0 : (lane + k * kLanes) * Slice<T>::kVec - place_of<T, kLanes, kWhole>(lane, k, cols);
}
// The row's vector that may be short; the same for all lanes.
template <typename T, int kLanes>
__device__ __forceinline__ int last_of(int cols) { return cols / Slice<T>::kVec / kLanes; }
template <typename T>
__device__ __forceinline__ uint4 load_from(const T *p, int from) {      // the elements from `from` on, behind zeros
    float v[kVecOf<T>];
#pragma unroll
    for (int e = 0; e < kVecOf<T>; ++e) v[e] = e >= from ? to_f32(p[e]) : 0.0f;
    return pack16<T>(v);
}
template <typename T, int kLanes, bool kWhole>
__device__ __forceinline__ void load_slice(Slice<T> &s, const T *row, int lane, int cols) {
    constexpr int kVec = Slice<T>::kVec;
#pragma unroll
    for (int k = 0; k < Slice<T>::kVecs; ++k) s.raw[k] = make_uint4(0, 0, 0, 0);
    if (!kWhole && kLanes == layer_norm_lanes(1) && cols < kVec) {
        if (lane == 0) s.raw[0] = load_from(row + (cols - kVec), kVec - cols);
        return;
    }
#pragma unroll
    for (int k = 0; k < Slice<T>::kVecs; ++k)
        if ((lane + k * kLanes) * kVec < cols) s.raw[k] = load_a1(row + place_of<T, kLanes, kWhole>(lane, k, cols));
}
// With kHere the tests of low_of are made here, and not held as masks in 50 scalar registers over the rows: forward 4099 x
// 2049 in binary32 13.6 us for 15.1, 16000 x 4097 in bfloat16 68.3 for 75.5; but backward, whose registers are full, 3000 x
// 10001 60.5 for 54.2.
template <typename T, int kLanes, bool kWhole, bool kHere>
__device__ __forceinline__ void store_slice(T *row, const float (&v)[kLnPer], int lane, int cols) {
    constexpr int kVec = Slice<T>::kVec;
#pragma unroll
    for (int k = 0; k < Slice<T>::kVecs; ++k) {
        const int at = place_of<T, kLanes, kWhole>(lane, k, cols);
        int low = low_of<T, kLanes, kWhole>(lane, k, cols);
        if (!kWhole && kHere) asm volatile("" : "+v"(low));
        if ((lane + k * kLanes) * kVec >= cols) continue;
        float w[kVec];
#pragma unroll
        for (int e = 0; e < kVec; ++e) w[e] = v[k * kVec + e];
        if (low == 0) {
            store_a1(row + at, pack16<T>(w));
        } else {
#pragma unroll
            for (int e = 0; e < kVec; ++e)
                if (e >= low) row[at + e] = from_f32<T>(w[e]);
        }
    }
}
// Zeros in the places of elements that count as none.
template <typename T, int kLanes, bool kWhole, bool kHere>
__device__ __forceinline__ void clear_low(float (&v)[kLnPer], int lane, int cols) {
    constexpr int kVec = Slice<T>::kVec;
#pragma unroll
    for (int k = 0; k < Slice<T>::kVecs; ++k) {
        if (kWhole || k != last_of<T, kLanes>(cols)) continue;
        int low = low_of<T, kLanes, kWhole>(lane, k, cols);
        if (kHere) asm volatile("" : "+v"(low));
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[k * kVec + e] = e >= low ? v[k * kVec + e] : 0.0f;
    }
}
template <typename T>
__device__ __forceinline__ void unpack_slice(const Slice<T> &s, float (&v)[kLnPer]) {
    constexpr int kVec = Slice<T>::kVec;
#pragma unroll
    for (int k = 0; k < Slice<T>::kVecs; ++k) {
        float w[kVec];
        unpack16<T>(s.raw[k], w);
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[k * kVec + e] = w[e];
    }
}
// A weight's elements in the places of T's vectors, in its own type; `none` where there is no weight.
template <typename T, typename W>
struct Weight {
    static constexpr int kVec = Slice<T>::kVec, kIn = kVecOf<W>, kVecs = kLnPer / kIn;
    uint4 raw[kVecs];
    template <int kLanes, bool kWhole>
    __device__ __forceinline__ void load(const W *w, float none, int lane, int cols) {
#pragma unroll
        for (int k = 0; k < kVecs; ++k) {
            const int i = k * kIn, at = place_of<T, kLanes, kWhole>(lane, i / kVec, cols) + i % kVec;
            float v[kIn];
#pragma unroll
            for (int e = 0; e < kIn; ++e) v[e] = none;
            raw[k] = pack16<W>(v);
            if (w == nullptr || (lane + i / kVec * kLanes) * kVec >= cols) continue;
            if (!kWhole && kLanes == layer_norm_lanes(1) && at < 0) raw[k] = load_from(w + at, -at);
            else raw[k] = load_a1(w + at);
        }
    }
    __device__ __forceinline__ void values(float (&v)[kLnPer]) const {
#pragma unroll
        for (int k = 0; k < kVecs; ++k) {
            float u[kIn];
            unpack16<W>(raw[k], u);
#pragma unroll
            for (int e = 0; e < kIn; ++e) v[k * kIn + e] = u[e];
        }
    }
};

__device__ __forceinline__ float not_below_zero(float v) { return v < 0.0f ? 0.0f : v; }      // NaN stays

struct Moments {
    float ref, off, m2;      // the mean is ref + off, off small; sum of squares about it
};
// Moments of `count` elements that kIn lanes (at most a wave) hold of rows of kLanes lanes; elements at or
// past cols count as none. x becomes x - ref.
template <typename T, int kIn, int kLanes, bool kWhole>
__device__ __forceinline__ Moments lanes_moments(float (&x)[kLnPer], int lane, int cols, float count) {
    constexpr int kVec = Slice<T>::kVec;
    const float inv = count > 0.0f ? 1.0f / count : 0.0f;
    float s = 0.0f, s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int i = 0; i < kLnPer; ++i) s += x[i];
    const float ref = lanes_sum<kIn>(s) * inv;
#pragma unroll
    for (int i = 0; i < kLnPer; ++i) x[i] -= ref;
    clear_low<T, kLanes, kWhole, true>(x, lane, cols);
#pragma unroll
    for (int k = 0; k < Slice<T>::kVecs; ++k) {
        const bool any = (lane + k * kLanes) * kVec < cols;
        float t1 = 0.0f, t2 = 0.0f;
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
            const float d = x[k * kVec + e];
            t1 += d;
            t2 = __builtin_fmaf(d, d, t2);
        }
        s1 += any ? t1 : 0.0f;
        s2 += any ? t2 : 0.0f;
    }
    s1 = lanes_sum<kIn>(s1);
    s2 = lanes_sum<kIn>(s2);
    const float off = s1 * inv;
    return {ref, off, not_below_zero(__builtin_fmaf(-s1, off, s2))};
}

template <typename T, typename W, int kLanes, bool kWhole>
__global__ __launch_bounds__(kLanes > kLnForward ? kLanes : kLnForward) void layer_norm_kernel(
    const T *__restrict__ x, int64_t rows, int cols, int64_t stride, const W *__restrict__ weight,
    const W *__restrict__ bias, float eps, T *__restrict__ out, int64_t out_stride, float *__restrict__ stats) {
    constexpr int kThreads = kLanes > kLnForward ? kLanes : kLnForward, kRows = kThreads / kLanes;
    constexpr int kIn = kLanes < kWave ? kLanes : kWave, kWaves = kLanes / kIn;      // lanes of a wave, waves of a row
    constexpr int kVec = Slice<T>::kVec, kVecs = Slice<T>::kVecs;
    __shared__ float4 slots[2][kRows * kWaves];
    const int group = group_of<kLanes>(), lane = (int)threadIdx.x % kLanes, wave = lane / kIn;
    float count = 0.0f;                                // columns that the row's lanes in this wave have
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
        const int left = cols - (wave * kIn + k * kLanes) * kVec;
        count += (float)(left < 0 ? 0 : (left < kIn * kVec ? left : kIn * kVec));
    }
    const float inv = 1.0f / (float)cols;
    const int64_t step = (int64_t)gridDim.x * kRows;
    int64_t base = (int64_t)blockIdx.x * kRows;
    auto row_of = [&](int64_t b) { return b + group < rows ? b + group : rows - 1; };      // loops are the workgroup's
    Slice<T> next;
    load_slice<T, kLanes, kWhole>(next, x + row_of(base) * stride, lane, cols);
    Weight<T, W> weights, biases;
    weights.template load<kLanes, kWhole>(weight, 1.0f, lane, cols);
    biases.template load<kLanes, kWhole>(bias, 0.0f, lane, cols);
    for (int turn = 0; base < rows; base += step, turn ^= 1) {
        float v[kLnPer];
        unpack_slice<T>(next, v);
        clear_low<T, kLanes, kWhole, true>(v, lane, cols);
        if (base + step < rows) load_slice<T, kLanes, kWhole>(next, x + row_of(base + step) * stride, lane, cols);
        Moments m = lanes_moments<T, kIn, kLanes, kWhole>(v, lane, cols, count);
        if constexpr (kWaves > 1) {
            float4 *slot = slots[turn] + group * kWaves;
            if (lane % kIn == 0) slot[wave] = make_float4(m.ref, m.off, m.m2, count);
            __syncthreads();                           // the other turn's slots are read before the next barrier
            // Lane k takes wave k's, in rows of 16 lanes: each wave's comes 16 / kWaves times.
            const float4 part = slot[lane % kWaves];
            constexpr float kShare = (float)kWaves / 16.0f;
            const float ref = __builtin_bit_cast(float, readlane_i32(__builtin_bit_cast(int32_t, part.x), 0));
            const float d = (part.x - ref) + part.y;
            const float off = lanes_sum<16>(part.w * d) * (inv * kShare), e = d - off;
            m.off = (ref - m.ref) + off;               // of the wave's own ref, which v has left behind
            m.m2 = lanes_sum<16>(part.w > 0.0f ? __builtin_fmaf(part.w * e, e, part.z) : 0.0f) * kShare;
        }
        // The chip's inverse root, a unit of 2^-23: its argument is eps at least, a normal number.
        const float rstd = __builtin_amdgcn_rsqf(m.m2 * inv + eps), shift = -m.off * rstd;
        const int64_t row = base + group;
        float w[kLnPer], b[kLnPer];
        weights.values(w);
        biases.values(b);
#pragma unroll
        for (int i = 0; i < kLnPer; ++i) v[i] = __builtin_fmaf(__builtin_fmaf(v[i], rstd, shift), w[i], b[i]);
        if (row < rows) {
            store_slice<T, kLanes, kWhole, true>(out + row * out_stride, v, lane, cols);
            if (stats && lane == 0) {
                stats[2 * row] = m.ref + m.off;
                stats[2 * row + 1] = rstd;
            }
        }
    }
}

// Four consecutive columns' sums, those below `low` left out.
__device__ __forceinline__ void store_sums(float *p, int low, float a, float b, float d, float e) {
    if (low <= 0) {
        store_a1(p, make_uint4(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, d), __builtin_bit_cast(uint32_t, e)));
    } else {
        if (low <= 1) p[1] = b;
        if (low <= 2) p[2] = d;
        if (low <= 3) p[3] = e;
    }
}

// Adds this workgroup's column sums of all its rows' lanes and writes them; dw or db may be null.
template <typename T, int kLanes, bool kWhole, int kThreads>
__device__ __forceinline__ void write_sums(const float (&dw)[kLnPer], const float (&db)[kLnPer], float *dw_out, float *db_out, int cols) {
    constexpr int kVec = Slice<T>::kVec, kRows = kThreads / kLanes;
    int thread = (int)threadIdx.x;
    asm volatile("" : "+v"(thread));                   // places are worked out here, not kept in registers over the rows
    const int lane = thread % kLanes;
    if constexpr (kRows == 1) {
#pragma unroll
        for (int i = 0; i < kLnPer; i += 4) {
            if ((lane + i / kVec * kLanes) * kVec >= cols) continue;
            const int c = place_of<T, kLanes, kWhole>(lane, i / kVec, cols) + i % kVec, low = low_of<T, kLanes, kWhole>(lane, i / kVec, cols) - i % kVec;
            if (dw_out) store_sums(dw_out + c, low, dw[i], dw[i + 1], dw[i + 2], dw[i + 3]);
            if (db_out) store_sums(db_out + c, low, db[i], db[i + 1], db[i + 2], db[i + 3]);
        }
    } else {
        __shared__ float sums[kLnPer][kThreads];
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            float *out = which ? db_out : dw_out;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kLnPer; ++i) sums[i][threadIdx.x] = which ? db[i] : dw[i];
            __syncthreads();
            for (int o = (int)threadIdx.x; o < kLnPer * kLanes; o += kThreads) {
                const int i = o / kLanes, l = o % kLanes, k = i / kVec;
                const int c = place_of<T, kLanes, kWhole>(l, k, cols) + i % kVec;
                const bool mine = (l + k * kLanes) * kVec < cols && i % kVec >= low_of<T, kLanes, kWhole>(l, k, cols);
                float s = 0.0f;
#pragma unroll
                for (int r = 0; r < kRows; ++r) s += sums[i][r * kLanes + l];
                if (out && mine) out[c] = s;
            }
        }
    }
}

// dx may be dy itself: a row is read before it is written. There is one workgroup a CU (kLnParts), so registers for two
// waves a SIMD would do; with 128 the rows of several waves are faster all the same (16384 x 4096 79 us, 82), but those of
// less than a wave spill (131077 x 128 27, 24), and so do ragged ones and binary32 with a row ahead.
template <typename T, typename W, int kLanes, bool kWhole>
__global__ __launch_bounds__(kLanes > kLnBackward ? kLanes : kLnBackward, kLanes > kLnBackward || (kLanes > kWave && kWhole && sizeof(T) == 2) ? 4 : 2) void layer_norm_backward_kernel(
    const T *__restrict__ x, int64_t rows, int cols, int64_t stride, const W *__restrict__ weight,
    const float *__restrict__ stats, const T *dy, int64_t dy_stride, T *dx, int64_t dx_stride, float *__restrict__ dw_out,
    float *__restrict__ db_out, int64_t part_stride) {
    constexpr int kThreads = kLanes > kLnBackward ? kLanes : kLnBackward, kRows = kThreads / kLanes;
    constexpr int kIn = kLanes < kWave ? kLanes : kWave, kWaves = kLanes / kIn;
    __shared__ float2 slots[2][kRows * kWaves];
    const int group = group_of<kLanes>(), lane = (int)threadIdx.x % kLanes, wave = lane / kIn;
    const float inv = 1.0f / (float)cols;
    const int64_t step = (int64_t)gridDim.x * kRows;
    int64_t base = (int64_t)blockIdx.x * kRows;
    auto row_of = [&](int64_t b) { return b + group < rows ? b + group : rows - 1; };
    // A row's bytes are on their way while the one before is summed. Of binary32 a row takes twice the registers, which
    // workgroups of 1024 lanes do not have (1000 x 8192 26.7 us, 28.8 without the row ahead, 4096 x 4096 44.0, 45.7).
    constexpr bool kAhead = sizeof(T) == 2 || kLanes <= kLnBackward;
    Slice<T> nx, ng;
    float mean = 0.0f, rstd = 0.0f;
    auto take = [&](int64_t b) {
        const int64_t r = row_of(b);
        load_slice<T, kLanes, kWhole>(nx, x + r * stride, lane, cols);
        load_slice<T, kLanes, kWhole>(ng, dy + r * dy_stride, lane, cols);
        mean = stats[2 * r];
        rstd = stats[2 * r + 1];
    };
    if (kAhead) take(base);
    Weight<T, W> weights;
    weights.template load<kLanes, kWhole>(weight, 1.0f, lane, cols);
    float dw[kLnPer], db[kLnPer];
#pragma unroll
    for (int i = 0; i < kLnPer; ++i) dw[i] = db[i] = 0.0f;
    for (int turn = 0; base < rows; base += step, turn ^= 1) {
        const int64_t row = base + group;
        if (!kAhead) take(base);
        float h[kLnPer], a[kLnPer], w[kLnPer];
        unpack_slice<T>(nx, h);
        const Slice<T> g = ng;
        unpack_slice<T>(g, a);
        clear_low<T, kLanes, kWhole, false>(a, lane, cols);
        weights.values(w);
        const float r = rstd;
        const bool live = row < rows;
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < kLnPer; ++i) {
            h[i] = (h[i] - mean) * r;
            if (kRows > 1 && !live) a[i] = 0.0f, h[i] = 0.0f;       // lanes behind the last row add nothing
            dw[i] = __builtin_fmaf(a[i], h[i], dw[i]);
            db[i] += a[i];
            a[i] *= w[i];
            s1 += a[i];
            s2 = __builtin_fmaf(a[i], h[i], s2);
        }
        if (kAhead && base + step < rows) take(base + step);
        s1 = lanes_sum<kIn>(s1);
        s2 = lanes_sum<kIn>(s2);
        if constexpr (kWaves > 1) {
            float2 *slot = slots[turn] + group * kWaves;
            if (lane % kIn == 0) slot[wave] = make_float2(s1, s2);
            __syncthreads();
            const float2 part = slot[lane % kWaves];       // in rows of 16 lanes, each wave's 16 / kWaves times
            s1 = lanes_sum<16>(part.x) * ((float)kWaves / 16.0f);
            s2 = lanes_sum<16>(part.y) * ((float)kWaves / 16.0f);
        }
        s1 *= inv;
        s2 *= inv;
        unpack_slice<T>(g, a);                         // half the registers that the products would take from above
#pragma unroll
        for (int i = 0; i < kLnPer; ++i) a[i] = ((a[i] * w[i] - s1) - h[i] * s2) * r;
        if (live) store_slice<T, kLanes, kWhole, false>(dx + row * dx_stride, a, lane, cols);
    }
    if (dw_out || db_out) {
        const int64_t at = (int64_t)blockIdx.x * part_stride;
        write_sums<T, kLanes, kWhole, kThreads>(dw, db, dw_out ? dw_out + at : nullptr, db_out ? db_out + at : nullptr, cols);
    }
}

// ---- rows wider than registers hold -------------------------------------------------
constexpr int kLnWide = 1024;

// Sums of two numbers over the workgroup, in every thread.
__device__ __forceinline__ void block_sums(float &a, float &b, float (*slot)[2]) {
    a = lanes_sum<kWave>(a);
    b = lanes_sum<kWave>(b);
    __syncthreads();
    if (lane_id() == 0) {
        slot[threadIdx.x / kWave][0] = a;
        slot[threadIdx.x / kWave][1] = b;
    }
    __syncthreads();
    a = b = 0.0f;
#pragma unroll
    for (int k = 0; k < kLnWide / kWave; ++k) {
        a += slot[k][0];
        b += slot[k][1];
    }
}

// f(column, its elements as binary32, how many) for the thread's vectors of two rows.
template <typename T, typename F>
__device__ __forceinline__ void each_vector(const T *p, const T *q, int64_t cols, F f) {
    constexpr int kVec = kVecOf<T>;
    for (int64_t c = (int64_t)threadIdx.x * kVec; c < cols; c += kLnWide * kVec) {
        float u[kVec], v[kVec];
        const int n = cols - c < kVec ? (int)(cols - c) : kVec;
        if (n == kVec) {
            unpack16<T>(load_a1(p + c), u);
            unpack16<T>(load_a1(q + c), v);
        } else {
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                u[e] = e < n ? to_f32(p[c + e]) : 0.0f;
                v[e] = e < n ? to_f32(q[c + e]) : 0.0f;
            }
        }
        f(c, u, v, n);
    }
}
template <typename T, int kVec>
__device__ __forceinline__ void store_vector(T *p, const float (&v)[kVec], int n) {
    if (n == kVec) {
        store_a1(p, pack16<T>(v));
    } else {
#pragma unroll
        for (int e = 0; e < kVec; ++e)
            if (e < n) p[e] = from_f32<T>(v[e]);
    }
}

template <typename T, typename W>
__global__ __launch_bounds__(kLnWide) void layer_norm_wide_kernel(const T *__restrict__ x, int64_t cols, int64_t stride,
                                                                  const W *__restrict__ weight, const W *__restrict__ bias,
                                                                  float eps, T *__restrict__ out, int64_t out_stride,
                                                                  float *__restrict__ stats) {
    constexpr int kVec = kVecOf<T>;
    __shared__ float slot[kLnWide / kWave][2];
    const int64_t row = blockIdx.x;
    const T *p = x + row * stride;
    const float inv = 1.0f / (float)cols;
    float s = 0.0f, s1 = 0.0f, s2 = 0.0f;
    each_vector<T>(p, p, cols, [&](int64_t, const float(&u)[kVec], const float(&)[kVec], int) {
        float t = 0.0f;
#pragma unroll
        for (int e = 0; e < kVec; ++e) t += u[e];
        s += t;
    });
    block_sums(s, s1, slot);
    const float ref = s * inv;
    s1 = 0.0f;
    each_vector<T>(p, p, cols, [&](int64_t, const float(&u)[kVec], const float(&)[kVec], int n) {
        float t1 = 0.0f, t2 = 0.0f;
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
            const float d = e < n ? u[e] - ref : 0.0f;
            t1 += d;
            t2 = __builtin_fmaf(d, d, t2);
        }
        s1 += t1;
        s2 += t2;
    });
    block_sums(s1, s2, slot);
    const float off = s1 * inv;
    const float m2 = not_below_zero(__builtin_fmaf(-s1, off, s2));
    const float rstd = 1.0f / sqrtf(m2 * inv + eps);
    T *o = out + row * out_stride;
    each_vector<T>(p, p, cols, [&](int64_t c, const float(&u)[kVec], const float(&)[kVec], int n) {
        float y[kVec];
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
            const float w = weight && e < n ? to_f32(weight[c + e]) : 1.0f, b = bias && e < n ? to_f32(bias[c + e]) : 0.0f;
            y[e] = __builtin_fmaf(((u[e] - ref) - off) * rstd, w, b);
        }
        store_vector<T, kVec>(o + c, y, n);
    });
    if (stats && threadIdx.x == 0) {
        stats[2 * row] = ref + off;
        stats[2 * row + 1] = rstd;
    }
}

template <typename T, typename W>
__global__ __launch_bounds__(kLnWide) void layer_norm_backward_wide_kernel(
    const T *__restrict__ x, int64_t cols, int64_t stride, const W *__restrict__ weight, const float *__restrict__ stats,
    const T *dy, int64_t dy_stride, T *dx, int64_t dx_stride) {
    constexpr int kVec = kVecOf<T>;
    __shared__ float slot[kLnWide / kWave][2];
    const int64_t row = blockIdx.x;
    const T *p = x + row * stride, *q = dy + row * dy_stride;
    const float inv = 1.0f / (float)cols, mean = stats[2 * row], rstd = stats[2 * row + 1];
    float s1 = 0.0f, s2 = 0.0f;
    each_vector<T>(p, q, cols, [&](int64_t c, const float(&u)[kVec], const float(&g)[kVec], int n) {
        float t1 = 0.0f, t2 = 0.0f;
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
            if (e >= n) continue;
            const float a = weight ? g[e] * to_f32(weight[c + e]) : g[e];
            t1 += a;
            t2 = __builtin_fmaf(a, (u[e] - mean) * rstd, t2);
        }
        s1 += t1;
        s2 += t2;
    });
    block_sums(s1, s2, slot);
    s1 *= inv;
    s2 *= inv;
    T *o = dx + row * dx_stride;
    each_vector<T>(p, q, cols, [&](int64_t c, const float(&u)[kVec], const float(&g)[kVec], int n) {
        float v[kVec];
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
            const float a = weight && e < n ? g[e] * to_f32(weight[c + e]) : g[e];
            v[e] = ((a - s1) - (u[e] - mean) * rstd * s2) * rstd;
        }
        store_vector<T, kVec>(o + c, v, n);
    });
}

// Column sums of wide rows, before dy may be overwritten: workgroup (x, y) has kLnColumns vectors of columns and every
// gridDim.y-th row.
constexpr int kLnColumns = 256;
template <typename T>
__global__ __launch_bounds__(kLnColumns) void layer_norm_columns_kernel(const T *__restrict__ x, int64_t rows, int64_t cols,
                                                                        int64_t stride, const float *__restrict__ stats,
                                                                        const T *__restrict__ dy, int64_t dy_stride,
                                                                        float *__restrict__ dw_out, float *__restrict__ db_out,
                                                                        int64_t part_stride) {
    constexpr int kVec = kVecOf<T>;
    const int64_t c = ((int64_t)blockIdx.x * kLnColumns + threadIdx.x) * kVec;
    if (c >= cols) return;
    const int n = cols - c < kVec ? (int)(cols - c) : kVec;
    float dw[kVec], db[kVec];
#pragma unroll
    for (int e = 0; e < kVec; ++e) dw[e] = db[e] = 0.0f;
    for (int64_t r = blockIdx.y; r < rows; r += gridDim.y) {
        const float mean = stats[2 * r], rstd = stats[2 * r + 1];
        const T *p = x + r * stride + c, *q = dy + r * dy_stride + c;
        float u[kVec], g[kVec];
        if (n == kVec) {
            unpack16<T>(load_a1(p), u);
            unpack16<T>(load_a1(q), g);
        } else {
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                u[e] = e < n ? to_f32(p[e]) : 0.0f;
                g[e] = e < n ? to_f32(q[e]) : 0.0f;
            }
        }
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
            dw[e] = __builtin_fmaf(g[e], (u[e] - mean) * rstd, dw[e]);
            db[e] += g[e];
        }
    }
    const int64_t at = (int64_t)blockIdx.y * part_stride + c;
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
        if (dw_out && e < n) dw_out[at + e] = dw[e];
        if (db_out && e < n) db_out[at + e] = db[e];
    }
}

// The parts' sums: 32 columns a workgroup, 32 threads a column.
constexpr int kLnJoin = 1024, kLnJoinCols = 32;
__global__ __launch_bounds__(kLnJoin) void layer_norm_join_kernel(const float *__restrict__ parts, int64_t n_parts, int64_t pitch,
                                                                  int64_t cols, float *__restrict__ dw, float *__restrict__ db) {
    constexpr int kSplit = kLnJoin / kLnJoinCols;
    __shared__ float sums[kSplit][kLnJoinCols + 1];
    const int mine = (int)threadIdx.x % kLnJoinCols, at = (int)threadIdx.x / kLnJoinCols;
    const int64_t c = (int64_t)blockIdx.x * kLnJoinCols + mine;
    float *out = blockIdx.y ? db : dw;
    if (out == nullptr) return;                        // the whole workgroup
    float s = 0.0f;
    if (c < cols) {
        const float *p = parts + (blockIdx.y ? pitch : 0) + c;
#pragma unroll 8
        for (int64_t k = at; k < n_parts; k += kSplit) s += p[k * 2 * pitch];
    }
    sums[at][mine] = s;
    __syncthreads();
    if (at == 0 && c < cols) {
        s = 0.0f;
#pragma unroll
        for (int k = 0; k < kSplit; ++k) s += sums[k][mine];
        out[c] = s;
    }
}

// Runs f with the weight's type: binary32 or that of the rows.
template <typename T, typename F>
hipError_t with_weight(int weight_dtype, F f) {
    if constexpr (sizeof(T) == 4) return f(float{});
    else return weight_dtype == kF32 ? f(float{}) : f(T{});
}
// Runs f with the lanes of a row of up to kLnRegister columns, and whether it ends with a vector.
template <typename T, typename F>
hipError_t with_lanes(int64_t cols, F f) {
    auto whole = [&](auto lanes) {
        return cols % kVecOf<T> == 0 ? f(lanes, std::true_type{}) : f(lanes, std::false_type{});
    };
    switch (layer_norm_lanes(cols)) {
        case 8: return whole(std::integral_constant<int, 8>{});
        case 16: return whole(std::integral_constant<int, 16>{});
        case 32: return whole(std::integral_constant<int, 32>{});
        case 64: return whole(std::integral_constant<int, 64>{});
        case 128: return whole(std::integral_constant<int, 128>{});
        case 256: return whole(std::integral_constant<int, 256>{});
        case 512: return whole(std::integral_constant<int, 512>{});
        default: return whole(std::integral_constant<int, 1024>{});
    }
}

int64_t pitch_of(int64_t cols) { return (cols + 3) / 4 * 4; }

}  // namespace

hipError_t launch_layer_norm(const void *x, int dtype, int64_t rows, int64_t cols, int64_t stride, const void *weight,
                             const void *bias, int weight_dtype, double eps, void *out, int64_t out_stride, float *stats,
                             hipStream_t stream) {
    if (rows == 0) return hipSuccess;
    return with_elem(dtype, [&](auto t) {
        using T = decltype(t);
        return with_weight<T>(weight_dtype, [&](auto u) {
            using W = decltype(u);
            const T *p = (const T *)x;
            const W *w = (const W *)weight, *b = (const W *)bias;
            T *o = (T *)out;
            if (cols > kLnRegister)
                return in_launches(rows, kLnWide, [&](int64_t first, int64_t count) {
                    return launch(kPhaseAux, layer_norm_wide_kernel<T, W>, dim3((unsigned)count), dim3(kLnWide), stream, p + first * stride,
                                  cols, stride, w, b, (float)eps, o + first * out_stride, out_stride, stats ? stats + 2 * first : nullptr);
                });
            return with_lanes<T>(cols, [&](auto lanes, auto whole) {
                constexpr int kLanes = decltype(lanes)::value, kThreads = kLanes > kLnForward ? kLanes : kLnForward;
                const int64_t need = (rows + kThreads / kLanes - 1) / (kThreads / kLanes), most = resident_waves() / (kThreads / kWave);
                return launch(kPhaseAux, layer_norm_kernel<T, W, kLanes, decltype(whole)::value>, dim3((unsigned)(need < most ? need : most)), dim3(kThreads), stream,
                              p, rows, (int)cols, stride, w, b, (float)eps, o, out_stride, stats);
            });
        });
    });
}

size_t layer_norm_backward_ws_bytes(int64_t rows, int64_t cols) {
    return align256((size_t)layer_norm_backward_parts(rows, cols) * 2 * (size_t)pitch_of(cols) * sizeof(float)) + 256;
}
size_t layer_norm_backward_ws_most(int64_t rows, int64_t cols) {
    return align256((size_t)layer_norm_part_floats_most(rows, cols) * sizeof(float)) + 256;
}

hipError_t launch_layer_norm_backward(const void *x, int dtype, int64_t rows, int64_t cols, int64_t stride, const void *weight,
                                      int weight_dtype, const float *stats, const void *dy, int64_t dy_stride, void *dx,
                                      int64_t dx_stride, float *dw, float *db, void *ws, hipStream_t stream) {
    const int64_t n_parts = layer_norm_backward_parts(rows, cols), pitch = pitch_of(cols);
    // Each workgroup's sums go to its part, or, where there is one workgroup, where they are wanted.
    const bool sums = dw || db, parts = sums && n_parts != 1;
    float *part = (float *)ws, *dw_to = parts ? part : dw, *db_to = parts ? part + pitch : db;
    const int64_t part_stride = parts ? 2 * pitch : 0;
    hipError_t e = hipSuccess;
    if (rows > 0)
        e = with_elem(dtype, [&](auto t) {
            using T = decltype(t);
            return with_weight<T>(weight_dtype, [&](auto u) {
                using W = decltype(u);
                const T *p = (const T *)x, *g = (const T *)dy;
                const W *w = (const W *)weight;
                T *o = (T *)dx;
                if (cols > kLnRegister) {
                    hipError_t err = hipSuccess;
                    if (sums) {
                        const int64_t per = kLnColumns * kVecOf<T>;
                        err = launch(-1, layer_norm_columns_kernel<T>, dim3((unsigned)((cols + per - 1) / per), (unsigned)n_parts),
                                     dim3(kLnColumns), stream, p, rows, cols, stride, stats, g, dy_stride, dw_to, db_to, part_stride);
                    }
                    if (err != hipSuccess) return err;
                    return in_launches(rows, kLnWide, [&](int64_t first, int64_t count) {
                        return launch(kPhaseAux, layer_norm_backward_wide_kernel<T, W>, dim3((unsigned)count), dim3(kLnWide), stream,
                                      p + first * stride, cols, stride, w, stats + 2 * first, g + first * dy_stride, dy_stride,
                                      o + first * dx_stride, dx_stride);
                    });
                }
                return with_lanes<T>(cols, [&](auto lanes, auto whole) {
                    constexpr int kLanes = decltype(lanes)::value, kThreads = kLanes > kLnBackward ? kLanes : kLnBackward;
                    static_assert(kThreads / kLanes == layer_norm_backward_rows(kLanes), "rows of a workgroup");
                    const int64_t need = (rows + kThreads / kLanes - 1) / (kThreads / kLanes), blocks = sums || need > kLnAlone ? n_parts : need;
                    return launch(kPhaseAux, layer_norm_backward_kernel<T, W, kLanes, decltype(whole)::value>, dim3((unsigned)blocks), dim3(kThreads), stream, p,
                                  rows, (int)cols, stride, w, stats, g, dy_stride, o, dx_stride, dw_to, db_to, part_stride);
                });
            });
        });
    if (e == hipSuccess && parts)
        e = launch(-1, layer_norm_join_kernel, dim3((unsigned)((cols + kLnJoinCols - 1) / kLnJoinCols), 2), dim3(kLnJoin), stream, (const float *)part,
                   n_parts, pitch, cols, dw, db);
    return e;
}

}  // namespace pace
