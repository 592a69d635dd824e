// Layer norm and its backward pass for gfx950. For a row x of n elements
//   mu = mean x,  rstd = 1 / sqrt(mean (x - mu)^2 + eps),  h = (x - mu) rstd,  y = h w + b
// and with the gradient dy of y, a = dy w:
//   dx = rstd (a - mean a - h mean(a h)),  dw = sum over rows of dy h,  db = sum over rows of dy.
//
// HBM-bound: the forward pass reads x and writes y, the backward pass reads x
// and dy and writes dx, with some 10 and 16 vector instructions an element. A
// row is held in registers, 16 elements a lane, by 16 lanes up to 256 columns
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
#include "elem.hpp"
#include "kernels.hpp"

#pragma clang fp contract(off)

namespace pace {

namespace {

constexpr int kLnForward = 256;                    // threads of a workgroup, or a row's lanes where these are more
constexpr int kLnBackward = 512;

// Sum over kLanes consecutive lanes (16, 32 or a wave), in every lane.
template <int kLanes>
__device__ __forceinline__ float lanes_sum(float v) {
    auto step = [&](uint32_t got) { v += __builtin_bit_cast(float, got); };
    step(dpp_u32<0xb1, 0xf>(0u, __builtin_bit_cast(uint32_t, v)));       // quads: lane ^ 1, lane ^ 2
    step(dpp_u32<0x4e, 0xf>(0u, __builtin_bit_cast(uint32_t, v)));
    step(dpp_u32<0x141, 0xf>(0u, __builtin_bit_cast(uint32_t, v)));      // mirrored within 8, then within 16
    step(dpp_u32<0x140, 0xf>(0u, __builtin_bit_cast(uint32_t, v)));
    if constexpr (kLanes == 16) return v;
    if constexpr (kLanes == 32) return v + __builtin_bit_cast(float, __builtin_amdgcn_ds_swizzle(__builtin_bit_cast(int, v), 0x401f));
    auto row = [&](int k) { return __builtin_bit_cast(float, readlane_i32(__builtin_bit_cast(int32_t, v), k)); };
    return (row(0) + row(16)) + (row(32) + row(48));
}

// The vectors that a lane holds of a row: lane l has l, l + kLanes, ..
template <typename T>
struct Slice {
    static constexpr int kVec = kVecOf<T>, kVecs = kLnPer / kVec;
    uint4 raw[kVecs];
};
template <typename T, int kLanes>
__device__ __forceinline__ void load_slice(Slice<T> &s, const T *row, int lane, int cols) {
    constexpr int kVec = Slice<T>::kVec;
#pragma unroll
    for (int k = 0; k < Slice<T>::kVecs; ++k) {
        const int c = (lane + k * kLanes) * kVec;
        s.raw[k] = make_uint4(0, 0, 0, 0);
        if (c + kVec <= cols) {
            s.raw[k] = load_a1(row + c);
        } else if (c < cols) {
            float v[kVec];
#pragma unroll
            for (int e = 0; e < kVec; ++e) v[e] = c + e < cols ? to_f32(row[c + e]) : 0.0f;
            s.raw[k] = pack16<T>(v);
        }
    }
}
template <typename T, int kLanes>
__device__ __forceinline__ void store_slice(T *row, const float (&v)[kLnPer], int lane, int cols) {
    constexpr int kVec = Slice<T>::kVec;
#pragma unroll
    for (int k = 0; k < Slice<T>::kVecs; ++k) {
        const int c = (lane + k * kLanes) * kVec;
        float w[kVec];
#pragma unroll
        for (int e = 0; e < kVec; ++e) w[e] = v[k * kVec + e];
        if (c + kVec <= cols) {
            store_a1(row + c, pack16<T>(w));
        } else {
#pragma unroll
            for (int e = 0; e < kVec; ++e)
                if (c + e < cols) row[c + e] = from_f32<T>(w[e]);
        }
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
// A weight's elements in the places of T's vectors; `none` where there is no weight.
template <typename T, typename W, int kLanes>
__device__ __forceinline__ void load_weight(float (&v)[kLnPer], const W *w, float none, int lane, int cols) {
    constexpr int kVec = Slice<T>::kVec;
#pragma unroll
    for (int i = 0; i < kLnPer; ++i) {
        const int c = (lane + i / kVec * kLanes) * kVec + i % kVec;
        v[i] = w && c < cols ? to_f32(w[c]) : none;
    }
}

__device__ __forceinline__ float not_below_zero(float v) { return v < 0.0f ? 0.0f : v; }      // NaN stays

struct Moments {
    float ref, off, m2;      // the mean is ref + off, off small; sum of squares about it
};
// Moments of `count` elements that kLanes lanes (at most a wave) hold; elements at or past cols count as none.
template <typename T, int kLanes, int kStep>
__device__ __forceinline__ Moments lanes_moments(const float (&x)[kLnPer], int lane, int cols, int count) {
    constexpr int kVec = Slice<T>::kVec;
    const float inv = count > 0 ? 1.0f / (float)count : 0.0f;
    float s = 0.0f, s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int i = 0; i < kLnPer; ++i) s += x[i];
    const float ref = lanes_sum<kLanes>(s) * inv;
#pragma unroll
    for (int k = 0; k < Slice<T>::kVecs; ++k) {
        const int left = cols - (lane + k * kStep) * kVec;
        float d[kVec];
#pragma unroll
        for (int e = 0; e < kVec; ++e) d[e] = x[k * kVec + e] - ref;
        if (left < kVec) {
#pragma unroll
            for (int e = 0; e < kVec; ++e) d[e] = e < left ? d[e] : 0.0f;
        }
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
            s1 += d[e];
            s2 = __builtin_fmaf(d[e], d[e], s2);
        }
    }
    s1 = lanes_sum<kLanes>(s1);
    s2 = lanes_sum<kLanes>(s2);
    const float off = s1 * inv;
    return {ref, off, not_below_zero(__builtin_fmaf(-s1, off, s2))};
}

template <typename T, typename W, int kLanes>
__global__ __launch_bounds__(kLanes > kLnForward ? kLanes : kLnForward) void layer_norm_kernel(
    const T *__restrict__ x, int64_t rows, int cols, int64_t stride, const W *__restrict__ weight,
    const W *__restrict__ bias, float eps, T *__restrict__ out, int64_t out_stride, float *__restrict__ stats) {
    constexpr int kThreads = kLanes > kLnForward ? kLanes : kLnForward, kRows = kThreads / kLanes;
    constexpr int kIn = kLanes < kWave ? kLanes : kWave, kWaves = kLanes / kIn;      // lanes of a wave, waves of a row
    constexpr int kVec = Slice<T>::kVec, kVecs = Slice<T>::kVecs;
    __shared__ float slots[2][kRows * kWaves][3];
    const int group = (int)threadIdx.x / kLanes, lane = (int)threadIdx.x % kLanes, wave = lane / kIn;
    auto count_of = [&](int w) {                       // columns that the row's wave w has
        int n = 0;
#pragma unroll
        for (int k = 0; k < kVecs; ++k) {
            const int left = cols - (w * kIn + k * kLanes) * kVec;
            n += left < 0 ? 0 : (left < kIn * kVec ? left : kIn * kVec);
        }
        return n;
    };
    const int count = count_of(wave);
    const float inv = 1.0f / (float)cols;
    const int64_t step = (int64_t)gridDim.x * kRows;
    int64_t base = (int64_t)blockIdx.x * kRows;
    auto row_of = [&](int64_t b) { return b + group < rows ? b + group : rows - 1; };      // loops are the workgroup's
    Slice<T> next;
    load_slice<T, kLanes>(next, x + row_of(base) * stride, lane, cols);
    float w[kLnPer], b[kLnPer];
    load_weight<T, W, kLanes>(w, weight, 1.0f, lane, cols);
    load_weight<T, W, kLanes>(b, bias, 0.0f, lane, cols);
    for (int turn = 0; base < rows; base += step, turn ^= 1) {
        float v[kLnPer];
        unpack_slice<T>(next, v);
        if (base + step < rows) load_slice<T, kLanes>(next, x + row_of(base + step) * stride, lane, cols);
        Moments m = lanes_moments<T, kIn, kLanes>(v, lane, cols, count);
        if constexpr (kWaves > 1) {
            float(*slot)[3] = slots[turn] + group * kWaves;
            if (lane % kIn == 0) {
                slot[wave][0] = m.ref;
                slot[wave][1] = m.off;
                slot[wave][2] = m.m2;
            }
            __syncthreads();                           // the other turn's slots are read before the next barrier
            const float ref = slot[0][0];
            float off = 0.0f, m2 = 0.0f;
#pragma unroll
            for (int k = 0; k < kWaves; ++k) off += (float)count_of(k) * ((slot[k][0] - ref) + slot[k][1]);
            off *= inv;
#pragma unroll
            for (int k = 0; k < kWaves; ++k) {
                const float d = ((slot[k][0] - ref) + slot[k][1]) - off;
                const int n = count_of(k);
                if (n > 0) m2 += slot[k][2] + (float)n * (d * d);
            }
            m = {ref, off, m2};
        }
        const float rstd = 1.0f / sqrtf(m.m2 * inv + eps);
        const int64_t row = base + group;
#pragma unroll
        for (int i = 0; i < kLnPer; ++i) v[i] = __builtin_fmaf(((v[i] - m.ref) - m.off) * rstd, w[i], b[i]);
        if (row < rows) {
            store_slice<T, kLanes>(out + row * out_stride, v, lane, cols);
            if (stats && lane == 0) {
                stats[2 * row] = m.ref + m.off;
                stats[2 * row + 1] = rstd;
            }
        }
    }
}

// Adds this workgroup's column sums of all its rows' lanes and writes them as its part: [2][pitch].
template <typename T, int kLanes, int kThreads>
__device__ __forceinline__ void write_part(const float (&dw)[kLnPer], const float (&db)[kLnPer], float *part, int64_t pitch, int cols) {
    constexpr int kVec = Slice<T>::kVec, kRows = kThreads / kLanes;
    const int lane = (int)threadIdx.x % kLanes;
    auto column = [&](int l, int i) { return (l + i / kVec * kLanes) * kVec + i % kVec; };
    if constexpr (kRows == 1) {
#pragma unroll
        for (int i = 0; i < kLnPer; i += 4) {
            const int c = column(lane, i);
            if (c < cols) {                            // the pitch is a multiple of 4
                *reinterpret_cast<float4 *>(part + c) = make_float4(dw[i], dw[i + 1], dw[i + 2], dw[i + 3]);
                *reinterpret_cast<float4 *>(part + pitch + c) = make_float4(db[i], db[i + 1], db[i + 2], db[i + 3]);
            }
        }
    } else {
        __shared__ float sums[kLnPer][kThreads];
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kLnPer; ++i) sums[i][threadIdx.x] = which ? db[i] : dw[i];
            __syncthreads();
            for (int o = (int)threadIdx.x; o < kLnPer * kLanes; o += kThreads) {
                const int i = o / kLanes, l = o % kLanes, c = column(l, i);
                float s = 0.0f;
#pragma unroll
                for (int r = 0; r < kRows; ++r) s += sums[i][r * kLanes + l];
                if (c < cols) part[which * pitch + c] = s;
            }
        }
    }
}

// dx may be dy itself: a row is read before it is written.
template <typename T, typename W, int kLanes>
__global__ __launch_bounds__(kLanes > kLnBackward ? kLanes : kLnBackward) void layer_norm_backward_kernel(
    const T *__restrict__ x, int64_t rows, int cols, int64_t stride, const W *__restrict__ weight,
    const float *__restrict__ stats, const T *dy, int64_t dy_stride, T *dx, int64_t dx_stride, float *__restrict__ parts,
    int64_t pitch) {
    constexpr int kThreads = kLanes > kLnBackward ? kLanes : kLnBackward, kRows = kThreads / kLanes;
    constexpr int kIn = kLanes < kWave ? kLanes : kWave, kWaves = kLanes / kIn;
    __shared__ float slots[2][kRows * kWaves][2];
    const int group = (int)threadIdx.x / kLanes, lane = (int)threadIdx.x % kLanes, wave = lane / kIn;
    const float inv = 1.0f / (float)cols;
    const int64_t step = (int64_t)gridDim.x * kRows;
    int64_t base = (int64_t)blockIdx.x * kRows;
    auto row_of = [&](int64_t b) { return b + group < rows ? b + group : rows - 1; };
    Slice<T> nx, ng;
    load_slice<T, kLanes>(nx, x + row_of(base) * stride, lane, cols);
    load_slice<T, kLanes>(ng, dy + row_of(base) * dy_stride, lane, cols);
    float mean = stats[2 * row_of(base)], rstd = stats[2 * row_of(base) + 1];
    float w[kLnPer], dw[kLnPer], db[kLnPer];
    load_weight<T, W, kLanes>(w, weight, 1.0f, lane, cols);
#pragma unroll
    for (int i = 0; i < kLnPer; ++i) dw[i] = db[i] = 0.0f;
    for (int turn = 0; base < rows; base += step, turn ^= 1) {
        const int64_t row = base + group;
        float h[kLnPer], a[kLnPer];
        unpack_slice<T>(nx, h);
        unpack_slice<T>(ng, a);
        const float r = rstd;
        const bool live = row < rows;
#pragma unroll
        for (int i = 0; i < kLnPer; ++i) {
            h[i] = (h[i] - mean) * r;
            if (!live) a[i] = 0.0f, h[i] = 0.0f;       // lanes behind the last row add nothing
            dw[i] = __builtin_fmaf(a[i], h[i], dw[i]);
            db[i] += a[i];
            a[i] *= w[i];
        }
        if (base + step < rows) {
            const int64_t to = row_of(base + step);
            load_slice<T, kLanes>(nx, x + to * stride, lane, cols);
            load_slice<T, kLanes>(ng, dy + to * dy_stride, lane, cols);
            mean = stats[2 * to];
            rstd = stats[2 * to + 1];
        }
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < kLnPer; ++i) {
            s1 += a[i];
            s2 = __builtin_fmaf(a[i], h[i], s2);
        }
        s1 = lanes_sum<kIn>(s1);
        s2 = lanes_sum<kIn>(s2);
        if constexpr (kWaves > 1) {
            float(*slot)[2] = slots[turn] + group * kWaves;
            if (lane % kIn == 0) {
                slot[wave][0] = s1;
                slot[wave][1] = s2;
            }
            __syncthreads();
            s1 = s2 = 0.0f;
#pragma unroll
            for (int k = 0; k < kWaves; ++k) {
                s1 += slot[k][0];
                s2 += slot[k][1];
            }
        }
        s1 *= inv;
        s2 *= inv;
#pragma unroll
        for (int i = 0; i < kLnPer; ++i) a[i] = ((a[i] - s1) - h[i] * s2) * r;
        if (live) store_slice<T, kLanes>(dx + row * dx_stride, a, lane, cols);
    }
    if (parts) write_part<T, kLanes, kThreads>(dw, db, parts + (int64_t)blockIdx.x * 2 * pitch, pitch, cols);
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
                                                                        float *__restrict__ parts, int64_t pitch) {
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
    float *part = parts + (int64_t)blockIdx.y * 2 * pitch + c;
#pragma unroll
    for (int e = 0; e < kVec; ++e)
        if (e < n) {
            part[e] = dw[e];
            part[pitch + e] = db[e];
        }
}

// The parts' sums: 64 columns a workgroup, 16 threads a column.
constexpr int kLnJoin = 1024;
__global__ __launch_bounds__(kLnJoin) void layer_norm_join_kernel(const float *__restrict__ parts, int64_t n_parts, int64_t pitch,
                                                                  int64_t cols, float *__restrict__ dw, float *__restrict__ db) {
    constexpr int kSplit = kLnJoin / kWave;
    __shared__ float sums[kSplit][kWave];
    const int64_t c = (int64_t)blockIdx.x * kWave + lane_id();
    const int at = (int)threadIdx.x / kWave;
    float *out = blockIdx.y ? db : dw;
    if (out == nullptr) return;                        // the whole workgroup
    float s = 0.0f;
    if (c < cols) {
        const float *p = parts + (blockIdx.y ? pitch : 0) + c;
#pragma unroll 8
        for (int64_t k = at; k < n_parts; k += kSplit) s += p[k * 2 * pitch];
    }
    sums[at][lane_id()] = s;
    __syncthreads();
    if (at == 0 && c < cols) {
        s = 0.0f;
#pragma unroll
        for (int k = 0; k < kSplit; ++k) s += sums[k][lane_id()];
        out[c] = s;
    }
}

// Runs f with the weight's type: binary32 or that of the rows.
template <typename T, typename F>
hipError_t with_weight(int weight_dtype, F f) {
    if constexpr (sizeof(T) == 4) return f(float{});
    else return weight_dtype == kF32 ? f(float{}) : f(T{});
}
// Runs f with the lanes of a row of up to kLnRegister columns.
template <typename F>
hipError_t with_lanes(int64_t cols, F f) {
    switch (layer_norm_lanes(cols)) {
        case 16: return f(std::integral_constant<int, 16>{});
        case 32: return f(std::integral_constant<int, 32>{});
        case 64: return f(std::integral_constant<int, 64>{});
        case 128: return f(std::integral_constant<int, 128>{});
        case 256: return f(std::integral_constant<int, 256>{});
        case 512: return f(std::integral_constant<int, 512>{});
        default: return f(std::integral_constant<int, 1024>{});
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
            return with_lanes(cols, [&](auto lanes) {
                constexpr int kLanes = decltype(lanes)::value, kThreads = kLanes > kLnForward ? kLanes : kLnForward;
                const int64_t need = (rows + kThreads / kLanes - 1) / (kThreads / kLanes), most = resident_waves() * 2 / (kThreads / kWave);
                return launch(kPhaseAux, layer_norm_kernel<T, W, kLanes>, dim3((unsigned)(need < most ? need : most)), dim3(kThreads), stream,
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
    float *parts = dw || db ? (float *)ws : nullptr;
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
                    if (parts) {
                        const int64_t per = kLnColumns * kVecOf<T>;
                        err = launch(-1, layer_norm_columns_kernel<T>, dim3((unsigned)((cols + per - 1) / per), (unsigned)n_parts),
                                     dim3(kLnColumns), stream, p, rows, cols, stride, stats, g, dy_stride, parts, pitch);
                    }
                    if (err != hipSuccess) return err;
                    return in_launches(rows, kLnWide, [&](int64_t first, int64_t count) {
                        return launch(kPhaseAux, layer_norm_backward_wide_kernel<T, W>, dim3((unsigned)count), dim3(kLnWide), stream,
                                      p + first * stride, cols, stride, w, stats + 2 * first, g + first * dy_stride, dy_stride,
                                      o + first * dx_stride, dx_stride);
                    });
                }
                return with_lanes(cols, [&](auto lanes) {
                    constexpr int kLanes = decltype(lanes)::value, kThreads = kLanes > kLnBackward ? kLanes : kLnBackward;
                    static_assert(kThreads / kLanes == layer_norm_backward_rows(kLanes), "rows of a workgroup");
                    return launch(kPhaseAux, layer_norm_backward_kernel<T, W, kLanes>, dim3((unsigned)n_parts), dim3(kThreads), stream, p,
                                  rows, (int)cols, stride, w, stats, g, dy_stride, o, dx_stride, parts, pitch);
                });
            });
        });
    if (e == hipSuccess && parts)
        e = launch(-1, layer_norm_join_kernel, dim3((unsigned)((cols + kWave - 1) / kWave), 2), dim3(kLnJoin), stream, (const float *)parts,
                   rows > 0 ? n_parts : 0, pitch, cols, dw, db);
    return e;
}

}  // namespace pace
