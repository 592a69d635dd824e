// Products in 8-bit integers for gfx950, with a scale for each row of both
// sides (tokens and output channels), and the rows' quantisation.
//
//   s = max |x| / 127,  q = rint(x (127 (1 / max |x|)));   out = (sum_k a b) sa sb
//
// The integer sums are exact in 32 bits (k < 131072). They are converted once,
// multiplied by the product of the scales in binary32 and rounded once.
#include "elem.hpp"
#include "kernels.hpp"
#include "mfma_tile.hpp"

#pragma clang fp contract(off)

namespace pace {

namespace {

constexpr int kQuantThreads = 256;

template <typename T>
__global__ __launch_bounds__(kQuantThreads) void quantize_rows_kernel(const T *__restrict__ x, int64_t cols, int64_t stride,
                                                                      int8_t *__restrict__ q, float *__restrict__ scale) {
    constexpr int V = kVecOf<T>;
    __shared__ float part[kQuantThreads / kWave];
    const int64_t row_i = blockIdx.x;
    const T *row = x + row_i * stride;
    int8_t *to = q + row_i * cols;
    const int64_t nv = cols / V;
    // The maximum as bits: |x| is in order, and a NaN is above all numbers.
    uint32_t most = 0;
    auto see = [&](float v) {
        const uint32_t b = __builtin_bit_cast(uint32_t, v) & 0x7fffffffu;
        most = b > most ? b : most;
    };
    for (int64_t v = threadIdx.x; v < nv; v += kQuantThreads) {
        float z[V];
        unpack16<T>(load_a1(row + v * V), z);
#pragma unroll
        for (int e = 0; e < V; ++e) see(z[e]);
    }
    if (nv * V + threadIdx.x < cols) see(to_f32(row[nv * V + threadIdx.x]));
    most = (uint32_t)(wave_max_u64(most));
    if (lane_id() == 0) part[threadIdx.x / kWave] = __builtin_bit_cast(float, most);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kQuantThreads / kWave; ++k) see(part[k]);
    const float amax = __builtin_bit_cast(float, most);
    // A row below 2^-119 would have a scale that is no normal number: it is nothing.
    // One with an infinity or a NaN has a NaN scale and zeros.
    const bool bad = most >= 0x7f800000u, none = bad || amax < 1.5046327690525280e-36f;
    const float inv = none ? 0.0f : 127.0f * (1.0f / amax);
    if (threadIdx.x == 0) scale[row_i] = bad ? __builtin_nanf("") : (none ? 0.0f : amax / 127.0f);
    auto code = [&](float v) { return none ? 0 : (int)__builtin_rintf(v * inv); };
    for (int64_t v = threadIdx.x; v < nv; v += kQuantThreads) {
        float z[V];
        unpack16<T>(load_a1(row + v * V), z);
        struct { int8_t b[V]; } w;
#pragma unroll
        for (int e = 0; e < V; ++e) w.b[e] = (int8_t)code(z[e]);
        __builtin_memcpy(to + v * V, &w, V);
    }
    if (nv * V + threadIdx.x < cols) to[nv * V + threadIdx.x] = (int8_t)code(to_f32(row[nv * V + threadIdx.x]));
}

// Four values in consecutive columns of a row of the output, from column c on.
template <typename O>
__device__ __forceinline__ void store4(O *row, int64_t c, int64_t n, const float (&v)[4]) {
    struct __attribute__((packed)) { O e[4]; } w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w.e[e] = from_f32<O>(v[e]);
    if (c + 4 <= n) {
        *reinterpret_cast<decltype(w) *>(row + c) = w;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < n) row[c + e] = w.e[e];
    }
}

// The channels are the tile's rows, so that a lane holds four consecutive ones
// of a token and stores them together.
template <typename O, int kBN, int kBM, int kWN, int kWM, bool kDirect>
__global__ __launch_bounds__(kWM *kWN *kWave) void matmul_i8_kernel(Rows b, Rows a, const float *__restrict__ sb,
                                                                    const float *__restrict__ sa, O *__restrict__ out,
                                                                    int64_t ldo) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    int64_t tn, tm;
    tile_of<8>(blockIdx.x, (b.rows + kBN - 1) / kBN, (a.rows + kBM - 1) / kBM, tn, tm);
    TileProduct<MulI8, kBN, kBM, kWN, kWM, kDirect> t;
    t.run(b, tn * kBN, a, tm * kBM, lds, 0, a.bytes);
    // All scales first: a lane's channels are 4 kTM, its tokens kTN.
    using P = decltype(t);
    float s[P::kTM][4];
#pragma unroll
    for (int i = 0; i < P::kTM; ++i) {
        const int64_t c = tn * kBN + P::row4(i);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[i][e] = sb[c + e < b.rows ? c + e : b.rows - 1];
    }
#pragma unroll
    for (int j = 0; j < P::kTN; ++j) {
        const int64_t row = tm * kBM + P::col(j);
        if (row >= a.rows) continue;
        const float sr = sa[row];
        O *to = out + row * ldo;
#pragma unroll
        for (int i = 0; i < P::kTM; ++i) {
            const int64_t c = tn * kBN + P::row4(i);
            float y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = (float)t.acc[i][j][e] * (sr * s[i][e]);
            store4(to, c, b.rows, y);
        }
    }
}

}  // namespace

hipError_t launch_quantize_rows(const void *x, int dtype, int64_t rows, int64_t cols, int64_t stride, int8_t *q,
                                float *scale, hipStream_t stream) {
    if (rows == 0) return hipSuccess;
    return with_elem(dtype, [&](auto tag) {
        using T = decltype(tag);
        return launch(kPhaseAux, quantize_rows_kernel<T>, dim3((unsigned)rows), dim3(kQuantThreads), stream, (const T *)x, cols,
                      stride, q, scale);
    });
}

namespace {

template <typename O, int kBN, int kBM, int kWN, int kWM, bool kDirect>
hipError_t launch_tiles(const Rows &b, const Rows &a, const float *sb, const float *sa, void *out, int64_t ldo,
                        hipStream_t stream) {
    using T = TileProduct<MulI8, kBN, kBM, kWN, kWM, kDirect>;
    const int64_t tiles = ((a.rows + kBM - 1) / kBM) * ((b.rows + kBN - 1) / kBN);
    return launch_lds(kPhaseAux, matmul_i8_kernel<O, kBN, kBM, kWN, kWM, kDirect>, dim3((unsigned)tiles), dim3(T::kThreads),
                      T::kLdsBytes, stream, b, a, sb, sa, (O *)out, ldo);
}

}  // namespace

size_t matmul_i8_ws_bytes(int64_t, int64_t, int64_t) { return 256; }

hipError_t launch_matmul_i8(const int8_t *a, int64_t lda, const float *sa, const int8_t *b, int64_t ldb, const float *sb,
                            int64_t m, int64_t n, int64_t k, void *out, int dtype, int64_t ldo, void *, hipStream_t stream) {
    if (m == 0 || n == 0) return hipSuccess;
    const Rows ra{(const char *)a, lda, m, k}, rb{(const char *)b, ldb, n, k};
    // a tile's rows are numbered by 32-bit byte offsets
    const bool direct = (((uintptr_t)a | (uintptr_t)b | (uint64_t)lda | (uint64_t)ldb | (uint64_t)k) & 15) == 0 &&
                        lda < (1 << 23) && ldb < (1 << 23);
    return with_elem(dtype, [&](auto tag) {
        using O = decltype(tag);
        const int64_t big = ((m + 255) / 256) * ((n + 255) / 256);
        if (m > 128 && big >= 128)
            return direct ? launch_tiles<O, 256, 256, 2, 4, true>(rb, ra, sb, sa, out, ldo, stream)
                          : launch_tiles<O, 256, 256, 2, 4, false>(rb, ra, sb, sa, out, ldo, stream);
        return direct ? launch_tiles<O, 64, 64, 2, 2, true>(rb, ra, sb, sa, out, ldo, stream)
                      : launch_tiles<O, 64, 64, 2, 2, false>(rb, ra, sb, sa, out, ldo, stream);
    });
}

}  // namespace pace
