// Orthogonalised updates for gfx950, by Newton-Schulz steps on the matrix cores.
//
//   X = G / (|G|_F + eps);   steps times:  A = X X^T,  C = a I + b A + c A A,  X <- C X
//
// on the orientation with m <= n rows. Three products a step: A and A A are
// symmetric, so only their lower tiles are formed and both halves written.
// Between products X, A and C are held as binary16, scaled by powers of two:
// the singular values are at most about 1.2, so their range is known, and 11 bits
// lose eight times less than bfloat16 (the result's type) would; the products'
// sums are binary32. X is kept by rows for X X^T and by columns for C X, so that
// every product reads both sides along the summed axis.
#include "elem.hpp"
#include "kernels.hpp"
#include "mfma_tile.hpp"

#pragma clang fp contract(off)

namespace pace {

namespace {

constexpr float kScaleX = 1024.0f;                 // X up to 32 in binary16
constexpr float kScaleA = 256.0f;                  // A and C up to 128
constexpr int kNormThreads = 256;
constexpr int kNormBlocks = 64;                    // partial sums of squares of a matrix, at most
constexpr int kTurn = 64;                          // side of the tiles that are turned

// The m x n orientation of one matrix of the batch and its workspace; the rows'
// ends up to a multiple of 64 elements are zeros, so that products have whole steps.
struct OrthoShape {
    int64_t m, n, mp, np;                          // mp, np: m and n up to 64
    int64_t x, xt, xt2, a, c, bytes;               // byte offsets in a matrix's workspace, and its size
    bool turned;                                   // the update has more rows than columns
};
OrthoShape ortho_shape(int64_t rows, int64_t cols) {
    OrthoShape s;
    s.turned = rows > cols;
    s.m = s.turned ? cols : rows;
    s.n = s.turned ? rows : cols;
    s.mp = (s.m + 63) / 64 * 64;
    s.np = (s.n + 63) / 64 * 64;
    int64_t at = (int64_t)align256(kNormBlocks * sizeof(double));
    auto take = [&](int64_t elems) {
        const int64_t p = at;
        at += (int64_t)align256((size_t)elems * 2);
        return p;
    };
    s.x = take(s.m * s.np);
    s.xt = take(s.n * s.mp);
    s.xt2 = take(s.n * s.mp);
    s.a = take(s.m * s.mp);
    s.c = take(s.m * s.mp);
    s.bytes = at;
    return s;
}
int ortho_norm_blocks(int64_t rows, int64_t cols) {
    const int64_t b = rows * cols / (kNormThreads * 32);
    return (int)(b < 1 ? 1 : (b > kNormBlocks ? kNormBlocks : b));
}

// Sums of squares over every gridDim.x-th row, in binary64: no square of a
// finite binary32 number leaves its range.
template <typename T>
__global__ __launch_bounds__(kNormThreads) void ortho_norm_kernel(const T *__restrict__ g, int64_t rows, int64_t cols,
                                                                  int64_t stride, int64_t batch_stride, char *ws,
                                                                  int64_t ws_stride) {
    constexpr int V = kVecOf<T>;
    __shared__ double part[kNormThreads / kWave];
    const T *mat = g + blockIdx.y * batch_stride;
    const int64_t nv = cols / V;
    double sum = 0.0;
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const T *row = mat + r * stride;
        for (int64_t v = threadIdx.x; v < nv; v += kNormThreads) {
            float z[V];
            unpack16<T>(load_a1(row + v * V), z);
#pragma unroll
            for (int e = 0; e < V; ++e) sum += (double)z[e] * (double)z[e];
        }
        if (nv * V + threadIdx.x < cols) {
            const double x = (double)to_f32(row[nv * V + threadIdx.x]);
            sum += x * x;
        }
    }
#pragma unroll
    for (int off = kWave / 2; off >= 1; off >>= 1) sum += __shfl_xor(sum, off, kWave);
    if (lane_id() == 0) part[threadIdx.x / kWave] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int k = 1; k < kNormThreads / kWave; ++k) sum += part[k];
        reinterpret_cast<double *>(ws + blockIdx.y * ws_stride)[blockIdx.x] = sum;
    }
}

// X by rows and by columns from the update, a 64 x 64 tile a workgroup.
template <typename T>
__global__ __launch_bounds__(256) void ortho_start_kernel(const T *__restrict__ g, int64_t rows, int64_t cols,
                                                          int64_t stride, int64_t batch_stride, int norm_blocks, double eps,
                                                          OrthoShape s, char *ws) {
    __shared__ f16_t tile[kTurn][kTurn + 2];
    char *w = ws + blockIdx.z * s.bytes;
    double sum = 0.0;
    for (int k = 0; k < norm_blocks; ++k) sum += reinterpret_cast<const double *>(w)[k];
    const double inv = (double)kScaleX / (sqrt(sum) + eps);      // binary64: updates of any size
    const T *mat = g + blockIdx.z * batch_stride;
    const int64_t r0 = (int64_t)blockIdx.y * kTurn, c0 = (int64_t)blockIdx.x * kTurn;      // in the update
    const int x = threadIdx.x % kTurn, y0 = threadIdx.x / kTurn;
    for (int y = y0; y < kTurn; y += 256 / kTurn) {
        const bool in = r0 + y < rows && c0 + x < cols;
        tile[y][x] = (f16_t)(float)(in ? (double)to_f32(mat[(r0 + y) * stride + c0 + x]) * inv : 0.0);
    }
    __syncthreads();
    // by the update's rows, and by its columns; the ends of rows are zeros
    f16_t *by_rows = (f16_t *)(w + (s.turned ? s.xt : s.x)), *by_cols = (f16_t *)(w + (s.turned ? s.x : s.xt));
    const int64_t ld_rows = s.turned ? s.mp : s.np, ld_cols = s.turned ? s.np : s.mp;
    for (int y = y0; y < kTurn; y += 256 / kTurn) {
        if (r0 + y < rows && c0 + x < ld_rows) by_rows[(r0 + y) * ld_rows + c0 + x] = tile[y][x];
        if (c0 + y < cols && r0 + x < ld_cols) by_cols[(c0 + y) * ld_cols + r0 + x] = tile[x][y];
    }
}

// The id-th tile of a lower triangle of tiles, row by row.
__device__ __forceinline__ void lower_tile(uint32_t id, int &tm, int &tn) {
    int64_t t = (int64_t)((sqrt((double)(8 * (int64_t)id + 1)) - 1.0) * 0.5);
    while (t * (t + 1) / 2 > id) --t;
    while ((t + 1) * (t + 2) / 2 <= id) ++t;
    tm = __builtin_amdgcn_readfirstlane((int)t);
    tn = __builtin_amdgcn_readfirstlane((int)(id - t * (t + 1) / 2));
}

struct alignas(8) Four {
    f16_t e[4];
};

// Elements (r .. r + 3, c) of a symmetric matrix with zeros up to column mp, to
// both of their places.
__device__ __forceinline__ void store_both(f16_t *to, int64_t m, int64_t mp, int64_t r, int64_t c, const float (&v)[4],
                                           bool mirror) {
    Four w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w.e[e] = (f16_t)(r + e < m ? v[e] : 0.0f);
    if (mirror && c < m && r < mp) *reinterpret_cast<Four *>(to + c * mp + r) = w;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (r + e < m && c < mp) to[(r + e) * mp + c] = c < m ? w.e[e] : (f16_t)0.0f;
}

// A workgroup takes a tile of one matrix of the batch; a matrix's tiles are neighbours.
// kSquare: C = a I + b A + c A A from A, else A = X X^T.
template <bool kSquare, int kB, int kWM, int kWN>
__global__ __launch_bounds__(kWM *kWN *kWave) void ortho_gram_kernel(OrthoShape s, char *ws, uint32_t tiles, float ca,
                                                                     float cb, float cc) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    using P = TileProduct<MulF16, kB, kB, kWM, kWN, true>;
    P t;
    const uint32_t mat = __builtin_amdgcn_readfirstlane((int)(blockIdx.x / tiles));
    char *w = ws + mat * s.bytes;
    int tm, tn;
    lower_tile(blockIdx.x - mat * tiles, tm, tn);
    const int64_t r0 = (int64_t)tm * kB, c0 = (int64_t)tn * kB;
    const Rows x = kSquare ? Rows{w + s.a, s.mp * 2, s.m, s.mp * 2} : Rows{w + s.x, s.np * 2, s.m, s.np * 2};
    t.run(x, r0, x, c0, lds);
    const f16_t *a = (const f16_t *)(w + s.a);
    f16_t *to = (f16_t *)(w + (kSquare ? s.c : s.a));
#pragma unroll
        for (int j = 0; j < P::kTN; ++j) {
            const int64_t col = c0 + P::col(j);
            Four g[P::kTM];
            if (kSquare) {
                // A's elements of this column, by its row of the same number
#pragma unroll
                for (int i = 0; i < P::kTM; ++i) {
                    const int64_t row = r0 + P::row4(i);
                    g[i] = *reinterpret_cast<const Four *>(a + (col < s.m ? col : 0) * s.mp + (row < s.mp ? row : 0));
                }
            }
#pragma unroll
            for (int i = 0; i < P::kTM; ++i) {
                const int64_t row = r0 + P::row4(i);
                float y[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float v = t.acc[i][j][e];
                    if (kSquare)
                        y[e] = __builtin_fmaf(cc / kScaleA, v, cb * (float)g[i].e[e]) + (row + e == col ? ca * kScaleA : 0.0f);
                    else
                        y[e] = v * (kScaleA / (kScaleX * kScaleX));
                }
                store_both(to, s.m, s.mp, row, col, y, r0 != c0);
            }
        }
}

// X <- C X by rows and by columns, or, in the last step, the result.
template <bool kLast, int kB, int kWM, int kWN>
__global__ __launch_bounds__(kWM *kWN *kWave) void ortho_apply_kernel(OrthoShape s, char *ws, int64_t xt_from, int64_t xt_to,
                                                                      uint32_t tiles_m, uint32_t tiles_n,
                                                                      bf16_t *__restrict__ out) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    using P = TileProduct<MulF16, kB, kB, kWM, kWN, true>;
    P t;
    const int mat = __builtin_amdgcn_readfirstlane((int)(blockIdx.x / (tiles_m * tiles_n)));
    int tm, tn;
    tile_of<8>(blockIdx.x - mat * (tiles_m * tiles_n), tiles_m, tiles_n, tm, tn);
    char *w = ws + mat * s.bytes;
    const int64_t r0 = (int64_t)tm * kB, c0 = (int64_t)tn * kB;
    const Rows c{w + s.c, s.mp * 2, s.m, s.mp * 2}, x{w + xt_from, s.mp * 2, s.n, s.mp * 2};
    t.run(c, r0, x, c0, lds);
    f16_t *by_rows = (f16_t *)(w + s.x), *by_cols = (f16_t *)(w + xt_to);
    bf16_t *o = kLast ? out + mat * s.m * s.n : nullptr;
#pragma unroll
        for (int j = 0; j < P::kTN; ++j) {
            const int64_t col = c0 + P::col(j);
#pragma unroll
            for (int i = 0; i < P::kTM; ++i) {
                const int64_t row = r0 + P::row4(i);
                const mfma_v4f v = t.acc[i][j];
                if constexpr (kLast) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (row + e < s.m && col < s.n)
                            o[s.turned ? col * s.m + row + e : (row + e) * s.n + col] = from_f32<bf16_t>(v[e] * (1.0f / (kScaleA * kScaleX)));
                } else {
                    Four y;
#pragma unroll
                    for (int e = 0; e < 4; ++e) y.e[e] = (f16_t)(row + e < s.m ? v[e] * (1.0f / kScaleA) : 0.0f);
                    if (col < s.n && row < s.mp) *reinterpret_cast<Four *>(by_cols + col * s.mp + row) = y;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (row + e < s.m && col < s.np) by_rows[(row + e) * s.np + col] = col < s.n ? y.e[e] : (f16_t)0.0f;
                }
            }
        }
}

// No steps: the normalised update itself.
__global__ __launch_bounds__(256) void ortho_copy_kernel(OrthoShape s, char *ws, bf16_t *__restrict__ out) {
    const f16_t *x = (const f16_t *)(ws + blockIdx.y * s.bytes + (s.turned ? s.xt : s.x));
    const int64_t rows = s.turned ? s.n : s.m, cols = s.turned ? s.m : s.n, ld = s.turned ? s.mp : s.np;
    bf16_t *o = out + blockIdx.y * rows * cols;
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
        for (int64_t c = threadIdx.x; c < cols; c += 256) o[r * cols + c] = from_f32<bf16_t>((float)x[r * ld + c] * (1.0f / kScaleX));
}

template <int kB, int kWM, int kWN>
hipError_t ortho_steps(const OrthoShape &s, char *ws, int64_t batch, int steps, const float *coefs, bf16_t *out,
                       hipStream_t stream) {
    using T = TileProduct<MulF16, kB, kB, kWM, kWN, true>;
    const int64_t tm = (s.m + kB - 1) / kB, tn = (s.n + kB - 1) / kB;
    const int64_t lower = tm * (tm + 1) / 2;
    const dim3 half((unsigned)(lower * batch)), all((unsigned)(tm * tn * batch)), block(T::kThreads);
    int64_t from = s.xt, to = s.xt2;
    hipError_t e = hipSuccess;
    for (int k = 0; k < steps && e == hipSuccess; ++k) {
        e = launch_lds(-1, ortho_gram_kernel<false, kB, kWM, kWN>, half, block, T::kLdsBytes, stream, s, ws, lower, 0.0f, 0.0f, 0.0f);
        if (e == hipSuccess)
            e = launch_lds(-1, ortho_gram_kernel<true, kB, kWM, kWN>, half, block, T::kLdsBytes, stream, s, ws, lower, coefs[0], coefs[1], coefs[2]);
        if (e == hipSuccess)
            e = k + 1 < steps ? launch_lds(kPhaseAux, ortho_apply_kernel<false, kB, kWM, kWN>, all, block, T::kLdsBytes, stream, s, ws,
                                           from, to, tm, tn, out)
                              : launch_lds(kPhaseAux, ortho_apply_kernel<true, kB, kWM, kWN>, all, block, T::kLdsBytes, stream, s, ws,
                                           from, to, tm, tn, out);
        const int64_t x = from;
        from = to;
        to = x;
    }
    return e;
}

}  // namespace

size_t ortho_ws_bytes(int64_t batch, int64_t rows, int64_t cols) { return (size_t)(batch * ortho_shape(rows, cols).bytes) + 256; }

hipError_t launch_orthogonalize(const void *g, int dtype, int64_t batch, int64_t rows, int64_t cols, int64_t stride,
                                int64_t batch_stride, int steps, const double *coefs, double eps, void *out, void *ws,
                                hipStream_t stream) {
    if (batch == 0) return hipSuccess;
    const OrthoShape s = ortho_shape(rows, cols);
    const int blocks = ortho_norm_blocks(rows, cols);
    char *w = (char *)ws;
    hipError_t e = with_elem(dtype, [&](auto tag) {
        using T = decltype(tag);
        hipError_t r = launch(-1, ortho_norm_kernel<T>, dim3((unsigned)blocks, (unsigned)batch), dim3(kNormThreads), stream, (const T *)g, rows,
                              cols, stride, batch_stride, w, s.bytes);
        // the padded ends too: both sides up to a multiple of 64
        if (r == hipSuccess)
            r = launch(-1, ortho_start_kernel<T>, dim3((unsigned)((cols + 63) / 64), (unsigned)((rows + 63) / 64), (unsigned)batch), dim3(256), stream,
                       (const T *)g, rows, cols, stride, batch_stride, blocks, eps, s, w);
        return r;
    });
    if (e != hipSuccess) return e;
    if (steps == 0)
        return launch(-1, ortho_copy_kernel, dim3((unsigned)(rows < 1024 ? rows : 1024), (unsigned)batch), dim3(256), stream, s, w, (bf16_t *)out);
    const float c[3] = {(float)coefs[0], (float)coefs[1], (float)coefs[2]};
    const int64_t big = ((s.m + 255) / 256) * ((s.n + 255) / 256) * batch;
    if (big >= 128) return ortho_steps<256, 2, 4>(s, w, batch, steps, c, (bf16_t *)out, stream);
    return ortho_steps<64, 2, 2>(s, w, batch, steps, c, (bf16_t *)out, stream);
}

}  // namespace pace
