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

// The channels are the tile's rows, so that a lane holds four consecutive ones
// of a token. A wave turns its part in LDS and stores each token's channels in
// 16-byte pieces of one run; the scales, which the first bytes' wait covers, lie
// behind.
template <typename O, typename P>
struct I8Tile {
    static constexpr int kChan = P::kRowsW, kTok = P::kColsW;      // of a wave
    static constexpr int kPass = sizeof(O) == 2 ? kTok : (kTok % 32 ? 16 : kTok / 2);      // tokens turned at a time
    static_assert(kTok % kPass == 0 && kPass % 16 == 0, "whole columns of products");
    static constexpr int kRun = kChan * (int)sizeof(O) + 16;       // a token's bytes in LDS: 4 banks on from the last token's
    static constexpr int kTurn = P::kWaves * kPass * kRun;
    static constexpr int kScales = P::kLdsBytes > kTurn ? P::kLdsBytes : kTurn;
    static constexpr int kLds = kScales + (P::kRows + P::kCols) * (int)sizeof(float);
};

template <typename O, typename P>
__global__ __launch_bounds__(P::kThreads) void matmul_i8_kernel(Rows b, Rows a, const float *__restrict__ sb,
                                                                const float *__restrict__ sa, O *__restrict__ out,
                                                                int64_t ldo) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    using T = I8Tile<O, P>;
    constexpr int kBN = P::kRows, kBM = P::kCols;
    int tn, tm;
    tile_of<8>(xcd_run(blockIdx.x, gridDim.x), (uint32_t)((b.rows + kBN - 1) / kBN), (uint32_t)((a.rows + kBM - 1) / kBM), tn, tm);
    const int64_t n0 = (int64_t)tn * kBN, m0 = (int64_t)tm * kBM;
    float *sn = reinterpret_cast<float *>(lds + T::kScales), *sm = sn + kBN;
    for (int v = threadIdx.x; v < kBN + kBM; v += P::kThreads) {
        const bool chan = v < kBN;
        const int64_t at = chan ? n0 + v : m0 + v - kBN, n = chan ? b.rows : a.rows;
        sn[v] = (chan ? sb : sa)[at < n ? at : n - 1];
    }
    P t;
    t.run(b, n0, a, m0, lds);
    __syncthreads();                                 // nobody reads the operands any more
    constexpr int kPer = 16 / (int)sizeof(O);        // channels of a piece
    const int wave = threadIdx.x / kWave, lane = lane_id();
    char *mine = lds + wave * (T::kPass * T::kRun);
    const int c0 = wave / P::kWavesN * T::kChan, r0 = wave % P::kWavesN * T::kTok;
#pragma unroll
    for (int pass = 0; pass < T::kTok / T::kPass; ++pass) {
        constexpr int kJ = T::kPass / 16;
#pragma unroll
        for (int jj = 0; jj < kJ; ++jj) {
            const int j = pass * kJ + jj;
            const float sr = sm[P::col(j)];
#pragma unroll
            for (int i = 0; i < P::kTM; ++i) {
                const float4 s = *reinterpret_cast<const float4 *>(sn + P::row4(i));
                struct __attribute__((packed, aligned(4))) { O e[4]; } y = {{from_f32<O>((float)t.acc[i][j][0] * (sr * s.x)), from_f32<O>((float)t.acc[i][j][1] * (sr * s.y)),
                                                        from_f32<O>((float)t.acc[i][j][2] * (sr * s.z)), from_f32<O>((float)t.acc[i][j][3] * (sr * s.w))}};
                __builtin_memcpy(mine + (P::col(j) - r0 - pass * T::kPass) * T::kRun + (P::row4(i) - c0) * (int)sizeof(O), &y, sizeof(y));
            }
        }
        // Only this wave's part of LDS: no barrier, the wave's own accesses are in order.
        constexpr int kPieces = T::kChan / kPer, kAll = kPieces * T::kPass;      // of a token; of the pass
#pragma unroll
        for (int p = 0; p < kAll; p += kWave) {
            const int at = p + lane;
            if (kAll % kWave != 0 && at >= kAll) break;
            const uint4 v = *reinterpret_cast<const uint4 *>(mine + at / kPieces * T::kRun + at % kPieces * 16);
            const int64_t row = m0 + r0 + pass * T::kPass + at / kPieces, c = n0 + c0 + at % kPieces * kPer;
            if (row >= a.rows) continue;
            O *to = out + row * ldo + c;
            if (c + kPer <= b.rows) {
                store_a1(to, v);
            } else {
                struct { O e[kPer]; } w = __builtin_bit_cast(decltype(w), v);
#pragma unroll
                for (int e = 0; e < kPer; ++e)
                    if (c + e < b.rows) to[e] = w.e[e];
            }
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

template <typename O, typename P>
hipError_t launch_tiles(const Rows &b, const Rows &a, const float *sb, const float *sa, void *out, int64_t ldo,
                        hipStream_t stream) {
    const int64_t tiles = ((a.rows + P::kCols - 1) / P::kCols) * ((b.rows + P::kRows - 1) / P::kRows);
    return launch_lds(kPhaseAux, matmul_i8_kernel<O, P>, dim3((unsigned)tiles), dim3(P::kThreads), I8Tile<O, P>::kLds, stream, b, a, sb, sa,
                      (O *)out, ldo);
}

}  // namespace

size_t matmul_i8_ws_bytes(int64_t, int64_t, int64_t) { return 256; }

hipError_t launch_matmul_i8(const int8_t *a, int64_t lda, const float *sa, const int8_t *b, int64_t ldb, const float *sb,
                            int64_t m, int64_t n, int64_t k, void *out, int dtype, int64_t ldo, void *, hipStream_t stream) {
    if (m == 0 || n == 0) return hipSuccess;
    const Rows ra{(const char *)a, lda, m, k}, rb{(const char *)b, ldb, n, k};
    // a tile's rows are numbered by 32-bit byte offsets
    const bool direct = (((uintptr_t)a | (uintptr_t)b | (uint64_t)lda | (uint64_t)ldb) & 15) == 0 && k % kStepBytes == 0 &&
                        lda < (1 << 23) && ldb < (1 << 23);
    return with_elem(dtype, [&](auto tag) {
        using O = decltype(tag);
        auto tiles = [&](int64_t side) { return ((m + side - 1) / side) * ((n + side - 1) / side); };
        if (direct) {
            const int64_t cus = resident_waves() / 16;
            const int side = product_tile(k / kStepBytes, cus, tiles);
            return with_tile(side, tiles(side), cus, [&](auto shape) {
                return launch_tiles<O, typename decltype(shape)::template Product<MulI8>>(rb, ra, sb, sa, out, ldo, stream);
            });
        }
        // Off alignment the step's bytes pass through registers: 64 while that
        // leaves no CU without a tile.
        if (tiles(128) >= resident_waves() / 16)
            return launch_tiles<O, TileProduct<MulI8, 128, 128, 2, 2, 2, 1, false>>(rb, ra, sb, sa, out, ldo, stream);
        return launch_tiles<O, TileProduct<MulI8, 64, 64, 2, 2, 2, 1, false>>(rb, ra, sb, sa, out, ldo, stream);
    });
}

}  // namespace pace
