// Products in 8-bit integers for gfx950, with a scale for each row of both
// sides (tokens and output channels), and the rows' quantisation.
//
//   s = max |x| / 127,  q = rint(x (127 (1 / max |x|)));   out = (sum_k a b) sa sb
//
// The integer sums are exact in 32 bits (k < 131072). They are converted once,
// multiplied by the product of the scales in binary32 and rounded once.
//
// Many tokens are bound by the matrix cores, in tiles of 256 where there are
// enough: 4096 tokens x 16384 channels x 4096 take 227 us (2.4 PTOP/s; a library's
// large product 2.07), with the quantisation 240. There the cores are busy 66% of
// the time at 1.8 GHz: the tile's LDS reads take as long as its products, and the
// clock falls with the power. 1021 x 150000 x 2048 take 360 (1.7 PTOP/s): 16 steps
// a tile, whose store of 309 MB nothing else covers. Few tokens are bound by the
// weights' bytes: 1 x 16384 x 4096 takes 11.5 us (5.8 TB/s), 64 x 16384 x 4096 12.9. Less
// than a tile a CU is bound by its steps' latency and, in parts, a second launch: 16 x
// 4096 x 8192 take 10 + 4 us, the waves waiting 55% of them. Off the step (see the rule
// below) it is the way through registers: waves wait 56% to 61%, the matrix cores are
// busy 21%.
#include "elem.hpp"
#include "kernels.hpp"
#include "mfma_tile.hpp"

#pragma clang fp contract(off)

namespace pace {

namespace {

// A workgroup a row, read twice (the second time from the cache): 4096 rows of 4096
// bfloat16 take 11.7 us (4.3 TB/s), one row 3, a launch's least.
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

template <typename O, TileWork kWork, typename P>
__global__ __launch_bounds__(P::kThreads) void matmul_i8_kernel(Rows b, Rows a, const float *__restrict__ sb,
                                                                const float *__restrict__ sa, O *__restrict__ out,
                                                                int64_t ldo, char *__restrict__ sums, int parts) {
    static_assert(kWork == kWhole || P::kRows == 64, "no other tile's steps are split");
    extern __shared__ __attribute__((aligned(16))) char lds[];
    using T = I8Tile<O, P>;
    constexpr int kBN = P::kRows, kBM = P::kCols;
    const uint32_t job = xcd_run(blockIdx.x, gridDim.x), id = kWork == kPart ? job / parts : job;
    int tn, tm;
    tile_of<8>(id, (uint32_t)((b.rows + kBN - 1) / kBN), (uint32_t)((a.rows + kBM - 1) / kBM), tn, tm);
    const int64_t n0 = (int64_t)tn * kBN, m0 = (int64_t)tm * kBM;
    P t;
    if constexpr (kWork == kPart) {
        t.run(part_of(b, job - id * parts, parts), n0, part_of(a, job - id * parts, parts), m0, lds);
        t.leave_sums(sums + (int64_t)job * P::kSumBytes);
        return;
    }
    float *sn = reinterpret_cast<float *>(lds + T::kScales), *sm = sn + kBN;
    for (int v = threadIdx.x; v < kBN + kBM; v += P::kThreads) {
        const bool chan = v < kBN;
        const int64_t at = chan ? n0 + v : m0 + v - kBN, n = chan ? b.rows : a.rows;
        sn[v] = (chan ? sb : sa)[at < n ? at : n - 1];
    }
    if constexpr (kWork == kJoin) t.add_sums(sums + (int64_t)id * parts * P::kSumBytes, parts);
    else t.run(b, n0, a, m0, lds);
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

// ---- a few tokens -----------------------------------------------------------------
// The weights are read once and bound the time: no tiles, no LDS on their way. A
// load of a wave is 8 channels by 128 bytes; a lane multiplies its 16 bytes with
// the same bytes of each token, four products an instruction. The waves of a
// workgroup take runs of the summed axis of the same channels.
constexpr int kFewWaves = 4;
constexpr int kFewSteps = 4;                         // steps of 128 bytes on their way together

// 16 bytes from `at` on of a row of `bytes` bytes, zeros behind its end.
__device__ __forceinline__ uint4 load_tail(const char *row, int64_t at, int64_t bytes) {
    if (at + 16 <= bytes) return load_a1(row + at);
    uint32_t w[4] = {0, 0, 0, 0};
    for (int k = 0; k < 16 && at + k < bytes; ++k) w[k >> 2] |= (uint32_t)(uint8_t)row[at + k] << (8 * (k & 3));
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ int dot16(const uint4 &a, const uint4 &b, int c) {
    c = __builtin_amdgcn_sdot4((int)a.x, (int)b.x, c, false);
    c = __builtin_amdgcn_sdot4((int)a.y, (int)b.y, c, false);
    c = __builtin_amdgcn_sdot4((int)a.z, (int)b.z, c, false);
    return __builtin_amdgcn_sdot4((int)a.w, (int)b.w, c, false);
}

// kTok tokens at most, kGroups groups of 8 channels a workgroup.
template <typename O, int kTok, int kGroups>
__global__ __launch_bounds__(kFewWaves *kWave) void matmul_i8_few_kernel(Rows b, Rows a, const float *__restrict__ sb,
                                                                         const float *__restrict__ sa, O *__restrict__ out,
                                                                         int64_t ldo) {
    __shared__ int part[kFewWaves][kGroups * 8][kTok];
    const int wave = threadIdx.x / kWave, lane = lane_id();
    const int64_t n0 = (int64_t)blockIdx.x * (kGroups * 8);
    const int64_t steps = (b.bytes + kStepBytes - 1) / kStepBytes, per = (steps + kFewWaves - 1) / kFewWaves;
    const int64_t k1 = (wave + 1) * per < steps ? (wave + 1) * per : steps;
    const char *rb[kGroups], *ra[kTok];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        const int64_t r = n0 + g * 8 + (lane >> 3);
        rb[g] = b.p + (r < b.rows ? r : b.rows - 1) * b.stride;
    }
#pragma unroll
    for (int t = 0; t < kTok; ++t) ra[t] = a.p + (t < a.rows ? t : a.rows - 1) * a.stride;
    int acc[kGroups][kTok];
#pragma unroll
    for (int g = 0; g < kGroups; ++g)
#pragma unroll
        for (int t = 0; t < kTok; ++t) acc[g][t] = 0;
    const int chunk = (lane & 7) * 16;
    int64_t k = wave * per;
    for (; k + kFewSteps <= k1 && (k + kFewSteps) * kStepBytes <= b.bytes; k += kFewSteps) {
        uint4 w[kFewSteps][kGroups];
#pragma unroll
        for (int s = 0; s < kFewSteps; ++s)
#pragma unroll
            for (int g = 0; g < kGroups; ++g) w[s][g] = load_a1(rb[g] + (k + s) * kStepBytes + chunk);
#pragma unroll
        for (int s = 0; s < kFewSteps; ++s)
#pragma unroll
            for (int t = 0; t < kTok; ++t) {
                const uint4 x = load_a1(ra[t] + (k + s) * kStepBytes + chunk);
#pragma unroll
                for (int g = 0; g < kGroups; ++g) acc[g][t] = dot16(w[s][g], x, acc[g][t]);
            }
    }
    for (; k < k1; ++k) {
        uint4 w[kGroups];
#pragma unroll
        for (int g = 0; g < kGroups; ++g) w[g] = load_tail(rb[g], k * kStepBytes + chunk, b.bytes);
#pragma unroll
        for (int t = 0; t < kTok; ++t) {
            const uint4 x = load_tail(ra[t], k * kStepBytes + chunk, b.bytes);
#pragma unroll
            for (int g = 0; g < kGroups; ++g) acc[g][t] = dot16(w[g], x, acc[g][t]);
        }
    }
#pragma unroll
    for (int g = 0; g < kGroups; ++g)
#pragma unroll
        for (int t = 0; t < kTok; ++t) {
            int v = acc[g][t];                       // over the eight lanes of a channel
            v += (int)dpp_u32<0xb1, 0xf>(0u, (uint32_t)v);
            v += (int)dpp_u32<0x4e, 0xf>(0u, (uint32_t)v);
            v += (int)dpp_u32<0x141, 0xf>(0u, (uint32_t)v);
            if ((lane & 7) == 0) part[wave][g * 8 + (lane >> 3)][t] = v;
        }
    __syncthreads();
    for (int i = threadIdx.x; i < kGroups * 8 * kTok; i += kFewWaves * kWave) {
        const int c = i % (kGroups * 8), t = i / (kGroups * 8);
        if (n0 + c >= b.rows || t >= a.rows) continue;
        int v = 0;
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) v += part[w][c][t];
        out[t * ldo + n0 + c] = from_f32<O>((float)v * (sa[t] * sb[n0 + c]));
    }
}

}  // namespace

hipError_t launch_quantize_rows(const void *x, int dtype, int64_t rows, int64_t cols, int64_t stride, int8_t *q,
                                float *scale, hipStream_t stream) {
    if (rows == 0) return hipSuccess;
    return with_elem(dtype, [&](auto tag) {
        using T = decltype(tag);
        return in_launches(rows, kQuantThreads, [&](int64_t r, int64_t count) {
            return launch(kPhaseAux, quantize_rows_kernel<T>, dim3((unsigned)count), dim3(kQuantThreads), stream, (const T *)x + r * stride, cols,
                          stride, q + r * cols, scale + r);
        });
    });
}

namespace {

// `count` rows of an operand from `first` on, or what is there of them.
Rows rows_from(const Rows &m, int64_t first, int64_t count) {
    return Rows{m.p + first * m.stride, m.stride, m.rows - first < count ? m.rows - first : count, m.bytes};
}

template <typename O, typename P>
hipError_t launch_tiles(const Rows &b, const Rows &a, const float *sb, const float *sa, void *out, int64_t ldo,
                        hipStream_t stream) {
    // Runs of whole columns of tiles, or, of one beyond a launch, of its rows.
    const int64_t tm = (a.rows + P::kCols - 1) / P::kCols, tn = (b.rows + P::kRows - 1) / P::kRows;
    return in_launches(tm, P::kThreads, [&](int64_t i, int64_t ni) {
        const Rows ai = rows_from(a, i * P::kCols, ni * P::kCols);
        return in_launches(tn, P::kThreads * ni, [&](int64_t j, int64_t nj) {
            const Rows bj = rows_from(b, j * P::kRows, nj * P::kRows);
            return launch_lds(kPhaseAux, matmul_i8_kernel<O, kWhole, P>, dim3((unsigned)(ni * nj)), dim3(P::kThreads), I8Tile<O, P>::kLds, stream,
                              bj, ai, sb + j * P::kRows, sa + i * P::kCols, (O *)out + i * P::kCols * ldo + j * P::kRows, ldo, nullptr, 1);
        });
    });
}
// Parts of the steps, then their sums.
template <typename O, typename P>
hipError_t launch_parts(const Rows &b, const Rows &a, const float *sb, const float *sa, void *out, int64_t ldo, int64_t tiles,
                        int parts, char *sums, hipStream_t stream) {
    const hipError_t e = launch_lds(kPhaseAux, matmul_i8_kernel<float, kPart, P>, dim3((unsigned)(tiles * parts)), dim3(P::kThreads), P::kLdsBytes,
                                    stream, b, a, nullptr, nullptr, nullptr, 0, sums, parts);
    if (e != hipSuccess) return e;
    return launch_lds(-1, matmul_i8_kernel<O, kJoin, P>, dim3((unsigned)tiles), dim3(P::kThreads), I8Tile<O, P>::kLds, stream, b, a, sb, sa,
                      (O *)out, ldo, sums, parts);
}

template <typename O, int kTok>
hipError_t launch_few(const Rows &b, const Rows &a, const float *sb, const float *sa, void *out, int64_t ldo,
                      hipStream_t stream) {
    // as many channels a workgroup as leave a workgroup for every CU
    const int64_t cus = resident_waves() / 16;
    auto go = [&](auto kernel, int64_t channels) {
        return in_launches((b.rows + channels - 1) / channels, kFewWaves * kWave, [&](int64_t g, int64_t groups) {
            const int64_t n = g * channels;
            return launch(kPhaseAux, kernel, dim3((unsigned)groups), dim3(kFewWaves * kWave), stream, rows_from(b, n, groups * channels), a, sb + n,
                          sa, (O *)out + n, ldo);
        });
    };
    if (b.rows >= 32 * cus) return go(matmul_i8_few_kernel<O, kTok, 4>, 32);
    if (b.rows >= 16 * cus) return go(matmul_i8_few_kernel<O, kTok, 2>, 16);
    return go(matmul_i8_few_kernel<O, kTok, 1>, 8);
}

}  // namespace

// Rows of whole steps and 16-byte chunks go straight into LDS; a tile's are numbered by
// 32-bit byte offsets.
static bool i8_direct(const int8_t *a, int64_t lda, const int8_t *b, int64_t ldb, int64_t k) {
    return (((uintptr_t)a | (uintptr_t)b | (uint64_t)lda | (uint64_t)ldb) & 15) == 0 && k % kStepBytes == 0 && lda < (1 << 23) && ldb < (1 << 23);
}
static size_t i8_ws_of(int64_t jobs) { return jobs ? (size_t)jobs * 64 * 64 * sizeof(int32_t) : 256; }
size_t matmul_i8_ws_bytes(const int8_t *a, int64_t lda, const int8_t *b, int64_t ldb, int64_t m, int64_t n, int64_t k) {
    if (m <= 4 || k < kI8PartSteps * kStepBytes) return i8_ws_of(0);      // most calls, without asking for the device
    const int parts = i8_parts(m, n, k, i8_direct(a, lda, b, ldb, k), resident_waves() / 16);
    return i8_ws_of(parts == 1 ? 0 : ((m + 63) / 64) * ((n + 63) / 64) * parts);
}
size_t matmul_i8_ws_most(int64_t m, int64_t n, int64_t k) { return i8_ws_of(i8_jobs_most(m, n, k, resident_waves() / 16)); }

hipError_t launch_matmul_i8(const int8_t *a, int64_t lda, const float *sa, const int8_t *b, int64_t ldb, const float *sb,
                            int64_t m, int64_t n, int64_t k, void *out, int dtype, int64_t ldo, void *ws, hipStream_t stream) {
    if (m == 0 || n == 0) return hipSuccess;
    const Rows ra{(const char *)a, lda, m, k}, rb{(const char *)b, ldb, n, k};
    const bool direct = i8_direct(a, lda, b, ldb, k);
    return with_elem(dtype, [&](auto tag) {
        using O = decltype(tag);
        auto tiles = [&](int64_t side) { return ((m + side - 1) / side) * ((n + side - 1) / side); };
        const int64_t cus = resident_waves() / 16;
        // Up to 4 tokens the products on the vector units hide behind the weights'
        // bytes at every size: 1 x 4096 x 4096 takes 7.9 us (tiles 10.5), 1 x 16384 x
        // 4096 11.5 (12.7), 4 x 150000 x 2048 49 (55). With 5 to 8 they do where
        // tiles leave CUs without work, 8 x 4096 x 4096 9.3 (11.1), or come through
        // registers, 8 x 16385 x 4099 30 (37), and not elsewhere: 8 x 150000 x 2048
        // 67 (55).
        if (m == 1) return launch_few<O, 1>(rb, ra, sb, sa, out, ldo, stream);
        if (m == 2) return launch_few<O, 2>(rb, ra, sb, sa, out, ldo, stream);
        if (m <= 4) return launch_few<O, 4>(rb, ra, sb, sa, out, ldo, stream);
        if (i8_few(m, n, direct, cus)) return launch_few<O, 8>(rb, ra, sb, sa, out, ldo, stream);
        if (direct) {
            // 16 x 4096 x 8192 takes 14.3 us in 8 parts (17.6 whole), 16 x 300 x 8192
            // 10.8 in 8 (17.1), 128 x 4096 x 8192 16.9 in 4 (20.1), but 20 x 1024 x 3968,
            // of 31 steps, 11.0 in 3 (10.2).
            if (const int parts = i8_parts(m, n, k, direct, cus); parts > 1)
                return with_tile_of_64(tiles(64) * parts, cus, [&](auto shape) {
                    return launch_parts<O, typename decltype(shape)::template Product<MulI8>>(rb, ra, sb, sa, out, ldo, tiles(64), parts, (char *)ws, stream);
                });
            const int side = product_tile(k / kStepBytes, cus, tiles);
            return with_tile(side, tiles(side), cus, [&](auto shape) {
                return launch_tiles<O, typename decltype(shape)::template Product<MulI8>>(rb, ra, sb, sa, out, ldo, stream);
            });
        }
        // Off alignment the step's bytes pass through registers. 170 x 150000 x 7097
        // takes 569 us in tiles of 192 (3 a CU), 711 in tiles of 128 and 853 in tiles
        // of 64; 2000 x 9000 x 3001 162 (2 a CU), 132 and 195; 1000 x 4000 x 1001 19 in
        // tiles of 128 (one a CU) and 23 in tiles of 64.
        if (tiles(192) >= 3 * cus) return launch_tiles<O, TileProduct<MulI8, 192, 192, 2, 4, 2, 1, false>>(rb, ra, sb, sa, out, ldo, stream);
        if (tiles(128) >= cus) return launch_tiles<O, TileProduct<MulI8, 128, 128, 2, 4, 2, 1, false>>(rb, ra, sb, sa, out, ldo, stream);
        return launch_tiles<O, TileProduct<MulI8, 64, 64, 4, 2, 2, 1, false>>(rb, ra, sb, sa, out, ldo, stream);
    });
}

}  // namespace pace
