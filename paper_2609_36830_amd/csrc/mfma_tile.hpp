// One output tile of a product A B^T on the matrix cores of gfx950: A and B
// are rows of bytes along the summed axis, 8-bit integers or 16-bit floats.
//
// Tiles of both go from memory to LDS without passing registers, 128 bytes of
// the summed axis a step, kDepth steps' buffers in turn: while the products of
// one step run, the next ones' bytes are in flight. A row's eight 16-byte
// chunks lie in LDS at chunk ^ (row & 7), so the eight lanes that read one chunk
// of eight neighbouring rows touch all banks; since the memory side writes LDS
// in lane order, each lane fetches the chunk that belongs in its place.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "elem.hpp"
#include "rules.hpp"

namespace pace {

typedef int mfma_v4i __attribute__((ext_vector_type(4)));
typedef float mfma_v4f __attribute__((ext_vector_type(4)));
typedef _Float16 mfma_v8h __attribute__((ext_vector_type(8)));

// 16x16 products over 64 bytes of the summed axis: lane l holds 16 bytes of row
// l & 15 of each side; result element i is (row 4 (l >> 4) + i, column l & 15).
// (32x32 products are no faster, and their results lie in 16-byte pieces of 32
// rows to a store where these lie in 32-byte pieces of 16.)
struct MulI8 {
    using Acc = mfma_v4i;
    static __device__ __forceinline__ Acc mul(mfma_v4i a, mfma_v4i b, Acc c) {
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
    }
};
struct MulF16 {
    using Acc = mfma_v4f;
    static __device__ __forceinline__ Acc mul(mfma_v4i a, mfma_v4i b, Acc c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(mfma_v8h, a), __builtin_bit_cast(mfma_v8h, b), c,
                                                      0, 0, 0);
    }
};

constexpr int kStepBytes = 128;            // of the summed axis

// A row operand: `rows` rows of `bytes` bytes, `stride` bytes apart.
struct Rows {
    const char *p;
    int64_t stride, rows, bytes;
};

// What a workgroup does with a tile: all of its steps, one of several runs of them,
// whose sums it leaves in memory, or adding those up.
enum TileWork { kWhole, kPart, kJoin };
// The part-th of `parts` runs of an operand's steps, by rows of whole steps.
__device__ __forceinline__ Rows part_of(Rows m, uint32_t part, int parts) {
    const int64_t run = (m.bytes / kStepBytes + parts - 1) / parts * kStepBytes, at = part * run;
    return Rows{m.p + at, m.stride, m.rows, m.bytes - at < run ? m.bytes - at : run};
}

// kBM x kBN tiles by kWM x kWN waves. kDirect: rows are whole steps, their
// starts and strides whole 16-byte chunks, and the bytes go straight into LDS;
// otherwise they pass through registers.
template <typename Mul, int kBM, int kBN, int kWM, int kWN, int kDepth, int kUnit, bool kDirect>
struct TileProduct {
    static constexpr int kRows = kBM, kCols = kBN, kWavesN = kWN, kWaves = kWM * kWN, kThreads = kWaves * kWave;
    static constexpr int kTM = kBM / kWM / 16, kTN = kBN / kWN / 16;
    static constexpr int kBuf = (kBM + kBN) * kStepBytes, kLdsBytes = kDepth * kBuf, kB = kBM * kStepBytes;
    // Pieces of 8 rows, 1 KiB, an instruction; a wave takes every kWaves-th.
    static constexpr int kPieces = (kBM + kBN) / 8, kMine = kPieces / kWaves;
    static_assert(kPieces % kWaves == 0 && (kBM / 8) % kWaves == 0, "whole shares");
    static constexpr int kMineA = kBM / 8 / kWaves;
    // A stage is kUnit steps between two barriers: one, or two where a step has
    // few products to cover a barrier and the reads behind it.
    static constexpr int kStages = kDepth / kUnit;
    static_assert(kUnit == 1 || (kUnit == 2 && kDirect && kDepth % 2 == 0), "stages");
    static constexpr int64_t kStageBytes = kUnit * kStepBytes;
    using Acc = typename Mul::Acc;

    Acc acc[kTM][kTN];
    Rows a, b;
    int64_t row_a, row_b;
    const char *pa, *pb;                             // the tile's first rows
    uint32_t from[kDirect ? kMine : 1];              // this lane's pieces, in bytes behind them

    // The first of the four consecutive rows in the tile of acc[i][..], and the column of acc[..][j].
    static __device__ __forceinline__ int row4(int i) {
        return (int)(threadIdx.x / kWave) / kWN * (kBM / kWM) + i * 16 + (lane_id() >> 4) * 4;
    }
    static __device__ __forceinline__ int col(int j) {
        return (int)(threadIdx.x / kWave) % kWN * (kBN / kWN) + j * 16 + (lane_id() & 15);
    }

    // The sums of a part: each thread's, 16 bytes by 16 bytes.
    static constexpr int64_t kSumBytes = (int64_t)kBM * kBN * 4;
    __device__ __forceinline__ void leave_sums(char *to) const {
        Acc *mine = reinterpret_cast<Acc *>(to) + threadIdx.x;
#pragma unroll
        for (int k = 0; k < kTM * kTN; ++k) mine[k * kThreads] = acc[k / kTN][k % kTN];
    }
    // The parts' sums, in the order of the parts.
    __device__ __forceinline__ void add_sums(const char *from, int parts) {
        const Acc *mine = reinterpret_cast<const Acc *>(from) + threadIdx.x;
#pragma unroll
        for (int k = 0; k < kTM * kTN; ++k) acc[k / kTN][k % kTN] = mine[k * kThreads];
#pragma unroll 4
        for (int p = 1; p < parts; ++p)
#pragma unroll
            for (int k = 0; k < kTM * kTN; ++k) acc[k / kTN][k % kTN] += mine[(p * kTM * kTN + k) * kThreads];
    }

    // The row of an operand that this lane fetches in its i-th piece. Rows
    // beyond the last are that one again: what they give is not kept.
    static __device__ __forceinline__ int64_t row_of(const Rows &m, int64_t row0, int i) {
        const int64_t row = row0 + (i * kWaves + threadIdx.x / kWave) * 8 + (lane_id() >> 3);
        return row < m.rows ? row : m.rows - 1;
    }
    static __device__ __forceinline__ int lane_chunk() { return ((lane_id() & 7) ^ (lane_id() >> 3)) << 4; }
    static __device__ __forceinline__ char *piece(char *to, int i) { return to + (i * kWaves + threadIdx.x / kWave) * 1024; }

    static __device__ __forceinline__ uint4 load_chunk(const Rows &m, int64_t row, int64_t at) {
        const char *p = m.p + row * m.stride + at;
        if (at + 16 <= m.bytes) return load_a1(p);
        uint32_t w[4] = {0, 0, 0, 0};
        if (at < m.bytes)
            for (int k = 0; at + k < m.bytes; ++k) w[k >> 2] |= (uint32_t)(uint8_t)p[k] << (8 * (k & 3));
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ __forceinline__ uint4 staged(int64_t k, int i) const {
        return i < kMineA ? load_chunk(a, row_of(a, row_a, i), k + lane_chunk())
                          : load_chunk(b, row_of(b, row_b, i - kMineA), k + lane_chunk());
    }
    // Begins to fetch the whole step k.
    __device__ __forceinline__ void fetch(int64_t k, char *to) const {
#pragma unroll
        for (int i = 0; i < kMine; ++i)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)((i < kMineA ? pa : pb) + k + from[i]),
                                             (__attribute__((address_space(3))) void *)piece(to, i), 16, 0, 0);
    }
    // The stage from k on; a step that is not there is zeros.
    __device__ __forceinline__ void fetch_stage(int64_t k, char *to) const {
        fetch(k, to);
        if constexpr (kUnit == 2) {
            if (k + kStepBytes < a.bytes) {
                fetch(k + kStepBytes, to + kBuf);
            } else {
#pragma unroll
                for (int i = 0; i < kMine; ++i) *reinterpret_cast<uint4 *>(piece(to + kBuf, i) + lane_id() * 16) = make_uint4(0, 0, 0, 0);
            }
        }
    }
    // All but the newest kLeft steps on their way are there, and nobody reads
    // what was read before. (Fetches are counted in their order; a barrier with
    // a fence would wait for all of them.)
    template <int kLeft>
    static __device__ __forceinline__ void ready() {
        static_assert(kLeft * kMine < 64, "the counter's range");
        if constexpr (kLeft == 0) {
            __builtin_amdgcn_s_waitcnt(0);
            __syncthreads();
            return;
        }
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kLeft * kMine) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    }

    // The operands of half a stage (64 bytes times kUnit), and its products.
    struct Half {
        mfma_v4i a[kUnit][kTM], b[kUnit][kTN];
    };
    static __device__ __forceinline__ void half(const char *now, int s, Half &h) {
        if (kUnit == 2) now += s * kBuf;             // a whole step
        half_of(now, now + kB, s, h);
    }
    static __device__ __forceinline__ void half_of(const char *now_a, const char *now_b, int s, Half &h) {
        const int lane = lane_id(), wave = threadIdx.x / kWave;
#pragma unroll
        for (int u = 0; u < kUnit; ++u) {
            const int at = (lane & 15) * kStepBytes + (((4 * (kUnit == 2 ? u : s) + (lane >> 4)) ^ (lane & 7)) << 4);
            const char *ra = now_a + wave / kWN * (kBM / kWM) * kStepBytes + at;
            const char *rb = now_b + wave % kWN * (kBN / kWN) * kStepBytes + at;
#pragma unroll
            for (int i = 0; i < kTM; ++i) h.a[u][i] = *reinterpret_cast<const mfma_v4i *>(ra + i * 16 * kStepBytes);
#pragma unroll
            for (int j = 0; j < kTN; ++j) h.b[u][j] = *reinterpret_cast<const mfma_v4i *>(rb + j * 16 * kStepBytes);
        }
    }
    __device__ __forceinline__ void products(const Half &h) {
#pragma unroll
        for (int u = 0; u < kUnit; ++u)
#pragma unroll
            for (int i = 0; i < kTM; ++i)
#pragma unroll
                for (int j = 0; j < kTN; ++j) acc[i][j] = Mul::mul(h.a[u][i], h.b[u][j], acc[i][j]);
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < kTM; ++i)
#pragma unroll
            for (int j = 0; j < kTN; ++j) acc[i][j] = Acc{0, 0, 0, 0};
    }
    // The products of a step of operands that are in LDS already, onto acc.
    __device__ __forceinline__ void step(const char *now_a, const char *now_b) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            Half h;
            half_of(now_a, now_b, k, h);
            products(h);
        }
    }
    // Asks for an order of what stands before it: one read for every few products.
    template <int kReads>
    static __device__ __forceinline__ void interleave() {
        constexpr int kAll = kUnit * kTM * kTN, kEach = kAll / kReads > 0 ? kAll / kReads : 1;
#pragma unroll
        for (int i = 0; i < kReads; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x8, kEach, 0);
        }
    }

    // The tile of rows row_a_ .. of a_ and row_b_ .. of b_, into acc.
    __device__ __forceinline__ void run(const Rows &a_, int64_t row_a_, const Rows &b_, int64_t row_b_, char *lds) {
        a = a_, b = b_, row_a = row_a_, row_b = row_b_;
        const int64_t bytes = a.bytes;
        if constexpr (kDirect) {
            pa = a.p + row_a * a.stride;
            pb = b.p + row_b * b.stride;
#pragma unroll
            for (int i = 0; i < kMine; ++i)
                from[i] = (i < kMineA ? (uint32_t)((row_of(a, row_a, i) - row_a) * a.stride)
                                      : (uint32_t)((row_of(b, row_b, i - kMineA) - row_b) * b.stride)) + (uint32_t)lane_chunk();
#pragma unroll
            for (int d = 0; d < kStages; ++d)
                if (d * kStageBytes < bytes) fetch_stage(d * kStageBytes, lds + d * kUnit * kBuf);
        }
        clear();
        int64_t k = 0;
        if constexpr (kDirect) {
            // Half a stage ahead: while one half's products run, the next half is
            // read from LDS, and between the halves the buffers that have just
            // been read are given to the stage kStages further on.
            Half h0, h1;
            if (kStages * kStageBytes <= bytes)
                ready<(kStages - 1) * kUnit>();
            else
                ready<0>();
            half(lds, 0, h0);
            const char *now = lds;
            for (; k < bytes; k += kStageBytes) {
                half(now, 1, h1);
                products(h0);
                interleave<kUnit *(kTM + kTN)>();
                if (kStages == 2 || k + kStages * kStageBytes > bytes)
                    ready<0>();
                else
                    ready<(kStages - 2) * kUnit>();
                if (k + kStages * kStageBytes < bytes) fetch_stage(k + kStages * kStageBytes, const_cast<char *>(now));
                now = now + kUnit * kBuf == lds + kLdsBytes ? lds : now + kUnit * kBuf;
                half(now, 0, h0);                    // after the last stage nothing that is used
                products(h1);
                interleave<kUnit *(kTM + kTN)>();
            }
        } else {
            // kAhead steps' bytes are on their way into registers while one step's products
            // run: one for tiles with many registers of their own and many products a step.
            constexpr int kAhead = kBM > 64 ? 1 : 2;
            uint4 held[kAhead][kMine];
            const char *from_row[kMine];
#pragma unroll
            for (int i = 0; i < kMine; ++i)
                from_row[i] = (i < kMineA ? a.p + row_of(a, row_a, i) * a.stride : b.p + row_of(b, row_b, i - kMineA) * b.stride) + lane_chunk();
            auto load = [&](int64_t at, uint4 (&h)[kMine]) {
                if (at + kStepBytes <= bytes) {
#pragma unroll
                    for (int i = 0; i < kMine; ++i) h[i] = load_a1(from_row[i] + at);
                } else if (at < bytes) {             // the last step, in part
#pragma unroll
                    for (int i = 0; i < kMine; ++i) h[i] = staged(at, i);
                }
            };
#pragma unroll
            for (int d = 0; d < kAhead; ++d) load(d * kStepBytes, held[d]);
            static_assert(kDepth % kAhead == 0, "whole turns of the register stages");
            while (k < bytes) {
#pragma unroll
                for (int d = 0; d < kDepth; ++d) {
                    char *now = lds + d * kBuf;
#pragma unroll
                    for (int i = 0; i < kMine; ++i) *reinterpret_cast<uint4 *>(piece(now, i) + lane_id() * 16) = held[d % kAhead][i];
                    load(k + kAhead * kStepBytes, held[d % kAhead]);
                    // waits for LDS only: the loads of the steps to come stay on their way
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                    __builtin_amdgcn_s_barrier();
                    asm volatile("" ::: "memory");
                    Half h;
                    half(now, 0, h);
                    products(h);
                    half(now, 1, h);
                    products(h);
                    k += kStepBytes;
                    if (k >= bytes) break;
                }
            }
        }
    }

    // ---- results in 16 bits, by columns or by rows, through a wave's own part of LDS ----
    static constexpr int kRowsW = kBM / kWM, kColsW = kBN / kWN;
    static constexpr int kRunC = kRowsW * 2 + 16, kRunR = kColsW * 2 + 16;      // a line in LDS: 4 banks on from the last line's
    static constexpr int kTurnW = kColsW * kRunC > kRowsW * kRunR ? kColsW * kRunC : kRowsW * kRunR;
    static constexpr int kTurnBytes = kWaves * kTurnW;

    // bits(i, j) packs the values of acc[i][j] as two words; put(column, first
    // row, eight values) takes them along the rows. Coordinates are the tile's.
    template <typename Bits, typename Put>
    static __device__ __forceinline__ void by_columns(char *lds, Bits bits, Put put) {
        const int wave = threadIdx.x / kWave, lane = lane_id();
        char *mine = lds + wave * kTurnW;
        const int r0 = wave / kWN * kRowsW, c0 = wave % kWN * kColsW;
#pragma unroll
        for (int j = 0; j < kTN; ++j)
#pragma unroll
            for (int i = 0; i < kTM; ++i) *reinterpret_cast<uint2 *>(mine + (col(j) - c0) * kRunC + (row4(i) - r0) * 2) = bits(i, j);
        constexpr int kPieces = kRowsW / 8, kAll = kPieces * kColsW;
#pragma unroll
        for (int p = 0; p < kAll; p += kWave) {
            const int at = p + lane;
            if (kAll % kWave != 0 && at >= kAll) break;
            put(c0 + at / kPieces, r0 + at % kPieces * 8, *reinterpret_cast<const uint4 *>(mine + at / kPieces * kRunC + at % kPieces * 16));
        }
    }
    // The same by rows: neighbouring lanes, which hold neighbouring columns,
    // exchange two of their four rows. put(row, first column, eight values).
    template <typename Bits, typename Put>
    static __device__ __forceinline__ void by_rows(char *lds, Bits bits, Put put) {
        const int wave = threadIdx.x / kWave, lane = lane_id();
        char *mine = lds + wave * kTurnW;
        const int r0 = wave / kWN * kRowsW, c0 = wave % kWN * kColsW;
        const bool odd = lane & 1;
#pragma unroll
        for (int j = 0; j < kTN; ++j)
#pragma unroll
            for (int i = 0; i < kTM; ++i) {
                const uint2 b = bits(i, j);
                const uint32_t got = dpp_u32<0xb1, 0xf>(0u, odd ? b.x : b.y);      // from the lane of the pair
                const uint32_t left = odd ? got : b.x, right = odd ? b.y : got;    // two rows of the left and of the right column
                char *to = mine + (row4(i) + (odd ? 2 : 0) - r0) * kRunR + (col(j) - (odd ? 1 : 0) - c0) * 2;
                *reinterpret_cast<uint32_t *>(to) = (left & 0xffffu) | (right << 16);
                *reinterpret_cast<uint32_t *>(to + kRunR) = (left >> 16) | (right & 0xffff0000u);
            }
        constexpr int kPieces = kColsW / 8, kAll = kPieces * kRowsW;
#pragma unroll
        for (int p = 0; p < kAll; p += kWave) {
            const int at = p + lane;
            if (kAll % kWave != 0 && at >= kAll) break;
            put(r0 + at / kPieces, c0 + at % kPieces * 8, *reinterpret_cast<const uint4 *>(mine + at / kPieces * kRunR + at % kPieces * 16));
        }
    }
};

// Two 16-bit values of type T as a word.
template <typename T>
__device__ __forceinline__ uint32_t pair_bits(float a, float b) {
    return (uint32_t)__builtin_bit_cast(uint16_t, from_f32<T>(a)) | ((uint32_t)__builtin_bit_cast(uint16_t, from_f32<T>(b)) << 16);
}

// Which tile a workgroup takes. Workgroups go round the eight XCDs, each with
// an L2 of its own: xcd_run gives each XCD a run of neighbouring numbers, and
// the tiles of a run go down columns of kGroup row tiles, so that what an XCD's
// workgroups read at one time is a block of few rows and columns.
__device__ __forceinline__ uint32_t xcd_run(uint32_t id, uint32_t all) {
    const uint32_t per = all / 8, rest = all % 8, x = id % 8;
    return x * per + (x < rest ? x : rest) + id / 8;
}
template <int kGroup>
__device__ __forceinline__ void tile_of(uint32_t id, uint32_t tiles_m, uint32_t tiles_n, int &tm, int &tn) {
    const uint32_t band = kGroup * tiles_n, g = id / band;
    const uint32_t rows = tiles_m - g * kGroup < kGroup ? tiles_m - g * kGroup : kGroup;
    const uint32_t in = id - g * band;
    // the same in every lane
    tm = __builtin_amdgcn_readfirstlane((int)(g * kGroup + in % rows));
    tn = __builtin_amdgcn_readfirstlane((int)(in / rows));
}
// The same for the lower triangle of `tiles` x `tiles` tiles.
template <int kGroup>
__device__ __forceinline__ void lower_tile_of(uint32_t id, uint32_t tiles, int &tm, int &tn) {
    int64_t t = (int64_t)((sqrt((double)(8 * (int64_t)id + 1)) - 1.0) * 0.5);      // the row it would be in, row by row
    while (t * (t + 1) / 2 > id) --t;
    while ((t + 1) * (t + 2) / 2 <= id) ++t;
    const uint32_t r0 = (uint32_t)t / kGroup * kGroup, rows = tiles - r0 < kGroup ? tiles - r0 : kGroup;
    uint32_t in = id - r0 * (r0 + 1) / 2, c = 0, r = 0;
    if (in < rows * (r0 + 1)) {                      // columns that all rows of the band have
        c = in / rows;
        r = in % rows;
    } else {                                         // the band's own triangle
        in -= rows * (r0 + 1);
        for (c = r0 + 1; in >= rows - (c - r0); ++c) in -= rows - (c - r0);
        r = c - r0 + in;
    }
    tm = __builtin_amdgcn_readfirstlane((int)(r0 + r));
    tn = __builtin_amdgcn_readfirstlane((int)c);
}

// Runs f with the tile of a side of product_tile: eight waves, and as many
// steps in flight as the LDS of a CU holds, for 64 (the only side whose steps are
// split into parts) of two workgroups where there is work for more than one a CU.
template <int kBM, int kBN, int kWM, int kWN, int kDepth, int kUnit>
struct TileShape {
    template <typename Mul>
    using Product = TileProduct<Mul, kBM, kBN, kWM, kWN, kDepth, kUnit, true>;
};
template <typename F>
auto with_tile_of_64(int64_t jobs, int64_t cus, F f) {
    return jobs > cus ? f(TileShape<64, 64, 4, 2, 4, 2>{}) : f(TileShape<64, 64, 4, 2, 8, 2>{});
}
template <typename F>
auto with_tile(int side, int64_t tiles, int64_t cus, F f) {
    switch (side) {
        case 256: return f(TileShape<256, 256, 2, 4, 2, 1>{});
        case 192: return f(TileShape<192, 192, 2, 4, 2, 1>{});
        case 128: return f(TileShape<128, 128, 2, 4, 4, 1>{});
        default: return with_tile_of_64(tiles, cus, f);
    }
}

}  // namespace pace
