// One output tile of a product A B^T on the matrix cores of gfx950: A and B
// are rows of bytes along the summed axis, 8-bit integers or 16-bit floats.
//
// Tiles of both go from memory to LDS without passing registers, 128 bytes of
// the summed axis a step, two steps' buffers in turn: while the products of
// one step run, the next one's bytes are in flight. A row's eight 16-byte
// chunks lie in LDS at chunk ^ (row & 7), so the eight lanes that read one chunk
// of eight neighbouring rows touch all banks; since the memory side writes LDS
// in lane order, each lane fetches the chunk that belongs in its place.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "elem.hpp"

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

// kBM x kBN tiles by kWM x kWN waves. kDirect: rows are whole steps, their
// starts and strides whole 16-byte chunks, and the bytes go straight into LDS;
// otherwise they pass through registers.
template <typename Mul, int kBM, int kBN, int kWM, int kWN, bool kDirect>
struct TileProduct {
    static constexpr int kWaves = kWM * kWN, kThreads = kWaves * kWave;
    static constexpr int kTM = kBM / kWM / 16, kTN = kBN / kWN / 16;
    static constexpr int kBuf = (kBM + kBN) * kStepBytes, kLdsBytes = 2 * kBuf, kB = kBM * kStepBytes;
    // Pieces of 8 rows, 1 KiB, an instruction; a wave takes every kWaves-th.
    static constexpr int kPieces = (kBM + kBN) / 8, kMine = kPieces / kWaves;
    static_assert(kPieces % kWaves == 0 && (kBM / 8) % kWaves == 0, "whole shares");
    static constexpr int kMineA = kBM / 8 / kWaves;
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
    // The bytes on their way are there, and nobody reads what was read before.
    static __device__ __forceinline__ void ready() {
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
    }

    // The operands of half a step (64 bytes), and its products.
    struct Half {
        mfma_v4i a[kTM], b[kTN];
    };
    static __device__ __forceinline__ void half(const char *now, int s, Half &h) {
        const int lane = lane_id(), wave = threadIdx.x / kWave;
        const int at = (lane & 15) * kStepBytes + (((4 * s + (lane >> 4)) ^ (lane & 7)) << 4);
        const char *ra = now + wave / kWN * (kBM / kWM) * kStepBytes + at;
        const char *rb = now + kB + wave % kWN * (kBN / kWN) * kStepBytes + at;
#pragma unroll
        for (int i = 0; i < kTM; ++i) h.a[i] = *reinterpret_cast<const mfma_v4i *>(ra + i * 16 * kStepBytes);
#pragma unroll
        for (int j = 0; j < kTN; ++j) h.b[j] = *reinterpret_cast<const mfma_v4i *>(rb + j * 16 * kStepBytes);
    }
    __device__ __forceinline__ void products(const Half &h) {
#pragma unroll
        for (int i = 0; i < kTM; ++i)
#pragma unroll
            for (int j = 0; j < kTN; ++j) acc[i][j] = Mul::mul(h.a[i], h.b[j], acc[i][j]);
    }
    // Asks for an order of what stands before it: one read for every few products.
    template <int kReads>
    static __device__ __forceinline__ void interleave() {
        constexpr int kAll = kTM * kTN, kEach = kAll / kReads > 0 ? kAll / kReads : 1;
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
            fetch(0, lds);
            if (bytes >= 2 * kStepBytes) fetch(kStepBytes, lds + kBuf);
        }
#pragma unroll
        for (int i = 0; i < kTM; ++i)
#pragma unroll
            for (int j = 0; j < kTN; ++j) acc[i][j] = Acc{0, 0, 0, 0};
        int64_t k = 0;
        int buf = 0;
        if constexpr (kDirect) {
            // Half a step ahead: while one half's products run, the next half is
            // read from LDS, and between the halves the buffer that has just
            // been read is given to the step after the next.
            Half h0, h1;
            ready();
            half(lds, 0, h0);
            for (; k < bytes; k += kStepBytes) {
                half(lds + buf * kBuf, 1, h1);
                products(h0);
                interleave<kTM + kTN>();
                ready();
                if (k + 2 * kStepBytes < bytes) fetch(k + 2 * kStepBytes, lds + buf * kBuf);
                buf ^= 1;
                half(lds + buf * kBuf, 0, h0);       // after the last step nothing that is used
                products(h1);
                interleave<kTM + kTN>();
            }
        } else {
            // The next step's bytes are loaded while this one's products run.
            uint4 held[kMine];
#pragma unroll
            for (int i = 0; i < kMine; ++i) held[i] = staged(0, i);
            for (; k < bytes; k += kStepBytes) {
#pragma unroll
                for (int i = 0; i < kMine; ++i) *reinterpret_cast<uint4 *>(piece(lds + buf * kBuf, i) + lane_id() * 16) = held[i];
                ready();
                Half h;
                half(lds + buf * kBuf, 0, h);
                if (k + kStepBytes < bytes) {
#pragma unroll
                    for (int i = 0; i < kMine; ++i) held[i] = staged(k + kStepBytes, i);
                }
                products(h);
                half(lds + buf * kBuf, 1, h);
                products(h);
                buf ^= 1;
            }
        }
    }
};

// Which tile a workgroup takes. Workgroups go round the eight XCDs, each with
// an L2 of its own: each XCD takes a run of neighbouring tiles, and a run goes
// down columns of kGroup row tiles, so that what its workgroups read at one
// time is a block of few rows and columns.
template <int kGroup>
__device__ __forceinline__ void tile_of(uint32_t id, uint32_t tiles_m, uint32_t tiles_n, int &tm, int &tn) {
    const uint32_t all = tiles_m * tiles_n, per = all / 8, rest = all % 8;
    const uint32_t x = id % 8, i = id / 8;
    id = x * per + (x < rest ? x : rest) + i;
    const uint32_t band = kGroup * tiles_n, g = id / band;
    const uint32_t rows = tiles_m - g * kGroup < kGroup ? tiles_m - g * kGroup : kGroup;
    const uint32_t in = id - g * band;
    // the same in every lane
    tm = __builtin_amdgcn_readfirstlane((int)(g * kGroup + in % rows));
    tn = __builtin_amdgcn_readfirstlane((int)(in / rows));
}

}  // namespace pace
