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

// kBM x kBN tiles by kWM x kWN waves. kDirect: rows and strides are whole,
// aligned 16-byte chunks, fetched straight into LDS; otherwise, and for a last
// step that is not whole, the bytes pass through registers.
template <typename Mul, int kBM, int kBN, int kWM, int kWN, bool kDirect>
struct TileProduct {
    static constexpr int kWaves = kWM * kWN, kThreads = kWaves * kWave;
    static constexpr int kTM = kBM / kWM / 16, kTN = kBN / kWN / 16;
    static constexpr int kBuf = (kBM + kBN) * kStepBytes, kLdsBytes = 2 * kBuf;
    // Pieces of 8 rows, 1 KiB, an instruction; a wave takes every kWaves-th.
    static constexpr int kPieces = (kBM + kBN) / 8, kMine = kPieces / kWaves;
    static_assert(kPieces % kWaves == 0 && (kBM / 8) % kWaves == 0, "whole shares");
    static constexpr int kMineA = kBM / 8 / kWaves;
    using Acc = typename Mul::Acc;

    Acc acc[kTM][kTN];

    // The row of the operand that this lane fetches in its i-th piece. Rows
    // beyond the last are that one again: what they give is not kept.
    static __device__ __forceinline__ int64_t row_of(const Rows &m, int64_t row0, int i) {
        const int64_t row = row0 + (i * kWaves + threadIdx.x / kWave) * 8 + (lane_id() >> 3);
        return row < m.rows ? row : m.rows - 1;
    }
    static __device__ __forceinline__ int lane_chunk() { return ((lane_id() & 7) ^ (lane_id() >> 3)) << 4; }

    static __device__ __forceinline__ uint4 load_chunk(const Rows &m, int64_t row, int64_t at) {
        const char *from = m.p + row * m.stride + at;
        if (at + 16 <= m.bytes) return load_a1(from);
        uint32_t w[4] = {0, 0, 0, 0};
        if (at < m.bytes)
            for (int b = 0; at + b < m.bytes; ++b) w[b >> 2] |= (uint32_t)(uint8_t)from[b] << (8 * (b & 3));
        return make_uint4(w[0], w[1], w[2], w[3]);
    }

    __device__ __forceinline__ void run(const Rows &a, int64_t row_a, const Rows &b, int64_t row_b, char *lds, int64_t k0,
                                        int64_t k1) {
        const int wave = threadIdx.x / kWave, lane = lane_id();
        const int wm = wave / kWN, wn = wave % kWN;
#pragma unroll
        for (int i = 0; i < kTM; ++i)
#pragma unroll
            for (int j = 0; j < kTN; ++j) acc[i][j] = Acc{0, 0, 0, 0};
        if (k0 >= k1) return;
        constexpr int kB = kBM * kStepBytes;
        // Where this lane finds chunk 4 s + (lane >> 4) of row lane & 15 of a 16-row group.
        const int row = (lane & 15) * kStepBytes;
        const int c0 = row + ((((lane >> 4)) ^ (lane & 7)) << 4), c1 = row + (((4 + (lane >> 4)) ^ (lane & 7)) << 4);
        const int base_a = wm * (kBM / kWM) * kStepBytes, base_b = kB + wn * (kBN / kWN) * kStepBytes;

        // Where the lane's pieces come from, in bytes behind each tile's first row.
        const char *pa = a.p + row_a * a.stride, *pb = b.p + row_b * b.stride;
        uint32_t from[kDirect ? kMine : 1];
        if constexpr (kDirect) {
#pragma unroll
            for (int i = 0; i < kMine; ++i)
                from[i] = (i < kMineA ? (uint32_t)((row_of(a, row_a, i) - row_a) * a.stride)
                                      : (uint32_t)((row_of(b, row_b, i - kMineA) - row_b) * b.stride)) + (uint32_t)lane_chunk();
        }
        uint4 held[kDirect ? 1 : kMine];
        auto piece = [&](char *buf, int i) { return buf + (i * kWaves + wave) * 1024; };
        auto staged = [&](int64_t k, int i) {
            return i < kMineA ? load_chunk(a, row_of(a, row_a, i), k + lane_chunk())
                              : load_chunk(b, row_of(b, row_b, i - kMineA), k + lane_chunk());
        };
        // Begins to fetch the whole step k (into `to`), and ends it.
        auto fetch = [&](int64_t k, char *to) {
#pragma unroll
            for (int i = 0; i < kMine; ++i) {
                if constexpr (kDirect)
                    __builtin_amdgcn_global_load_lds(
                        (const __attribute__((address_space(1))) void *)((i < kMineA ? pa : pb) + k + from[i]),
                        (__attribute__((address_space(3))) void *)piece(to, i), 16, 0, 0);
                else
                    held[i] = staged(k, i);
            }
        };
        auto settle = [&](char *buf) {
            if constexpr (!kDirect) {
#pragma unroll
                for (int i = 0; i < kMine; ++i) *reinterpret_cast<uint4 *>(piece(buf, i) + lane * 16) = held[i];
            }
        };
        // The step that ends at k1, whole or not.
        auto fetch_last = [&](int64_t k, char *buf) {
            if (k + kStepBytes <= k1) {
                fetch(k, buf);
                settle(buf);
            } else {
#pragma unroll 1
                for (int i = 0; i < kMine; ++i) *reinterpret_cast<uint4 *>(piece(buf, i) + lane * 16) = staged(k, i);
            }
        };
        // The operands of half a step (64 bytes), and its products.
        struct Half {
            mfma_v4i a[kTM], b[kTN];
        };
        auto half = [&](const char *now, int s, Half &h) {
            const int c = s ? c1 : c0;
#pragma unroll
            for (int i = 0; i < kTM; ++i) h.a[i] = *reinterpret_cast<const mfma_v4i *>(now + base_a + i * 16 * kStepBytes + c);
#pragma unroll
            for (int j = 0; j < kTN; ++j) h.b[j] = *reinterpret_cast<const mfma_v4i *>(now + base_b + j * 16 * kStepBytes + c);
        };
        auto products = [&](const Half &h) {
#pragma unroll
            for (int i = 0; i < kTM; ++i)
#pragma unroll
                for (int j = 0; j < kTN; ++j) acc[i][j] = Mul::mul(h.a[i], h.b[j], acc[i][j]);
        };
        // The bytes on their way are there, and nobody reads what was read before.
        auto ready = [&]() {
            __builtin_amdgcn_s_waitcnt(0);
            __syncthreads();
        };
        int64_t k = k0, fetched = k0;
        int buf = 0;
        if constexpr (kDirect) {
            // Half a step ahead: while one half's products run, the next half is
            // read from LDS, and between the halves the buffer that has just
            // been read is given to the step after the next.
            if (k0 + 3 * kStepBytes <= k1) {
                fetch(k0, lds);
                ready();
                fetch(k0 + kStepBytes, lds + kBuf);
                Half h0, h1;
                half(lds, 0, h0);
                for (; k + 3 * kStepBytes <= k1; k += kStepBytes) {
                    half(lds + buf * kBuf, 1, h1);
                    products(h0);
                    interleave<kTM + kTN, 0>();
                    ready();
                    fetch(k + 2 * kStepBytes, lds + buf * kBuf);
                    buf ^= 1;
                    half(lds + buf * kBuf, 0, h0);
                    products(h1);
                    interleave<kTM + kTN, kMine>();
                }
                fetched = k + 2 * kStepBytes;
            }
        } else {
            if (k0 + 2 * kStepBytes <= k1) {
                fetch(k0, lds);
                settle(lds);
                for (; k + 2 * kStepBytes <= k1; k += kStepBytes) {
                    ready();
                    Half h;
                    half(lds + buf * kBuf, 0, h);
                    fetch(k + kStepBytes, nullptr);
                    products(h);
                    half(lds + buf * kBuf, 1, h);
                    products(h);
                    buf ^= 1;
                    settle(lds + buf * kBuf);
                }
                fetched = k + kStepBytes;
            }
        }
        // The last steps, whole or not.
        if (fetched == k0) {
            fetch_last(k0, lds);
            fetched += kStepBytes;
        }
        for (; k < k1; k += kStepBytes) {
            ready();
            if (fetched == k + kStepBytes && fetched < k1) {
                fetch_last(fetched, lds + (buf ^ 1) * kBuf);
                fetched += kStepBytes;
            }
            Half h;
            half(lds + buf * kBuf, 0, h);
            products(h);
            half(lds + buf * kBuf, 1, h);
            products(h);
            buf ^= 1;
        }
    }

    // Asks for an order of what stands before it: one read (and, while there
    // are some, one fetch) for every few products.
    template <int kReads, int kFetches>
    static __device__ __forceinline__ void interleave() {
        constexpr int kAll = kTM * kTN, kEach = kAll / kReads > 0 ? kAll / kReads : 1;
#pragma unroll
        for (int i = 0; i < kReads; ++i) {
            if (i < kFetches) __builtin_amdgcn_sched_group_barrier(0x10, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x8, kEach, 0);
        }
    }

    // The first of the four consecutive rows in the tile of acc[i][..], and the column of acc[..][j].
    static __device__ __forceinline__ int row4(int i) {
        return (int)(threadIdx.x / kWave) / kWN * (kBM / kWM) + (lane_id() >> 4) * 4 + i * 16;
    }
    static __device__ __forceinline__ int col(int j) {
        return (int)(threadIdx.x / kWave) % kWN * (kBN / kWN) + (lane_id() & 15) + j * 16;
    }
};

// Which tile a workgroup takes. Workgroups go round the eight XCDs, each with
// an L2 of its own: each XCD takes a run of neighbouring tiles, and a run goes
// down columns of kGroup row tiles, so that what its workgroups read at one
// time is a block of few rows and columns.
template <int kGroup>
__device__ __forceinline__ void tile_of(int64_t id, int64_t tiles_m, int64_t tiles_n, int64_t &tm, int64_t &tn) {
    const int64_t all = tiles_m * tiles_n, per = all / 8, rest = all % 8;
    const int64_t x = id % 8, i = id / 8;
    id = x * per + (x < rest ? x : rest) + i;
    const int64_t band = kGroup * tiles_n, g = id / band;
    const int64_t rows = tiles_m - g * kGroup < kGroup ? tiles_m - g * kGroup : kGroup;
    const int64_t in = id - g * band;
    tm = g * kGroup + in % rows;
    tn = in / rows;
}

}  // namespace pace
