// Orthogonalised updates for gfx950, by Newton-Schulz steps on the matrix cores.
//
//   X = G / (|G|_F + eps);   steps times:  A = X X^T,  C = a I + b A + c A A,  X <- C X
//
// on the orientation with m <= n rows. Three products a step: A and A A are
// symmetric, so only their lower tiles are formed and both halves written.
// Between products X, A and C are held as binary16, scaled by powers of two:
// the singular values are at most about 1.2, so their range is known, and 11 bits
// lose eight times less than bfloat16 (the result's type) would: five steps on noise,
// alone or over strong directions, end 1.9e-3 to 2.6e-3 from binary64's (2-norm,
// relative), the rounding of the result alone 1.7e-3. In directions that the update
// lacks the roundings grow as a small singular value would, 485 times in five
// quintic steps: an update of rank k ends some 0.2 / sqrt(k) away. Elements of X below 2^-24 of the norm, which lie far below the
// typical one's 1 / sqrt(m n), are held to 2^-35 of it. The products' sums are
// binary32. X is kept by rows for X X^T and by columns for C X, so that
// every product reads both sides along the summed axis.
//
// Large updates are bound by the matrix cores: five steps on 4096 x 16384 take
// 4.35 ms for 4.47e12 operations (1.03 PFLOP/s; a library's large product in
// binary16 1.43), X X^T 280 us, A A 77, C X 480 each, with the cores busy 52% to
// 62% of the time at 1.85 to 2.0 GHz, behind their tiles' LDS reads; the norm and
// the turning are 70 + 94 us at 3.8 and 5.7 TB/s. Small ones are bound by their 12 to
// 17 launches: 24 updates of 256 x 256 take 77 us; the smallest, in one launch, are
// bound by one workgroup's chain of products, each read from LDS before it runs: 24 of
// 64 x 64 take 12 us, 128 x 256 44, and 2000 of those 375 (8 rounds of workgroups, one a CU;
// the cores busy 24%, the waves waiting 36%, LDS conflicts 5%). Between, tiles do not
// fill the chip: 3001 x 1000 takes 193 us (X X^T in parts 10 + 4, A A 8, C X 16).
#include "elem.hpp"
#include "kernels.hpp"
#include "mfma_tile.hpp"

#pragma clang fp contract(off)

namespace pace {

namespace {

constexpr float kScaleX = 1024.0f;                 // X up to 64 in binary16, in steps of 2^-34 at least
constexpr float kScaleA = 256.0f;                  // A and C up to 256, of 2^-32
constexpr int kNormWaves = 4;                      // of a workgroup
constexpr int kNormBlocks = 1024;                  // partial sums of squares of a matrix, at most
constexpr int kTurn = 64;                          // side of the tiles that are turned
constexpr int kTurnRun = 4;                        // of them by a workgroup, where there are kTurnMany
constexpr int64_t kTurnMany = 8192;

// The m x n orientation of one matrix of the batch and its workspace; the rows'
// ends up to a multiple of 64 elements are zeros, so that products have whole steps.
struct OrthoShape {
    int64_t m, n, mp, np;                          // mp, np: m and n up to 64
    int64_t x, xt, xt2, a, c, bytes;               // byte offsets in a matrix's workspace, and its size
    int64_t split;                                 // behind all matrices': the split products' parts (0: none)
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
    s.split = 0;
    return s;
}
// Waves take pieces of kNormPiece elements of rows.
constexpr int kNormPiece = 4096;
int ortho_norm_blocks(int64_t rows, int64_t cols) {
    const int64_t pieces = rows * ((cols + kNormPiece - 1) / kNormPiece), b = (pieces + kNormWaves - 1) / kNormWaves;
    return (int)(b > kNormBlocks ? kNormBlocks : b);
}

// The workspace of the parts of X X^T.
size_t ortho_split_bytes(const OrthoShape &s, int64_t batch) {
    const int64_t t = (s.m + 63) / 64, tiles = t * (t + 1) / 2 * batch;
    const int parts = product_parts(s.np / 64, tiles);
    return parts == 1 ? 0 : (size_t)(tiles * parts) * 64 * 64 * sizeof(float);
}

// The factor of an update whose squares add up to `squares`, in binary64: updates of
// any size. A zero update's, with an eps near 0, is no number that leaves it 0.
__device__ __forceinline__ double ortho_factor(double squares, double eps) {
    const double f = (double)kScaleX / (sqrt(squares) + eps);
    return f == __builtin_inf() ? 0.0 : f;
}

// The sum over a workgroup of four waves, in thread order's tree, in every thread.
__device__ __forceinline__ double block_total(double v, double *part) {
#pragma unroll
    for (int off = kWave / 2; off >= 1; off >>= 1) v += __shfl_xor(v, off, kWave);
    if (lane_id() == 0) part[threadIdx.x / kWave] = v;
    __syncthreads();
    return (part[0] + part[1]) + (part[2] + part[3]);
}

// Sums of squares, in binary64: no square of a finite binary32 number leaves its range.
template <typename T>
__global__ __launch_bounds__(kNormWaves *kWave) void ortho_norm_kernel(const T *__restrict__ g, int64_t rows, int64_t cols,
                                                                       int64_t stride, int64_t batch_stride, char *ws,
                                                                       int64_t ws_stride) {
    constexpr int V = kVecOf<T>;
    __shared__ double part[kNormWaves];
    const T *mat = g + blockIdx.y * batch_stride;
    const int64_t pieces = (cols + kNormPiece - 1) / kNormPiece, all = rows * pieces;
    double sum[V];
#pragma unroll
    for (int e = 0; e < V; ++e) sum[e] = 0.0;
    for (int64_t p = (int64_t)blockIdx.x * kNormWaves + threadIdx.x / kWave; p < all; p += (int64_t)gridDim.x * kNormWaves) {
        const int64_t r = pieces == 1 ? p : p / pieces, c0 = (p - r * pieces) * kNormPiece;
        const int64_t c1 = c0 + kNormPiece < cols ? c0 + kNormPiece : cols;
        const T *row = mat + r * stride;
        int64_t c = c0 + lane_id() * V;
#pragma unroll 4
        for (; c + V <= c1; c += kWave * V) {
            float z[V];
            unpack16<T>(load_a1(row + c), z);
#pragma unroll
            for (int e = 0; e < V; ++e) sum[e] += (double)z[e] * (double)z[e];
        }
        for (; c < c1; ++c) {                        // the one lane at a row's end
            const double x = (double)to_f32(row[c]);
            sum[0] += x * x;
        }
    }
#pragma unroll
    for (int e = 1; e < V; ++e) sum[0] += sum[e];
    const double total = block_total(sum[0], part);
    if (threadIdx.x == 0) reinterpret_cast<double *>(ws + blockIdx.y * ws_stride)[blockIdx.x] = total;
}

// X by rows and by columns from the update, a run of 64 x 64 tiles a workgroup.
template <typename T>
__global__ __launch_bounds__(256) void ortho_start_kernel(const T *__restrict__ g, int64_t rows, int64_t cols,
                                                          int64_t stride, int64_t batch_stride, int norm_blocks, double eps,
                                                          int run, OrthoShape s, char *ws) {
    constexpr int V = kVecOf<T>;
    __shared__ f16_t tile[kTurn][kTurn + 8];
    __shared__ double part[4];
    char *w = ws + blockIdx.z * s.bytes;
    double sum = 0.0;
    for (int k = threadIdx.x; k < norm_blocks; k += 256) sum += reinterpret_cast<const double *>(w)[k];
    const double inv = ortho_factor(block_total(sum, part), eps);
    const T *mat = g + blockIdx.z * batch_stride;
    f16_t *by_rows = (f16_t *)(w + (s.turned ? s.xt : s.x)), *by_cols = (f16_t *)(w + (s.turned ? s.x : s.xt));
    const int64_t ld_rows = s.turned ? s.mp : s.np, ld_cols = s.turned ? s.np : s.mp;
    const int64_t r0 = (int64_t)blockIdx.y * kTurn;             // in the update
    for (int k = 0; k < run; ++k) {
        const int64_t c0 = ((int64_t)blockIdx.x * run + k) * kTurn;
        if (c0 >= cols) break;
        if (k) __syncthreads();
        constexpr int kAcross = kTurn / V;
#pragma unroll
        for (int p = threadIdx.x; p < kTurn * kAcross; p += 256) {
            const int y = p / kAcross, x = p % kAcross * V;
            const int64_t r = r0 + y, c = c0 + x;
            float z[V];
            if (r < rows && c + V <= cols) {
                unpack16<T>(load_a1(mat + r * stride + c), z);
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) z[e] = r < rows && c + e < cols ? to_f32(mat[r * stride + c + e]) : 0.0f;
            }
            // the rows' ends are zeros, also where the norm is no number
#pragma unroll
            for (int e = 0; e < V; ++e) tile[y][x + e] = r < rows && c + e < cols ? (f16_t)(float)((double)z[e] * inv) : (f16_t)0.0f;
        }
        __syncthreads();
        struct alignas(16) Eight { f16_t e[8]; } v;
#pragma unroll
        for (int p = threadIdx.x; p < kTurn * kTurn / 8; p += 256) {
            const int y = p / (kTurn / 8), x = p % (kTurn / 8) * 8;
            if (r0 + y < rows && c0 + x < ld_rows) {
                v = *reinterpret_cast<const Eight *>(&tile[y][x]);
                *reinterpret_cast<Eight *>(by_rows + (r0 + y) * ld_rows + c0 + x) = v;
            }
            if (c0 + y < cols && r0 + x < ld_cols) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v.e[e] = tile[x + e][y];
                *reinterpret_cast<Eight *>(by_cols + (c0 + y) * ld_cols + r0 + x) = v;
            }
        }
    }
}

// kSquare: C = a I + b A + c A A from A, else A = X X^T: the lower tiles, each
// to both of its places. A workgroup takes a tile of one matrix of the batch, or a
// part of its steps.
template <bool kSquare, TileWork kWork, typename P>
__global__ __launch_bounds__(P::kThreads) void ortho_gram_kernel(OrthoShape s, char *ws, uint32_t side, float ca, float cb, float cc, int parts) {
    static_assert(kWork == kWhole || P::kRows == 64, "no other tile's steps are split");
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const uint32_t job = xcd_run(blockIdx.x, gridDim.x), tiles = side * (side + 1) / 2;
    const uint32_t id = kWork == kPart ? job / parts : job;
    const uint32_t mat = __builtin_amdgcn_readfirstlane((int)(id / tiles));
    char *w = ws + mat * s.bytes;
    int tm, tn;
    lower_tile_of<4>(id - mat * tiles, side, tm, tn);
    const int64_t r0 = (int64_t)tm * P::kRows, c0 = (int64_t)tn * P::kCols;
    Rows x = kSquare ? Rows{w + s.a, s.mp * 2, s.m, s.mp * 2} : Rows{w + s.x, s.np * 2, s.m, s.np * 2};
    P t;
    char *sums = ws + s.split + (int64_t)(kWork == kPart ? job : id * parts) * P::kSumBytes;
    if constexpr (kWork == kPart) x = part_of(x, job - id * parts, parts);
    if constexpr (kWork == kJoin) {
        t.add_sums(sums, parts);
    } else {
        t.run(x, r0, x, c0, lds);
        __syncthreads();                             // nobody reads the operands any more
    }
    if constexpr (kWork == kPart) {
        t.leave_sums(sums);
        return;
    }
    const f16_t *a = (const f16_t *)(w + s.a);
    f16_t *to = (f16_t *)(w + (kSquare ? s.c : s.a));
#pragma unroll
    for (int j = 0; j < P::kTN; ++j) {
        const int64_t col = c0 + P::col(j);
#pragma unroll
        for (int i = 0; i < P::kTM; ++i) {
            const int64_t row = r0 + P::row4(i);
            if (kSquare) {
                // A's elements of this column, by its row of the same number
                struct alignas(8) { f16_t e[4]; } g;
                g = *reinterpret_cast<const decltype(g) *>(a + (col < s.m ? col : 0) * s.mp + (row < s.mp ? row : 0));
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    t.acc[i][j][e] = __builtin_fmaf(cc / kScaleA, t.acc[i][j][e], cb * (float)g.e[e]) + (row + e == col ? ca * kScaleA : 0.0f);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) t.acc[i][j][e] *= kScaleA / (kScaleX * kScaleX);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (row + e >= s.m || col >= s.m) t.acc[i][j][e] = 0.0f;       // the rows' ends
        }
    }
    auto bits = [&](int i, int j) {
        const mfma_v4f v = t.acc[i][j];
        return make_uint2(pair_bits<f16_t>(v[0], v[1]), pair_bits<f16_t>(v[2], v[3]));
    };
    auto put = [&](int64_t line, int64_t at, const uint4 &v) {
        if (line < s.m && at < s.mp) *reinterpret_cast<uint4 *>(to + line * s.mp + at) = v;
    };
    if (tm != tn) P::by_columns(lds, bits, [&](int c, int r, const uint4 &v) { put(c0 + c, r0 + r, v); });
    P::by_rows(lds, bits, [&](int r, int c, const uint4 &v) { put(r0 + r, c0 + c, v); });
}

// A tile of C X, from r0 and c0 on: X by rows and by columns, or, in the last step, the result.
template <bool kLast, typename P>
__device__ __forceinline__ void store_applied(const P &t, const OrthoShape &s, char *w, int64_t r0, int64_t c0, int64_t xt_to, bf16_t *o, char *lds) {
    if constexpr (kLast) {
        constexpr float f = 1.0f / (kScaleA * kScaleX);
        auto bits = [&](int i, int j) {
            const mfma_v4f v = t.acc[i][j];
            return make_uint2(pair_bits<bf16_t>(v[0] * f, v[1] * f), pair_bits<bf16_t>(v[2] * f, v[3] * f));
        };
        // lines of `len` elements
        auto put = [&](int64_t line, int64_t lines, int64_t at, int64_t len, const uint4 &v) {
            if (line >= lines) return;
            bf16_t *to = o + line * len + at;
            if (at + 8 <= len) {
                store_a1(to, v);
            } else {
                struct { bf16_t e[8]; } y = __builtin_bit_cast(decltype(y), v);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (at + e < len) to[e] = y.e[e];
            }
        };
        if (s.turned) P::by_columns(lds, bits, [&](int cl, int r, const uint4 &v) { put(c0 + cl, s.n, r0 + r, s.m, v); });
        else P::by_rows(lds, bits, [&](int r, int cl, const uint4 &v) { put(r0 + r, s.m, c0 + cl, s.n, v); });
    } else {
        f16_t *by_rows = (f16_t *)(w + s.x), *by_cols = (f16_t *)(w + xt_to);
        auto bits = [&](int i, int j) {
            const int64_t row = r0 + P::row4(i);
            const bool in = c0 + P::col(j) < s.n;
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = in && row + e < s.m ? t.acc[i][j][e] * (1.0f / kScaleA) : 0.0f;      // the rows' ends
            return make_uint2(pair_bits<f16_t>(v[0], v[1]), pair_bits<f16_t>(v[2], v[3]));
        };
        P::by_columns(lds, bits, [&](int cl, int r, const uint4 &v) {
            if (c0 + cl < s.n && r0 + r < s.mp) *reinterpret_cast<uint4 *>(by_cols + (c0 + cl) * s.mp + r0 + r) = v;
        });
        P::by_rows(lds, bits, [&](int r, int cl, const uint4 &v) {
            if (r0 + r < s.m && c0 + cl < s.np) *reinterpret_cast<uint4 *>(by_rows + (r0 + r) * s.np + c0 + cl) = v;
        });
    }
}

// X <- C X by rows and by columns, or, in the last step, the result.
template <bool kLast, typename P>
__global__ __launch_bounds__(P::kThreads) void ortho_apply_kernel(OrthoShape s, char *ws, int64_t xt_from, int64_t xt_to, uint32_t tiles_m,
                                                                  uint32_t tiles_n, bf16_t *__restrict__ out) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const uint32_t id = xcd_run(blockIdx.x, gridDim.x);
    const uint32_t mat = __builtin_amdgcn_readfirstlane((int)(id / (tiles_m * tiles_n)));
    int tm, tn;
    tile_of<8>(id - mat * (tiles_m * tiles_n), tiles_m, tiles_n, tm, tn);
    char *w = ws + mat * s.bytes;
    const int64_t r0 = (int64_t)tm * P::kRows, c0 = (int64_t)tn * P::kCols;
    const Rows c{w + s.c, s.mp * 2, s.m, s.mp * 2}, x{w + xt_from, s.mp * 2, s.n, s.mp * 2};
    P t;
    t.run(c, r0, x, c0, lds);
    __syncthreads();                                 // nobody reads the operands any more
    store_applied<kLast>(t, s, w, r0, c0, xt_to, out + mat * s.m * s.n, lds);
}

// kRows rows of kSteps steps of a row operand on their way from memory to LDS, each
// step's rows together as TileProduct reads them; zeros for rows that it does not have.
template <int kRows, int kSteps>
struct Held {
    static constexpr int kMine = kRows / 8 * kSteps / 8;      // pieces of 8 rows by 128 bytes, for each of eight waves
    uint4 v[kMine];
    __device__ __forceinline__ void load(const Rows &m, int64_t row0) {
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int p = i * 8 + threadIdx.x / kWave, chunk = (lane_id() & 7) ^ (lane_id() >> 3);
            const int64_t row = row0 + p % (kRows / 8) * 8 + (lane_id() >> 3);
            v[i] = make_uint4(0, 0, 0, 0);
            if (row < m.rows) v[i] = *reinterpret_cast<const uint4 *>(m.p + row * m.stride + p / (kRows / 8) * kStepBytes + chunk * 16);
        }
    }
    __device__ __forceinline__ void put(char *to) const {
#pragma unroll
        for (int i = 0; i < kMine; ++i) *reinterpret_cast<uint4 *>(to + (i * 8 + threadIdx.x / kWave) * 1024 + lane_id() * 16) = v[i];
    }
};

// Where a row's element k lies in LDS, in steps of `next` bytes; four from a multiple
// of four on lie together.
__device__ __forceinline__ int held_at(int row, int k, int next) {
    return k / 64 * next + row * kStepBytes + (((k % 64 / 8) ^ (row & 7)) << 4) + (k & 7) * 2;
}
// Four columns of C's row from k on, of the square's sums and A's elements there.
__device__ __forceinline__ uint2 four_of_c(const mfma_v4f &square, const char *a, int64_t row, int k, int64_t m, float ca, float cb, float cc) {
    struct alignas(8) { f16_t e[4]; } g;
    g = *reinterpret_cast<const decltype(g) *>(a);
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
        v[e] = __builtin_fmaf(cc / kScaleA, square[e], cb * (float)g.e[e]) + (k + e == row && row < m ? ca * kScaleA : 0.0f);
    return make_uint2(pair_bits<f16_t>(v[0], v[1]), pair_bits<f16_t>(v[2], v[3]));
}

// C and C X in one launch, for updates of at most kMP rows: a workgroup forms 64 rows
// of C in LDS, from all of A, and multiplies them with kCols columns of X. The sums are
// those of the two kernels, in their order.
template <int kMP, int kCols>
struct SmallStep {
    static constexpr int kSteps = kMP / 64, kNext = kMP * kStepBytes, kNextC = 64 * kStepBytes, kNextX = kCols * kStepBytes;
    using Square = TileProduct<MulF16, kMP, 64, 4, 2, 1, 1, true>;      // columns of C, which are its rows
    using Apply = TileProduct<MulF16, 64, kCols, 2, 4, 1, 1, true>;
    static constexpr int kC = kNext * kSteps, kLds = kC + kNextC * kSteps;      // X comes where A was
    static_assert(kCols <= kMP && Apply::kTurnBytes <= kLds, "and is turned where the operands were");
};
template <bool kLast, int kMP, int kCols>
__global__ __launch_bounds__(512) void ortho_small_step_kernel(OrthoShape s, char *ws, int64_t xt_from, int64_t xt_to, uint32_t tiles_m,
                                                               uint32_t tiles_n, float ca, float cb, float cc, bf16_t *__restrict__ out) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    using S = SmallStep<kMP, kCols>;
    const uint32_t id = xcd_run(blockIdx.x, gridDim.x), mat = id / (tiles_m * tiles_n), tile = id - mat * (tiles_m * tiles_n);
    const int r0 = (int)(tile % tiles_m) * 64;
    const int64_t c0 = (int64_t)(tile / tiles_m) * kCols;
    char *w = ws + mat * s.bytes;
    Held<kMP, S::kSteps> a;
    Held<kCols, S::kSteps> x;
    a.load(Rows{w + s.a, s.mp * 2, s.m, s.mp * 2}, 0);
    x.load(Rows{w + xt_from, s.mp * 2, s.n, s.mp * 2}, c0);
    a.put(lds);
    __syncthreads();
    typename S::Square q;
    q.clear();
#pragma unroll
    for (int k = 0; k < S::kSteps; ++k) q.step(lds + k * S::kNext, lds + k * S::kNext + r0 * kStepBytes);
#pragma unroll
    for (int j = 0; j < S::Square::kTN; ++j) {
        const int to = S::Square::col(j);            // row of C, and of A, in the strip
#pragma unroll
        for (int i = 0; i < S::Square::kTM; ++i) {
            const int k = S::Square::row4(i);        // four columns of C from here on
            *reinterpret_cast<uint2 *>(lds + S::kC + held_at(to, k, S::kNextC)) =
                four_of_c(q.acc[i][j], lds + held_at(r0 + to, k, S::kNext), (int64_t)r0 + to, k, s.m, ca, cb, cc);
        }
    }
    __syncthreads();                                 // nobody reads A any more
    x.put(lds);
    __syncthreads();
    typename S::Apply t;
    t.clear();
#pragma unroll
    for (int k = 0; k < S::kSteps; ++k) t.step(lds + S::kC + k * S::kNextC, lds + k * S::kNextX);
    __syncthreads();                                 // nobody reads the operands any more
    store_applied<kLast>(t, s, w, r0, c0, xt_to, out + mat * s.m * s.n, lds);
}

// Whole updates in LDS, one a workgroup, for the smallest: X by rows and by columns
// and A, then C in its place. Products and sums are those of the other kernels.
template <typename T, int kMP>
__global__ __launch_bounds__(512) void ortho_whole_kernel(const T *__restrict__ g, int rows, int cols, int64_t stride, int64_t batch_stride,
                                                          double eps, int steps, float ca, float cb, float cc, OrthoShape s,
                                                          bf16_t *__restrict__ out) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    constexpr int V = kVecOf<T>, kHold = 64 / V;     // 512 threads hold kMP x np elements, of which there are at most 2^15
    constexpr int kNextX = kMP * kStepBytes, kNextA = kNextX;
    const int np = (int)s.np, m = (int)s.m, next_t = np * kStepBytes;
    char *x = lds, *xt = lds + kMP * np * 2, *a = xt + kMP * np * 2;
    double *part = reinterpret_cast<double *>(a);     // before there is an A
    const T *mat = g + blockIdx.x * batch_stride;
    // The update, in vectors of its rows, and its norm.
    const uint32_t across = (cols + V - 1) / V, all = rows * across;
    uint4 held[kHold];
    double sum = 0.0;
#pragma unroll
    for (int k = 0; k < kHold; ++k) {
        const uint32_t at = k * 512 + threadIdx.x, r = at / across, c = (at - r * across) * V;
        held[k] = make_uint4(0, 0, 0, 0);
        if (at < all) {
            const T *from = mat + r * stride + c;
            if (c + V <= (uint32_t)cols) {
                held[k] = load_a1(from);
            } else {
                struct { T e[V]; } w = __builtin_bit_cast(decltype(w), held[k]);
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (c + e < (uint32_t)cols) w.e[e] = from[e];
                held[k] = __builtin_bit_cast(uint4, w);
            }
        }
    }
#pragma unroll
    for (int k = 0; k < kHold; ++k) {
        float z[V];
        unpack16<T>(held[k], z);
#pragma unroll
        for (int e = 0; e < V; ++e) sum += (double)z[e] * (double)z[e];
    }
#pragma unroll
    for (int off = kWave / 2; off >= 1; off >>= 1) sum += __shfl_xor(sum, off, kWave);
    if (lane_id() == 0) part[threadIdx.x / kWave] = sum;
    // The update's own order first, with zeros at the lines' ends and behind them; the
    // other one is read from it, by lanes on neighbouring lines.
    char *own = s.turned ? xt : x, *other = s.turned ? x : xt;
    const int lines = s.turned ? np : kMP, len = s.turned ? kMP : np, next_own = lines * kStepBytes, next_other = len * kStepBytes;
    for (int k = threadIdx.x; k < kMP * np * 2 / 16; k += 512) reinterpret_cast<uint4 *>(own)[k] = make_uint4(0, 0, 0, 0);
    __syncthreads();
    const double inv = ortho_factor(((part[0] + part[1]) + (part[2] + part[3])) + ((part[4] + part[5]) + (part[6] + part[7])), eps);
#pragma unroll
    for (int k = 0; k < kHold; ++k) {
        const uint32_t at = k * 512 + threadIdx.x, r = at / across, c = (at - r * across) * V;
        if (at >= all) continue;
        float z[V];
        unpack16<T>(held[k], z);
        struct alignas(2 * V) { f16_t e[V]; } y;
#pragma unroll
        for (int e = 0; e < V; ++e) y.e[e] = c + e < (uint32_t)cols ? (f16_t)(float)((double)z[e] * inv) : (f16_t)0.0f;
        *reinterpret_cast<decltype(y) *>(own + held_at(r, c, next_own)) = y;
    }
    __syncthreads();
    for (int p = threadIdx.x; p < len * lines / 8; p += 512) {
        const int line = p % len, at = p / len * 8;
        struct alignas(16) { uint16_t e[8]; } y;
#pragma unroll
        for (int e = 0; e < 8; ++e) y.e[e] = *reinterpret_cast<const uint16_t *>(own + held_at(at + e, line, next_own));
        *reinterpret_cast<decltype(y) *>(other + held_at(line, at, next_other)) = y;
    }
    constexpr int kWM = kMP == 64 ? 4 : 2, kWN = 8 / kWM, kSteps = kMP / 64;
    using Square = TileProduct<MulF16, kMP, kMP, kWM, kWN, 1, 1, true>;
    constexpr int kCols = kMP / 4, kTM = kMP / 16, kTN = kCols / 16;      // of X a wave at a time
    const int wave = threadIdx.x / kWave, lane = lane_id();
    for (int step = 0; step < steps; ++step) {
        const bool last = step + 1 == steps;
        __syncthreads();
        Square q;
        q.clear();
#pragma unroll 2
        for (int k = 0; k < np / 64; ++k) q.step(x + k * kNextX, x + k * kNextX);
#pragma unroll
        for (int j = 0; j < Square::kTN; ++j)
#pragma unroll
            for (int i = 0; i < Square::kTM; ++i) {
                const mfma_v4f v = q.acc[i][j] * (kScaleA / (kScaleX * kScaleX));
                *reinterpret_cast<uint2 *>(a + held_at(Square::col(j), Square::row4(i), kNextA)) = make_uint2(pair_bits<f16_t>(v[0], v[1]), pair_bits<f16_t>(v[2], v[3]));
            }
        __syncthreads();
        q.clear();
#pragma unroll
        for (int k = 0; k < kSteps; ++k) q.step(a + k * kNextA, a + k * kNextA);
        __syncthreads();                             // nobody reads A any more but in its own places
#pragma unroll
        for (int j = 0; j < Square::kTN; ++j)
#pragma unroll
            for (int i = 0; i < Square::kTM; ++i) {
                char *at = a + held_at(Square::col(j), Square::row4(i), kNextA);
                *reinterpret_cast<uint2 *>(at) = four_of_c(q.acc[i][j], at, Square::col(j), Square::row4(i), m, ca, cb, cc);
            }
        __syncthreads();
        // C X: a wave takes columns of X, which no other reads, and writes them where they were
        for (int c0 = wave * kCols; c0 < np; c0 += 8 * kCols) {
            mfma_v4f y[kTM][kTN];
#pragma unroll
            for (int i = 0; i < kTM; ++i)
#pragma unroll
                for (int j = 0; j < kTN; ++j) y[i][j] = mfma_v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int k = 0; k < 2 * kSteps; ++k) {
                const int at = (lane & 15) * kStepBytes + (((4 * (k % 2) + (lane >> 4)) ^ (lane & 7)) << 4);
                mfma_v4i b[kTN];
#pragma unroll
                for (int j = 0; j < kTN; ++j) b[j] = *reinterpret_cast<const mfma_v4i *>(xt + k / 2 * next_t + (c0 + j * 16) * kStepBytes + at);
#pragma unroll
                for (int i = 0; i < kTM; ++i) {
                    const mfma_v4i f = *reinterpret_cast<const mfma_v4i *>(a + k / 2 * kNextA + i * 16 * kStepBytes + at);
#pragma unroll
                    for (int j = 0; j < kTN; ++j) y[i][j] = MulF16::mul(f, b[j], y[i][j]);
                }
            }
#pragma unroll
            for (int j = 0; j < kTN; ++j)
#pragma unroll
                for (int i = 0; i < kTM; ++i) {
                    const int col = c0 + j * 16 + (lane & 15), row = i * 16 + (lane >> 4) * 4;
                    uint2 w;
                    if (last) {
                        const mfma_v4f v = y[i][j] * (1.0f / (kScaleA * kScaleX));
                        w = make_uint2(pair_bits<bf16_t>(v[0], v[1]), pair_bits<bf16_t>(v[2], v[3]));
                    } else {
                        const mfma_v4f v = y[i][j] * (1.0f / kScaleA);
                        w = make_uint2(pair_bits<f16_t>(v[0], v[1]), pair_bits<f16_t>(v[2], v[3]));
                    }
                    if (!last || s.turned) *reinterpret_cast<uint2 *>(xt + held_at(col, row, next_t)) = w;
                    if (!last || !s.turned) {
                        // lanes on neighbouring columns exchange two of their rows
                        const bool odd = lane & 1;
                        const uint32_t got = dpp_u32<0xb1, 0xf>(0u, odd ? w.x : w.y), l = odd ? got : w.x, r = odd ? w.y : got;
                        const int to = row + (odd ? 2 : 0), pair = col - (odd ? 1 : 0);
                        *reinterpret_cast<uint32_t *>(x + held_at(to, pair, kNextX)) = (l & 0xffffu) | (r << 16);
                        *reinterpret_cast<uint32_t *>(x + held_at(to + 1, pair, kNextX)) = (l >> 16) | (r & 0xffff0000u);
                    }
                }
        }
    }
    __syncthreads();
    // the result's lines, in pieces of eight
    const int pieces = (cols + 7) / 8;
    bf16_t *o = out + blockIdx.x * s.m * s.n;
    for (int p = threadIdx.x; p < rows * pieces; p += 512) {
        const int line = p / pieces, at = (p - line * pieces) * 8;
        const uint4 v = *reinterpret_cast<const uint4 *>(own + held_at(line, at, next_own));
        bf16_t *to = o + line * cols + at;
        if (at + 8 <= cols) {
            store_a1(to, v);
        } else {
            struct { bf16_t e[8]; } w = __builtin_bit_cast(decltype(w), v);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (at + e < cols) to[e] = w.e[e];
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

template <typename P>
constexpr int ortho_lds() {
    return P::kLdsBytes > P::kTurnBytes ? P::kLdsBytes : P::kTurnBytes;
}

template <bool kSquare>
hipError_t launch_gram(const OrthoShape &s, char *ws, int64_t batch, const float *c, hipStream_t stream) {
    auto tiles = [&](int64_t side) {
        const int64_t t = (s.m + side - 1) / side;
        return t * (t + 1) / 2 * batch;
    };
    const int64_t cus = resident_waves() / 16;
    int side = product_tile((kSquare ? s.mp : s.np) * 2 / kStepBytes, cus, tiles);
    auto go = [&](auto kernel, auto p, int64_t jobs, int parts) {
        using P = decltype(p);
        return launch_lds(-1, kernel, dim3((unsigned)jobs), dim3(P::kThreads), ortho_lds<P>(), stream, s, ws, (s.m + side - 1) / side, c[0], c[1], c[2], parts);
    };
    if constexpr (!kSquare) {
        if (s.split) {
            side = 64;
            const int parts = product_parts(s.np / 64, tiles(64));
            return with_tile_of_64(tiles(64) * parts, cus, [&](auto shape) {
                using P = typename decltype(shape)::template Product<MulF16>;
                const hipError_t e = go(ortho_gram_kernel<false, kPart, P>, P{}, tiles(64) * parts, parts);
                return e == hipSuccess ? go(ortho_gram_kernel<false, kJoin, P>, P{}, tiles(64), parts) : e;
            });
        }
    }
    return with_tile(side, tiles(side), cus, [&](auto shape) {
        using P = typename decltype(shape)::template Product<MulF16>;
        return go(ortho_gram_kernel<kSquare, kWhole, P>, P{}, tiles(side), 1);
    });
}
template <bool kLast>
hipError_t launch_apply(const OrthoShape &s, char *ws, int64_t batch, int64_t from, int64_t to, bf16_t *out, hipStream_t stream) {
    auto tiles = [&](int64_t side) { return ((s.m + side - 1) / side) * ((s.n + side - 1) / side) * batch; };
    const int64_t cus = resident_waves() / 16;
    const int side = product_tile(s.mp * 2 / kStepBytes, cus, tiles);
    return with_tile(side, tiles(side), cus, [&](auto shape) {
        using P = typename decltype(shape)::template Product<MulF16>;
        return launch_lds(kPhaseAux, ortho_apply_kernel<kLast, P>, dim3((unsigned)tiles(side)), dim3(P::kThreads), ortho_lds<P>(), stream, s, ws,
                          from, to, (s.m + side - 1) / side, (s.n + side - 1) / side, out);
    });
}

template <bool kLast>
hipError_t launch_small(const OrthoShape &s, char *ws, int64_t batch, int cols, int64_t from, int64_t to, const float *c, bf16_t *out, hipStream_t stream) {
    auto go = [&](auto kernel, auto shape) {
        const int64_t tiles_m = s.mp / 64, tiles_n = (s.n + cols - 1) / cols;
        return launch_lds(kPhaseAux, kernel, dim3((unsigned)(tiles_m * tiles_n * batch)), dim3(512), decltype(shape)::kLds, stream, s, ws, from, to,
                          tiles_m, tiles_n, c[0], c[1], c[2], out);
    };
    if (s.mp == 64) return go(ortho_small_step_kernel<kLast, 64, 64>, SmallStep<64, 64>{});
    if (s.mp == 128) return go(ortho_small_step_kernel<kLast, 128, 64>, SmallStep<128, 64>{});
    if (s.mp == 192) return cols == 64 ? go(ortho_small_step_kernel<kLast, 192, 64>, SmallStep<192, 64>{}) : go(ortho_small_step_kernel<kLast, 192, 128>, SmallStep<192, 128>{});
    return cols == 64 ? go(ortho_small_step_kernel<kLast, 256, 64>, SmallStep<256, 64>{}) : go(ortho_small_step_kernel<kLast, 256, 128>, SmallStep<256, 128>{});
}

hipError_t ortho_steps(const OrthoShape &s, char *ws, int64_t batch, int steps, const float *coefs, bf16_t *out, hipStream_t stream) {
    int64_t from = s.xt, to = s.xt2;
    const int cols = ortho_step_cols(s.mp, s.n, batch, resident_waves() / 16);
    hipError_t e = hipSuccess;
    for (int k = 0; k < steps && e == hipSuccess; ++k) {
        e = launch_gram<false>(s, ws, batch, coefs, stream);
        const bool last = k + 1 == steps;
        if (e == hipSuccess && cols) {
            e = last ? launch_small<true>(s, ws, batch, cols, from, to, coefs, out, stream) : launch_small<false>(s, ws, batch, cols, from, to, coefs, out, stream);
        } else {
            if (e == hipSuccess) e = launch_gram<true>(s, ws, batch, coefs, stream);
            if (e == hipSuccess) e = last ? launch_apply<true>(s, ws, batch, from, to, out, stream) : launch_apply<false>(s, ws, batch, from, to, out, stream);
        }
        const int64_t x = from;
        from = to;
        to = x;
    }
    return e;
}

// As many updates as one launch of each product takes.
hipError_t orthogonalize_some(const void *g, int dtype, int64_t batch, int64_t rows, int64_t cols, int64_t stride, int64_t batch_stride,
                              int steps, const double *coefs, double eps, void *out, void *ws, hipStream_t stream) {
    OrthoShape s = ortho_shape(rows, cols);
    if (ortho_split_bytes(s, batch)) s.split = batch * s.bytes;
    if (steps > 0 && ortho_whole(s.mp, s.np))
        return with_elem(dtype, [&](auto tag) {
            using T = decltype(tag);
            auto go = [&](auto kernel) {
                return launch_lds(kPhaseAux, kernel, dim3((unsigned)batch), dim3(512), (size_t)(4 * s.mp * s.np + 2 * s.mp * s.mp), stream, (const T *)g, rows,
                                  cols, stride, batch_stride, eps, steps, (float)coefs[0], (float)coefs[1], (float)coefs[2], s, (bf16_t *)out);
            };
            return s.mp == 64 ? go(ortho_whole_kernel<T, 64>) : go(ortho_whole_kernel<T, 128>);
        });
    const int blocks = ortho_norm_blocks(rows, cols);
    char *w = (char *)ws;
    hipError_t e = with_elem(dtype, [&](auto tag) {
        using T = decltype(tag);
        hipError_t r = launch(-1, ortho_norm_kernel<T>, dim3((unsigned)blocks, (unsigned)batch), dim3(kNormWaves * kWave), stream, (const T *)g, rows,
                              cols, stride, batch_stride, w, s.bytes);
        const int64_t across = (cols + kTurn - 1) / kTurn, down = (rows + kTurn - 1) / kTurn;
        const int run = across * down * batch >= kTurnMany ? kTurnRun : 1;
        if (r == hipSuccess)
            r = launch(-1, ortho_start_kernel<T>, dim3((unsigned)((across + run - 1) / run), (unsigned)down, (unsigned)batch), dim3(256), stream,
                       (const T *)g, rows, cols, stride, batch_stride, blocks, eps, run, s, w);
        return r;
    });
    if (e != hipSuccess) return e;
    if (steps == 0)
        return launch(-1, ortho_copy_kernel, dim3((unsigned)(rows < 1024 ? rows : 1024), (unsigned)batch), dim3(256), stream, s, w, (bf16_t *)out);
    const float c[3] = {(float)coefs[0], (float)coefs[1], (float)coefs[2]};
    return ortho_steps(s, w, batch, steps, c, (bf16_t *)out, stream);
}

}  // namespace

size_t ortho_ws_bytes(int64_t batch, int64_t rows, int64_t cols) {
    const OrthoShape s = ortho_shape(rows, cols);
    return (size_t)(batch * s.bytes) + ortho_split_bytes(s, batch) + 256;
}
size_t ortho_ws_most(int64_t batch, int64_t rows, int64_t cols) {
    const OrthoShape s = ortho_shape(rows, cols);
    const int64_t t = (s.m + 63) / 64;
    return (size_t)(batch * s.bytes) + (size_t)product_jobs_most(s.np / 64, t * (t + 1) / 2 * batch) * 64 * 64 * sizeof(float) + 256;
}

hipError_t launch_orthogonalize(const void *g, int dtype, int64_t batch, int64_t rows, int64_t cols, int64_t stride,
                                int64_t batch_stride, int steps, const double *coefs, double eps, void *out, void *ws,
                                hipStream_t stream) {
    const int64_t most = ortho_batch_most(rows, cols);
    hipError_t e = hipSuccess;
    // Runs of the batch one after another, in the same workspace.
    for (int64_t k = 0; k < batch && e == hipSuccess; k += most)
        e = orthogonalize_some((const char *)g + k * batch_stride * elem_bytes_of(dtype), dtype, batch - k < most ? batch - k : most, rows, cols,
                               stride, batch_stride, steps, coefs, eps, (bf16_t *)out + k * rows * cols, ws, stream);
    return e;
}

}  // namespace pace
