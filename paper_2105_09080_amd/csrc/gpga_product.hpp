// Products of matrices on the matrix units, for the operators whose parameters are matrices: C(i,j) = sum over k of A(i,k) B(j,k),
// one product a batch entry (a node, or a matrix of a node), fp32 sums, the rest of the operator at the tile's end.
//
// Operands are fp16, times powers of two that keep them below 2^15: a value v is one half (11 bits) or the sum of two, hi + lo (22
// bits), in two planes.  One plane each costs one matrix instruction a step, two against one two, two against two three: hi hi, lo hi
// and hi lo; what lo lo would add is below 2^-22 of a term.  That is fp32's precision at three of fp16's 2.5 PFLOP/s, where the fp32
// instructions reach 157 TFLOP/s; bf16 pieces would need six products for it, and two for what one of fp16 holds.
//
// An operand lies in memory with k along its rows ("rows") or down its columns ("columns": row k holds the i's); planes have rows and
// columns padded with zeros to multiples of kPad, so k needs no checks.  Tiles go to LDS by loads that bypass the registers, 16 bytes
// a lane, two buffers: where both operands are rows, the next tile arrives while this one is multiplied.  Where one is columns it does not: the
// compiler takes the transposing read to meet any such load and waits for the tile just asked for before it reads this one, so
// there only the other workgroups of a compute unit hide that wait.  Rows of a "rows" tile are read as they are (ds_read_b128,
// 8 k's of one i); of a "columns" tile through the transposing read (ds_read_b64_tr_b16, 16 lanes fetch 4 rows of 16 and get a column of
// 4 each).  LDS gets 16-byte pieces in an order xored with the row, by loading them so, and no two lanes that are served together
// meet in a bank.
#pragma once

#include "gpga_internal.hpp"
#include "gpga_spans.hpp"

typedef _Float16 half_t;
typedef half_t half4 __attribute__((ext_vector_type(4)));
typedef half_t half8 __attribute__((ext_vector_type(8)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef float acc16 __attribute__((ext_vector_type(16)));

constexpr int kPad = 64;
template <typename I>
__host__ __device__ constexpr I padded(I v) {
    return (v + kPad - 1) / kPad * kPad;
}

struct Operand {
    const half_t* p;   // first plane of batch entry 0
    int64_t plane;     // halves from a plane to the next
    int64_t batch;     // halves from a batch entry to the next
    int32_t ld;        // halves of a row, padded
    int32_t rows;      // rows of memory, padded
};

// WM x WN wavefronts share a tile's rows and columns, KW such groups the terms of a step.
template <int kBM, int kBN, int kWM, int kWN, int kBK, int kPA, int kPB, bool kColsA, bool kColsB, int kKW = 1, bool kFull = false>
struct Tile {
    static constexpr int BM = kBM, BN = kBN, WM = kWM, WN = kWN, BK = kBK, PA = kPA, PB = kPB, KW = kKW;
    static constexpr bool ColsA = kColsA, ColsB = kColsB;
    static constexpr bool Full = kFull;  // lo lo too
    static constexpr int Waves = WM * WN, Threads = Waves * KW * kWave;
    static constexpr int MI = BM / WM / 32, NI = BN / WN / 32;             // 32 x 32 blocks of a wavefront
    static constexpr int BytesA = BM * BK * 2, BytesB = BN * BK * 2;       // of a plane
    static constexpr int Stage = PA * BytesA + PB * BytesB;
    static_assert(kPad % BK == 0 && Stage * 2 <= 160 * 1024, "tile");
};

namespace product {

typedef __attribute__((address_space(1))) const void gvoid;
typedef __attribute__((address_space(3))) void lvoid;

// Where a piece of 16 bytes lies within its row of a tile: the banks of LDS repeat after 256 bytes, and 16 lanes that read pieces of
// 16 rows (or 32 that read 8 bytes each of 4 rows of 64) meet all of them once.
template <int R, int BK, bool Cols>
__device__ __forceinline__ int piece_slot(int row, int piece) {
    if constexpr (!Cols) return piece ^ (BK == 64 ? (row >> 1) & 7 : (row >> 2) & 3);
    else return piece ^ (R >= 128 ? (row & 3) << 2 : (row & 2) << 1);
}

// Offset in bytes, from the tile's first row (or column) at k = 0, of the piece that lane `t` loads in round r.
template <int R, int BK, bool Cols, int Threads>
__device__ __forceinline__ uint32_t piece_offset(int t, int r, uint32_t ld, int32_t left) {
    constexpr int C = (Cols ? R : BK) / 8;
    const int q = r * Threads + t, row = q / C, piece = piece_slot<R, BK, Cols>(row, q % C);
    if constexpr (!Cols) return (uint32_t)(row < left ? row : left - 1) * (ld * 2) + (uint32_t)piece * 16;
    else return (uint32_t)row * (ld * 2) + (uint32_t)(piece * 8 < left ? piece * 8 : left - 8) * 2;
}

// Where a lane's fragments begin within a plane's tile.  rows: for each 16 k's; columns: for each 32 i's.  Of KW groups of wavefronts each
// takes every KW-th 16 k's.
template <int R, int BK, bool Cols, int Blocks, int KW>
struct Reader {
    static constexpr int N = Cols ? Blocks : BK / 16 / KW;
    uint32_t at[N];
    __device__ __forceinline__ Reader(int lane, int first, int group) {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            if constexpr (!Cols) {
                const int row = lane & 31;
                at[n] = (uint32_t)((first + row) * BK * 2 + piece_slot<R, BK, false>(row, (n * KW + group) * 2 + (lane >> 5)) * 16);
            } else {
                const int g = lane >> 4, i = lane & 15, k = (g >> 1) * 8 + i / 4;
                at[n] = (uint32_t)((group * 16 + k) * R * 2 + piece_slot<R, BK, true>(k, (first + n * 32) / 8 + (g & 1) * 2 + (i % 4) / 2) * 16 + (i & 1) * 8);
            }
        }
    }
    // i's first + 32 * block .., the group's n-th 16 k's of the tile at `lds`; first is a multiple of 32.
    __device__ __forceinline__ half8 read(const char* lds, int block, int n) const {
        if constexpr (!Cols) {
            return *reinterpret_cast<const half8*>(lds + at[n] + block * 32 * BK * 2);
        } else {
            typedef __attribute__((address_space(3))) short4v lshort;
            const char* from = lds + at[block] + n * KW * 16 * R * 2;
            const half4 a = __builtin_bit_cast(half4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lshort*)(from)));
            const half4 b = __builtin_bit_cast(half4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lshort*)(from + 4 * R * 2)));
            return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
};

}  // namespace product

// The tile of rows m0 .., columns n0 .. of one batch entry, K (a multiple of kPad) terms: acc[block of 32 columns][block of 32
// rows], in which lane l holds row l % 32 and columns 8 (r / 4) + 4 (l / 32) + r % 4.
// `row_b(row)`: row of B's memory that holds column n0 + row (rows operands only).  `middle(row)`, if there is one: what the sum over the first half of
// the terms is multiplied by, for halves of two scales (K a multiple of 2 kPad then).  `under_way()` runs while the first tiles arrive.
struct NoMiddle {};
struct Nothing {
    __device__ __forceinline__ void operator()() const {}
};
template <typename S, typename RowB, typename Middle = NoMiddle, typename UnderWay = Nothing>
__device__ __forceinline__ void product_tile(const Operand& A, const Operand& B, int64_t batch, int32_t m0, int32_t n0, int32_t K, char* lds,
                                             acc16 (&acc)[S::NI][S::MI], RowB&& row_b, Middle&& middle = {}, UnderWay&& under_way = {}) {
    constexpr bool kMiddle = !__is_same(__remove_cvref(Middle), NoMiddle);
    using namespace product;
    const int t = threadIdx.x, lane = t & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(t / kWave);
    constexpr int RA = S::BytesA / 16 / S::Threads, RB = S::BytesB / 16 / S::Threads;
    static_assert(RA * S::Threads * 16 == S::BytesA && RB * S::Threads * 16 == S::BytesB, "whole rounds");

    const char* a = reinterpret_cast<const char*>(A.p + batch * A.batch + (S::ColsA ? (int64_t)m0 : (int64_t)m0 * A.ld));
    const char* b = reinterpret_cast<const char*>(B.p + batch * B.batch + (S::ColsB ? (int64_t)n0 : 0));
    const int64_t stepA = S::ColsA ? (int64_t)S::BK * A.ld * 2 : S::BK * 2, stepB = S::ColsB ? (int64_t)S::BK * B.ld * 2 : S::BK * 2;
    uint32_t fromA[RA], fromB[RB];
#pragma unroll
    for (int r = 0; r < RA; ++r)
        fromA[r] = piece_offset<S::BM, S::BK, S::ColsA, S::Threads>(t, r, (uint32_t)A.ld, (S::ColsA ? A.ld : A.rows) - m0);
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        if constexpr (S::ColsB) {
            fromB[r] = piece_offset<S::BN, S::BK, true, S::Threads>(t, r, (uint32_t)B.ld, B.ld - n0);
        } else {
            constexpr int C = S::BK / 8;
            const int q = r * S::Threads + t, row = q / C;
            const uint32_t inner = piece_offset<S::BN, S::BK, false, S::Threads>(t, r, 0u, S::BN);
            fromB[r] = (uint32_t)row_b(row) * ((uint32_t)B.ld * 2) + inner;
        }
    }
    auto fetch = [&](int stage) {
        char* to = lds + stage * S::Stage + wave * (kWave * 16);
#pragma unroll
        for (int p = 0; p < S::PA; ++p)
#pragma unroll
            for (int r = 0; r < RA; ++r)
                __builtin_amdgcn_global_load_lds((gvoid*)(a + p * A.plane * 2 + fromA[r]),
                                                 (lvoid*)(to + p * S::BytesA + r * S::Threads * 16), 16, 0, 0);
#pragma unroll
        for (int p = 0; p < S::PB; ++p)
#pragma unroll
            for (int r = 0; r < RB; ++r)
                __builtin_amdgcn_global_load_lds((gvoid*)(b + p * B.plane * 2 + fromB[r]),
                                                 (lvoid*)(to + S::PA * S::BytesA + p * S::BytesB + r * S::Threads * 16), 16, 0, 0);
        a += stepA;
        b += stepB;
    };
    const int group = wave / S::Waves;
    const int firstA = wave % S::Waves / S::WN * (S::BM / S::WM), firstB = wave % S::WN * (S::BN / S::WN);
    const Reader<S::BM, S::BK, S::ColsA, S::MI, S::KW> ra(lane, firstA, group);
    const Reader<S::BN, S::BK, S::ColsB, S::NI, S::KW> rb(lane, firstB, group);
#pragma unroll
    for (int j = 0; j < S::NI; ++j)
#pragma unroll
        for (int i = 0; i < S::MI; ++i) acc[j][i] = acc16{};

    float factor[kMiddle ? S::MI : 1];
    if constexpr (kMiddle) {
#pragma unroll
        for (int i = 0; i < S::MI; ++i) factor[i] = middle(m0 + firstA + i * 32 + (lane & 31));
    }
    const int steps = K / S::BK;
    fetch(0);
    under_way();
    __syncthreads();
    for (int s = 0; s < steps; ++s) {
        if (s + 1 < steps) fetch((s + 1) & 1);
        if constexpr (kMiddle) {
            if (s == steps / 2) {
#pragma unroll
                for (int j = 0; j < S::NI; ++j)
#pragma unroll
                    for (int i = 0; i < S::MI; ++i) acc[j][i] *= factor[i];
            }
        }
        const char* at = lds + (s & 1) * S::Stage;
#pragma unroll
        for (int kk = 0; kk < S::BK / 16 / S::KW; ++kk) {
            half8 fa[S::PA][S::MI], fb[S::PB][S::NI];
#pragma unroll
            for (int p = 0; p < S::PA; ++p)
#pragma unroll
                for (int i = 0; i < S::MI; ++i) fa[p][i] = ra.read(at + p * S::BytesA, i, kk);
#pragma unroll
            for (int p = 0; p < S::PB; ++p)
#pragma unroll
                for (int j = 0; j < S::NI; ++j) fb[p][j] = rb.read(at + S::PA * S::BytesA + p * S::BytesB, j, kk);
#pragma unroll
            for (int pa = 0; pa < S::PA; ++pa)
#pragma unroll
                for (int pb = 0; pb < S::PB; ++pb) {
                    if (pa + pb == 2 && !S::Full) continue;
#pragma unroll
                    for (int j = 0; j < S::NI; ++j)
#pragma unroll
                        for (int i = 0; i < S::MI; ++i)
                            acc[j][i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fb[pb][j], fa[pa][i], acc[j][i], 0, 0, 0);
                }
        }
        __syncthreads();
    }
    if constexpr (S::KW > 1) {  // the first group adds the others' sums, in their order
        float* mine = reinterpret_cast<float*>(lds) + (wave - S::Waves) * (S::NI * S::MI * 16 * kWave) + lane;
        static_assert((S::KW - 1) * S::Waves * S::NI * S::MI * 16 * kWave * 4 <= 2 * S::Stage, "sums");
        if (group > 0) {
#pragma unroll
            for (int j = 0; j < S::NI; ++j)
#pragma unroll
                for (int i = 0; i < S::MI; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) mine[((j * S::MI + i) * 16 + r) * kWave] = acc[j][i][r];
        }
        __syncthreads();
        if (group == 0) {
#pragma unroll
            for (int g = 1; g < S::KW; ++g)
#pragma unroll
                for (int j = 0; j < S::NI; ++j)
#pragma unroll
                    for (int i = 0; i < S::MI; ++i)
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            acc[j][i][r] += mine[(g * S::Waves * S::NI * S::MI * 16 + (j * S::MI + i) * 16 + r) * kWave];
        }
        __syncthreads();
    }
}

// A tile's accumulators by rows: a wavefront leaves 32 rows of its 64 columns at a time in LDS, which the operands no longer need, and
// every lane takes eight columns of a row from there, so that eight lanes read and write whole lines of memory.  As they come from the
// matrix unit a lane's columns are 16 bytes apart in 32 rows.
template <typename S>
struct Dump {
    static constexpr int kCols = S::NI * 32, kRow = kCols + 4, kWaveFloats = 32 * kRow;  // rows begin 4 banks apart
    static_assert(S::NI == 2 && S::Waves * kWaveFloats * 4 <= 2 * S::Stage, "dump");
    float* own;
    __device__ __forceinline__ explicit Dump(char* lds) : own(reinterpret_cast<float*>(lds) + threadIdx.x / kWave * kWaveFloats) {}
    __device__ __forceinline__ void put(const acc16 (&acc)[S::NI][S::MI], int i) const {
        const int lane = threadIdx.x & (kWave - 1);
        float* row = own + (lane & 31) * kRow + (lane >> 5) * 4;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int j = 0; j < S::NI; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<v4f*>(row + j * 32 + q * 8) =
                    v4f{acc[j][i][q * 4], acc[j][i][q * 4 + 1], acc[j][i][q * 4 + 2], acc[j][i][q * 4 + 3]};
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    __device__ __forceinline__ void get(int row, int col, float* v) const {
        const v4f a = *reinterpret_cast<const v4f*>(own + row * kRow + col), b = *reinterpret_cast<const v4f*>(own + row * kRow + col + 4);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = a[k], v[4 + k] = b[k];
    }
};
template <typename S>
__device__ __forceinline__ int32_t wave_row(int32_t m0) {
    return m0 + (int32_t)(threadIdx.x / kWave) / S::WN * (S::BM / S::WM);
}
template <typename S>
__device__ __forceinline__ int32_t wave_col(int32_t n0) {
    return n0 + (int32_t)(threadIdx.x / kWave) % S::WN * (S::BN / S::WN);
}

// f(row, column, eight columns' values) for a tile; with `mirror` then f(column, row, eight rows' values) too.
template <typename S, typename F>
__device__ __forceinline__ void each_octet(const acc16 (&acc)[S::NI][S::MI], char* lds, int32_t m0, int32_t n0, bool mirror, F&& f) {
    if ((int)threadIdx.x >= S::Waves * kWave) return;  // the first group of wavefronts has the sums
    const Dump<S> dump(lds);
    const int lane = threadIdx.x & (kWave - 1);
    const int32_t row0 = wave_row<S>(m0), col0 = wave_col<S>(n0);
#pragma unroll
    for (int i = 0; i < S::MI; ++i) {
        dump.put(acc, i);
#pragma unroll
        for (int it = 0; it < 4; ++it) {
            const int row = it * 8 + lane / 8, col = lane % 8 * 8;
            float v[8];
            dump.get(row, col, v);
            f(row0 + i * 32 + row, col0 + col, v);
        }
        if (mirror) {
#pragma unroll
            for (int it = 0; it < 4; ++it) {
                float v[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = dump.own[(it * 8 + k) * Dump<S>::kRow + lane];
                f(col0 + lane, row0 + i * 32 + it * 8, v);
            }
        }
    }
}

// f(row, column, eight values of the wavefront's first 32 columns, the same of its second 32), column counted in the first.
template <typename S, typename F>
__device__ __forceinline__ void each_octet_pair(const acc16 (&acc)[S::NI][S::MI], char* lds, int32_t m0, F&& f) {
    if ((int)threadIdx.x >= S::Waves * kWave) return;  // the first group of wavefronts has the sums
    const Dump<S> dump(lds);
    const int lane = threadIdx.x & (kWave - 1);
#pragma unroll
    for (int i = 0; i < S::MI; ++i) {
        dump.put(acc, i);
#pragma unroll
        for (int it = 0; it < 2; ++it) {
            const int row = it * 16 + lane / 4, col = lane % 4 * 8;
            float a[8], b[8];
            dump.get(row, col, a);
            dump.get(row, col + 32, b);
            f(wave_row<S>(m0) + i * 32 + row, col, a, b);
        }
    }
}

// Which tile a workgroup takes: the tiles of a batch entry stay on one XCD as far as they go (workgroups go round the eight by their
// number), and there in groups of kGroup rows of tiles, so that the ones under way together share rows and columns in its L2.
struct TileGrid {
    int32_t tm, tn;    // tiles of a batch entry; tn = 0: only those on and below the diagonal of a square of tm
    uint32_t total;    // of all
    __host__ void set(int32_t rows, int32_t cols, int32_t side, int32_t batch, bool lower) {
        tm = (rows + side - 1) / side;
        tn = lower ? 0 : (cols + side - 1) / side;
        total = (uint32_t)one() * (uint32_t)batch;
    }
    __host__ __device__ int32_t one() const { return tn ? tm * tn : tm * (tm + 1) / 2; }
    static constexpr uint32_t kXcds = 8;
    static constexpr int32_t kGroup = 8;
    __host__ __device__ uint32_t blocks() const { return (total + kXcds - 1) / kXcds * kXcds; }
    // false: none is left for this workgroup
    __device__ __forceinline__ bool at(uint32_t block, int32_t* batch, int32_t* i, int32_t* j) const {
        const uint32_t per = (total + kXcds - 1) / kXcds, id = block % kXcds * per + block / kXcds;
        if (id >= total) return false;
        const uint32_t each = (uint32_t)one();
        *batch = (int32_t)(id / each);
        const int32_t in = (int32_t)(id % each);
        if (tn == 0) {  // row i begins at i (i + 1) / 2
            int32_t row = (int32_t)((sqrtf(8.f * (float)in + 1.f) - 1.f) * 0.5f);
            while (row * (row + 1) / 2 > in) --row;
            while ((row + 1) * (row + 2) / 2 <= in) ++row;
            *i = row;
            *j = in - row * (row + 1) / 2;
            return true;
        }
        const int32_t group = in / (kGroup * tn), first = group * kGroup, h = min(kGroup, tm - first),
                      rest = in - group * kGroup * tn;
        *i = first + rest % h;
        *j = rest / h;
        return true;
    }
};

// Tiles: 256 x 256 (8 wavefronts, one workgroup a compute unit), 128 x 128 (4 wavefronts, two workgroups, so that one's end is hidden
// behind the other's products), 64 x 64 (two groups of 2 wavefronts, where there is little to do: 5 x 320 x 320 x 1024 with four planes
// 15.7 us in one group, 14.2 with steps twice as long, 13 in two).
template <int PA, int PB, bool CA, bool CB>
using Tile256 = Tile<256, 256, 2, 4, PA + PB == 2 ? 64 : 32, PA, PB, CA, CB>;
template <int PA, int PB, bool CA, bool CB>
using Tile128 = Tile<128, 128, 2, 2, PA + PB == 2 ? 64 : 32, PA, PB, CA, CB>;
template <int PA, int PB, bool CA, bool CB>
using Tile64 = Tile<64, 64, 2, 1, 64, PA, PB, CA, CB, 2>;

// The side of the tiles that take the least time, by what the kernels took on these shapes: a tile occupies its compute unit for so many
// us a thousand terms and so many at its ends, by the planes of both operands; one of the smallest alone there is no faster than
// kAlone.  us for 256, 128, 64: one plane each, 8 x 4096 x 4096 x 768 304, 346, 449; 8 x 4096 x 768 x 2048 163, 157, 220;
// 8 x 8192 x 1024 x 4096 558, 644, 956; three planes, 8 x 4096 x 2048 x 768 449, 420, 559; 2 x 11264 x 2048 x 2048 421, 412, 589; four
// planes, 5 x 513 x 257 x 1023 71, 30, 15.5; 16 x 1024 x 1024 x 1024 110, 120, 185.
struct TileTime {
    double tiles, us;  // tiles of a product, us each
    // t: side 64 << t
    TileTime(int t, int planes, int64_t rows, int64_t cols, int64_t K, int64_t batch, bool lower) {
        static constexpr double kRate[3][3] = {{3.8, 9.8, 33.5}, {6.8, 16.5, 65.}, {11.5, 25., 85.}}, kEnds[3][3] = {{0.8, 3.5, 12.}, {2.5, 10., 60.}, {1., 7., 20.}};
        const int64_t s = 64 << t, i = (rows + s - 1) / s, j = (cols + s - 1) / s;
        tiles = (double)((lower ? i * (i + 1) / 2 : i * j) * batch);
        us = kRate[planes - 2][t] * 1e-3 * (double)K + kEnds[planes - 2][t];
    }
    static double alone(int planes, int64_t K) {
        static constexpr double kAlone[3] = {6., 8.5, 11.};
        return kAlone[planes - 2] * 1e-3 * (double)K + 3.;
    }
};
inline int tile_side(int num_cus, int planes, int64_t rows, int64_t cols, int64_t K, int64_t batch, bool lower) {
    double best = 0.;
    int side = 0;
    for (int t = 0; t < 3; ++t) {
        const TileTime tile(t, planes, rows, cols, K, batch, lower);
        double us = ceil(tile.tiles / num_cus) * tile.us;
        if (t == 0 && us < TileTime::alone(planes, K)) us = TileTime::alone(planes, K);
        if (t == 0 || us < best) {
            best = us;
            side = 64 << t;
        }
    }
    return side;
}

// ---- values as halves ---------------------------------------------------------------------------------------------------
// The power of two that brings values of at most `bound` below 2^15, and its inverse.  Where there is nothing but zeros the inverse is 0:
// folded into another operand it must not outweigh rows that have values.  An infinity or NaN: NaN, which everything scaled by it becomes.
struct Scale {
    float up, down;
};
__device__ __forceinline__ Scale scale_for(float bound) {
    if (bound == 0.f) return {1.f, 0.f};
    if (!(bound < INFINITY)) return {NAN, NAN};
    const int e = (int)(__float_as_uint(bound) >> 23) - 127;
    const int up = min(max(14 - e, -126), 126);
    return {__uint_as_float((uint32_t)(127 + up) << 23), __uint_as_float((uint32_t)(127 - up) << 23)};
}

// v as the sum of two halves.  A product or sum that is rounded to a half in one instruction (v_fma_mix) can come out as another half than by way of
// fp32, where that lies in the middle of two: lo would then be what is left of a neighbour of hi.  So v is fixed before.
__device__ __forceinline__ void split(float v, half_t* hi, half_t* lo) {
    asm("" : "+v"(v));
    *hi = (half_t)v;
    *lo = (half_t)(v - (float)*hi);
}

// v as one half or the sum of two, eight at a time.
template <int Planes>
__device__ __forceinline__ void store_planes(half_t* to, int64_t plane, const float* v) {
    half8 hi, lo;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        half_t h, l;
        split(v[k], &h, &l);
        hi[k] = h;
        lo[k] = l;
    }
    *reinterpret_cast<half8*>(to) = hi;
    if constexpr (Planes == 2) *reinterpret_cast<half8*>(to + plane) = lo;
}
