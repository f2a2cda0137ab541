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
// a lane, two buffers: the next tile arrives while this one is multiplied.  Rows of a "rows" tile are read as they are (ds_read_b128,
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

template <int kBM, int kBN, int kWM, int kWN, int kBK, int kPA, int kPB, bool kColsA, bool kColsB>
struct Tile {
    static constexpr int BM = kBM, BN = kBN, WM = kWM, WN = kWN, BK = kBK, PA = kPA, PB = kPB;
    static constexpr bool ColsA = kColsA, ColsB = kColsB;
    static constexpr int Waves = WM * WN, Threads = Waves * kWave;
    static constexpr int MI = BM / WM / 32, NI = BN / WN / 32;             // 32 x 32 blocks of a wavefront
    static constexpr int BytesA = BM * BK * 2, BytesB = BN * BK * 2;       // of a plane
    static constexpr int Stage = PA * BytesA + PB * BytesB;
    static_assert(kPad % BK == 0 && Stage * 2 <= 160 * 1024, "tile");
};

namespace product {

typedef __attribute__((address_space(1))) const void gvoid;
typedef __attribute__((address_space(3))) void lvoid;

// Offset in bytes, from the tile's first row (or column) at k = 0, of the piece that lane `t` loads in round r.
template <int R, int BK, bool Cols, int Threads>
__device__ __forceinline__ uint32_t piece_offset(int t, int r, uint32_t ld, int32_t left) {
    const int q = r * Threads + t;
    if constexpr (!Cols) {
        constexpr int C = BK / 8;
        const int row = q / C, slot = q % C;
        const int piece = slot ^ (C == 8 ? row & 7 : (row >> 1) & 3);
        return (uint32_t)(row < left ? row : left - 1) * (ld * 2) + (uint32_t)piece * 16;
    } else {
        constexpr int C = R / 8;
        const int k = q / C, slot = q % C;
        const int col = (slot ^ ((k & 3) << 1)) * 8;
        return (uint32_t)k * (ld * 2) + (uint32_t)(col < left ? col : left - 8) * 2;
    }
}

// Where a lane's fragments begin within a plane's tile.  rows: [kk] for each 16 k's; columns: [block parity] of the 32 i's.
template <int R, int BK, bool Cols>
struct Reader {
    static constexpr int N = Cols ? 2 : BK / 16;
    uint32_t at[N];
    __device__ __forceinline__ explicit Reader(int lane, int first) {
        if constexpr (!Cols) {
            constexpr int C = BK / 8;
            const int row = lane & 31, swap = (lane >> 5) ^ (C == 8 ? row & 7 : (row >> 1) & 3);
#pragma unroll
            for (int kk = 0; kk < N; ++kk) at[kk] = (uint32_t)((first + row) * BK * 2 + (swap ^ (kk * 2)) * 16);
        } else {
            const int g = lane >> 4, i = lane & 15;
            const int k = (g >> 1) * 8 + i / 4, c = (g & 1) * 2 + (i % 4) / 2;
#pragma unroll
            for (int p = 0; p < 2; ++p) at[p] = (uint32_t)(k * R * 2 + first * 2 + ((c | p << 2) ^ (i / 4) << 1) * 16 + (i & 1) * 8);
        }
    }
    // i's first + 32 * block .., k's 16 * kk .. of the tile at `lds`.  first is a multiple of 64 where Cols.
    __device__ __forceinline__ half8 read(const char* lds, int block, int kk) const {
        if constexpr (!Cols) {
            return *reinterpret_cast<const half8*>(lds + at[kk] + block * 32 * BK * 2);
        } else {
            typedef __attribute__((address_space(3))) short4v lshort;
            const char* from = lds + at[block & 1] + (block >> 1) * 128 + kk * 16 * R * 2;
            const half4 a = __builtin_bit_cast(half4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lshort*)(from)));
            const half4 b = __builtin_bit_cast(half4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lshort*)(from + 4 * R * 2)));
            return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
};

}  // namespace product

// The tile of rows m0 .., columns n0 .. of one batch entry, K (a multiple of kPad) terms: acc[block of 32 columns][block of 32
// rows], in which lane l holds row l % 32 and columns 8 (r / 4) + 4 (l / 32) + r % 4.
// `offB(row)`: row of B's memory that holds column n0 + row (rows operands only; nullptr_t: n0 + row itself).
template <typename S, typename RowB>
__device__ __forceinline__ void product_tile(const Operand& A, const Operand& B, int64_t batch, int32_t m0, int32_t n0, int32_t K, char* lds,
                                             acc16 (&acc)[S::NI][S::MI], RowB&& row_b) {
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
    const int firstA = wave / S::WN * (S::BM / S::WM), firstB = wave % S::WN * (S::BN / S::WN);
    const Reader<S::BM, S::BK, S::ColsA> ra(lane, firstA);
    const Reader<S::BN, S::BK, S::ColsB> rb(lane, firstB);
#pragma unroll
    for (int j = 0; j < S::NI; ++j)
#pragma unroll
        for (int i = 0; i < S::MI; ++i) acc[j][i] = acc16{};

    const int steps = K / S::BK;
    fetch(0);
    __syncthreads();
    for (int s = 0; s < steps; ++s) {
        if (s + 1 < steps) fetch((s + 1) & 1);
        const char* at = lds + (s & 1) * S::Stage;
#pragma unroll
        for (int kk = 0; kk < S::BK / 16; ++kk) {
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
                    if (pa + pb == 2) continue;
#pragma unroll
                    for (int j = 0; j < S::NI; ++j)
#pragma unroll
                        for (int i = 0; i < S::MI; ++i)
                            acc[j][i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fb[pb][j], fa[pa][i], acc[j][i], 0, 0, 0);
                }
        }
        __syncthreads();
    }
}

// f(row, column, four columns' values) for every lane's share of a tile's accumulators.
template <typename S, typename F>
__device__ __forceinline__ void each_quad(const acc16 (&acc)[S::NI][S::MI], int32_t m0, int32_t n0, F&& f) {
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int32_t row0 = m0 + wave / S::WN * (S::BM / S::WM) + (lane & 31), col0 = n0 + wave % S::WN * (S::BN / S::WN) + (lane >> 5) * 4;
#pragma unroll
    for (int i = 0; i < S::MI; ++i)
#pragma unroll
        for (int j = 0; j < S::NI; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                f(row0 + i * 32, col0 + j * 32 + q * 8, v4f{acc[j][i][q * 4], acc[j][i][q * 4 + 1], acc[j][i][q * 4 + 2], acc[j][i][q * 4 + 3]});
}

// Which tile a workgroup takes: the tiles of a batch entry stay on one XCD as far as they go (workgroups go round the eight by their
// number), and there in groups of kGroup rows of tiles, so that the ones under way together share rows and columns in its L2.
struct TileGrid {
    int32_t tm, tn;    // tiles of a batch entry
    uint32_t total;    // of all
    static constexpr uint32_t kXcds = 8;
    static constexpr int32_t kGroup = 8;
    __host__ uint32_t blocks() const { return (total + kXcds - 1) / kXcds * kXcds; }
    // false: none is left for this workgroup
    __device__ __forceinline__ bool at(uint32_t block, int32_t* batch, int32_t* i, int32_t* j) const {
        const uint32_t per = (total + kXcds - 1) / kXcds, id = block % kXcds * per + block / kXcds;
        if (id >= total) return false;
        const uint32_t one = (uint32_t)(tm * tn);
        *batch = (int32_t)(id / one);
        const int32_t in = (int32_t)(id % one), group = in / (kGroup * tn), first = group * kGroup, h = min(kGroup, tm - first),
                      rest = in - group * kGroup * tn;
        *i = first + rest % h;
        *j = rest / h;
        return true;
    }
};

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

// v as one half or the sum of two.
__device__ __forceinline__ void split4(v4f v, half4* hi, half4* lo) {
    *hi = __builtin_convertvector(v, half4);
    *lo = __builtin_convertvector(v - __builtin_convertvector(*hi, v4f), half4);
}
template <int Planes>
__device__ __forceinline__ void store_planes(half_t* to, int64_t plane, v4f v) {
    half4 hi, lo;
    split4(v, &hi, &lo);
    *reinterpret_cast<half4*>(to) = hi;
    if constexpr (Planes == 2) *reinterpret_cast<half4*>(to + plane) = lo;
}
