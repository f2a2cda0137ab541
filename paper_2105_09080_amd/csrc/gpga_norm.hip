// Dropout with a residual sum, and layer norm of that sum, forward and backward, with a gamma and a beta for each node.
//
//   u = residual + mask * x * factor                                (dropout alone: y = u)
//   y = gamma_i * (u - mean(u)) * rstd + beta_i,  rstd = 1 / sqrt(var(u) + eps)
// backward, with h = gamma_i * dy and xh = (u - mean) * rstd:
//   du = rstd * (h - mean(h) - xh * mean(h * xh)) + more,  dx = mask * du * factor
//   dgamma_i = sum over t of dy * xh,  dbeta_i = sum over t of dy
//
// The mask is made anew wherever it is needed (gpga_rows.hpp).  Mean, variance and the backward means are fp32 sums over
// values in registers; the variance is that of the differences from the mean, not a difference of sums.  y comes from u
// before u is rounded for its own store.
//
// All of it is bound by the bytes of the activations: a row is read once, held in the registers of the lanes that share it, and
// its results are written once.  As many lanes share a row as hold it in one to three pieces each (8 to 64 of a wavefront,
// whose sums need no LDS, then a workgroup); rows of more than 8192 columns are read again.
#include "gpga_rows.hpp"

namespace {

constexpr int kThreads = 256;
constexpr int kLongThreads = 1024;  // rows that do not fit into a workgroup's registers

uint32_t blocks_for(int64_t items, int64_t per_block) { return (uint32_t)((items + per_block - 1) / per_block); }

template <typename E>
struct NormArgs {
    typedef typename E::mem mem;
    int32_t T, D;
    int64_t ld, ldx;         // of the activations, of X and g
    uint32_t per_node;       // workgroups of a node
    uint32_t first_block;    // of the launch
    DropArgs drop;
    bool stream;             // activations pass by the caches
    float eps;
    const mem* x;            // forward: x; backward: dy
    const mem* side;         // forward: residual; backward: more (may be NULL)
    const mem* u_in;         // backward
    mem* u;                  // forward: u (may be NULL); backward: du
    mem* y;                  // forward: y; backward: dx (may be NULL)
    float* stats;            // n*T pairs; forward: may be NULL
    const float* gamma;      // columns of node 0 in X
    const float* beta;
    float* partial;          // backward: n * per_node * 2 * D; NULL: one workgroup a node, straight to g
    float* g_gamma;          // columns of node 0 in g
    float* g_beta;
    bool accumulate;
};

// ---- dropout ----------------------------------------------------------------------------------------------------------
// 2^lanes_log2 lanes a row, one piece a lane and turn.  Bound by memory: 16 x 8192 x 1024 bf16 with a residual 127 us, 6.3 TB/s of three
// streams; the generator (18 quarter-rate products for eight elements) runs beside it.
template <typename E, bool kSide>
__global__ __launch_bounds__(kThreads) void k_dropout(NormArgs<E> a, int lanes_log2) {
    const uint32_t block = a.first_block + blockIdx.x, node = block / a.per_node;
    const int32_t t = (int32_t)((block - node * a.per_node) * (uint32_t)(kThreads >> lanes_log2)) + (int32_t)(threadIdx.x >> lanes_log2);
    if (t >= a.T) return;
    const int64_t row = ((int64_t)node * a.T + t) * a.ld;
    const DropNode mask(a.drop, node);
    const uint32_t octs = ((uint32_t)a.D + kOct - 1) / kOct;
    for (uint32_t q = threadIdx.x & ((1u << lanes_log2) - 1u); q < octs; q += 1u << lanes_log2) {
        const int32_t c = (int32_t)q * kOct;
        const Piece<E, kOct> in = piece_load<kOct, E>(a.x + row, c, a.D, a.stream);
        Piece<E, kOct> side;
        if (kSide) side = piece_load<kOct, E>(a.side + row, c, a.D, a.stream);
        float v[kOct];
        piece_get<kOct, E>(in, c, a.D, v);
        if (a.drop.drop) mask.apply(a.drop, (uint32_t)t * octs + q, v);
        if (kSide) {
            float r[kOct];
            piece_get<kOct, E>(side, c, a.D, r);
#pragma unroll
            for (int j = 0; j < kOct; ++j) v[j] += r[j];
        }
        piece_put<kOct, E>(a.y + row, c, a.D, v, a.stream);
    }
}

// What columns past the end of the row hold.
__device__ __forceinline__ void past_end(float* v, int32_t c, int32_t D, float value) {
#pragma unroll
    for (int j = 0; j < kOct; ++j) v[j] = c + j < D ? v[j] : value;
}

// u of eight columns, before rounding.
template <typename E>
__device__ __forceinline__ void norm_input(const NormArgs<E>& a, const DropNode& mask, const Piece<E, kOct>& x, const Piece<E, kOct>& side,
                                           uint32_t group, int32_t c, float* v) {
    piece_get<kOct, E>(x, c, a.D, v);
    if (a.drop.drop) mask.apply(a.drop, group, v);
    if (a.side) {
        float r[kOct];
        piece_get<kOct, E>(side, c, a.D, r);
#pragma unroll
        for (int j = 0; j < kOct; ++j) v[j] += r[j];
    }
}

// y of eight columns from u.
template <typename E>
__device__ __forceinline__ void norm_output(const NormArgs<E>& a, uint32_t node, int64_t row, int32_t c, float mean, float rstd, const float* u) {
    typedef Elem<float, E::kNarrow> P;
    float gm[kOct], bt[kOct], y[kOct];
    piece_read<kOct, P>(a.gamma + (int64_t)node * a.ldx, c, a.D, gm);
    piece_read<kOct, P>(a.beta + (int64_t)node * a.ldx, c, a.D, bt);
#pragma unroll
    for (int j = 0; j < kOct; ++j) y[j] = (u[j] - mean) * rstd * gm[j] + bt[j];
    piece_put<kOct, E>(a.y + row, c, a.D, y, a.stream);
}

// ---- forward: L lanes a row, N pieces a lane, the row in registers ----------------------------------------------------------
// 8 x 4096 rows of 768 bf16 with dropout and residual: 36 us, 5.6 TB/s of four streams.  gamma and beta are read again for every
// row, from the caches of the compute unit.  One row of 768 fp32 a node: 4 us, what a launch and two dependent loads take.
template <typename E, int L, int N>
__global__ __launch_bounds__(L > kThreads ? L : kThreads) void k_norm(NormArgs<E> a) {
    constexpr int kRows = L > kThreads ? 1 : kThreads / L;  // rows of a workgroup
    __shared__ float s_sum[2][L > kWave ? L / kWave : 1];
    const uint32_t block = a.first_block + blockIdx.x, node = block / a.per_node;
    const int32_t t = (int32_t)((block - node * a.per_node) * kRows + threadIdx.x / L);
    if (t >= a.T) return;  // all lanes of a row; no workgroup whose sums span wavefronts
    const int64_t r = (int64_t)node * a.T + t, row = r * a.ld;
    const int32_t lane = threadIdx.x & (L - 1);
    const uint32_t octs = ((uint32_t)a.D + kOct - 1) / kOct;
    const DropNode mask(a.drop, node);
    Piece<E, kOct> x[N], side[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        x[k] = piece_load<kOct, E>(a.x + row, (lane + k * L) * kOct, a.D, a.stream);
        if (a.side) side[k] = piece_load<kOct, E>(a.side + row, (lane + k * L) * kOct, a.D, a.stream);
    }
    float u[N][kOct], sum[1] = {0.f}, var[1] = {0.f};
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int32_t q = lane + k * L, c = q * kOct;
        norm_input<E>(a, mask, x[k], side[k], (uint32_t)t * octs + q, c, u[k]);
        if (c + kOct > a.D) past_end(u[k], c, a.D, 0.f);
#pragma unroll
        for (int j = 0; j < kOct; ++j) sum[0] += u[k][j];
    }
    lanes_sum<L>(sum, s_sum[0]);
    const float inv = 1.f / (float)a.D, mean = sum[0] * inv;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int32_t c = (lane + k * L) * kOct;
        if (c + kOct > a.D) past_end(u[k], c, a.D, mean);
#pragma unroll
        for (int j = 0; j < kOct; ++j) var[0] += (u[k][j] - mean) * (u[k][j] - mean);
    }
    lanes_sum<L>(var, s_sum[1]);
    const float rstd = 1.f / sqrtf(var[0] * inv + a.eps);
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int32_t c = (lane + k * L) * kOct;
        if (c < a.D) {
            if (a.u) piece_put<kOct, E>(a.u + row, c, a.D, u[k], a.stream);
            norm_output<E>(a, node, row, c, mean, rstd, u[k]);
        }
    }
    if (a.stats && lane == 0) {
        a.stats[2 * r] = mean;
        a.stats[2 * r + 1] = rstd;
    }
}

// Longer rows: one workgroup a row, which reads it three times (from the caches after the first).
template <typename E>
__global__ __launch_bounds__(kLongThreads) void k_norm_long(NormArgs<E> a) {
    __shared__ float s_sum[2][kLongThreads / kWave];
    const uint32_t block = a.first_block + blockIdx.x, node = block / a.per_node;
    const int32_t t = (int32_t)(block - node * a.per_node);
    const int64_t r = (int64_t)node * a.T + t, row = r * a.ld;
    const uint32_t octs = ((uint32_t)a.D + kOct - 1) / kOct;
    const DropNode mask(a.drop, node);
    float sum[1] = {0.f}, var[1] = {0.f}, u[kOct];
    auto input = [&](uint32_t q) {
        const int32_t c = (int32_t)q * kOct;
        const Piece<E, kOct> x = piece_load<kOct, E>(a.x + row, c, a.D);
        Piece<E, kOct> side;
        if (a.side) side = piece_load<kOct, E>(a.side + row, c, a.D);
        norm_input<E>(a, mask, x, side, (uint32_t)t * octs + q, c, u);
    };
    for (uint32_t q = threadIdx.x; q < octs; q += kLongThreads) {
        input(q);
#pragma unroll
        for (int j = 0; j < kOct; ++j) sum[0] += (int32_t)q * kOct + j < a.D ? u[j] : 0.f;
    }
    lanes_sum<kLongThreads>(sum, s_sum[0]);
    const float inv = 1.f / (float)a.D, mean = sum[0] * inv;
    for (uint32_t q = threadIdx.x; q < octs; q += kLongThreads) {
        input(q);
#pragma unroll
        for (int j = 0; j < kOct; ++j) var[0] += (int32_t)q * kOct + j < a.D ? (u[j] - mean) * (u[j] - mean) : 0.f;
    }
    lanes_sum<kLongThreads>(var, s_sum[1]);
    const float rstd = 1.f / sqrtf(var[0] * inv + a.eps);
    for (uint32_t q = threadIdx.x; q < octs; q += kLongThreads) {
        const int32_t c = (int32_t)q * kOct;
        input(q);
        if (a.u) piece_put<kOct, E>(a.u + row, c, a.D, u);
        norm_output<E>(a, node, row, c, mean, rstd, u);
    }
    if (a.stats && threadIdx.x == 0) {
        a.stats[2 * r] = mean;
        a.stats[2 * r + 1] = rstd;
    }
}

// ---- backward -----------------------------------------------------------------------------------------------------------
// What a lane has of a row: dy, u and the residual stream's gradient, as they lie in memory.
template <typename E, int N, bool kSide>
struct GradRow {
    Piece<E, kOct> dy[N], u[N], more[kSide ? N : 1];
    float mean, rstd;
};
template <int L, int N, typename E, bool kSide>
__device__ __forceinline__ void grad_load(const NormArgs<E>& a, int64_t r, int32_t lane, GradRow<E, N, kSide>& in) {
    const int64_t row = r * a.ld;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int32_t c = (lane + k * L) * kOct;
        in.dy[k] = piece_load<kOct, E>(a.x + row, c, a.D);
        in.u[k] = piece_load<kOct, E>(a.u_in + row, c, a.D);
        if (kSide) in.more[k] = piece_load<kOct, E>(a.side + row, c, a.D);
    }
    in.mean = a.stats[2 * r];
    in.rstd = a.stats[2 * r + 1];
}
// dy and xh of eight columns; 0 past the end of the row.
template <typename E>
__device__ __forceinline__ void grad_input(const Piece<E, kOct>& dy_in, const Piece<E, kOct>& u_in, int32_t c, int32_t D, float mean, float rstd,
                                           float* dy, float* xh) {
    piece_get<kOct, E>(dy_in, c, D, dy);
    piece_get<kOct, E>(u_in, c, D, xh);
#pragma unroll
    for (int j = 0; j < kOct; ++j) xh[j] = (xh[j] - mean) * rstd;
    if (c + kOct > D) {
        past_end(dy, c, D, 0.f);
        past_end(xh, c, D, 0.f);
    }
}
// du and dx of eight columns.
template <bool kSide, typename E>
__device__ __forceinline__ void grad_output(const NormArgs<E>& a, const DropNode& mask, const Piece<E, kOct>& more_in, int64_t row, uint32_t group,
                                            int32_t c, float rstd, float m1, float m2, const float* h, const float* xh) {
    float du[kOct], more[kOct] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (kSide) piece_get<kOct, E>(more_in, c, a.D, more);
#pragma unroll
    for (int j = 0; j < kOct; ++j) du[j] = rstd * (h[j] - m1 - xh[j] * m2) + more[j];
    piece_put<kOct, E>(a.u + row, c, a.D, du, a.stream);
    if (a.y) {
        mask.apply(a.drop, group, du);
        piece_put<kOct, E>(a.y + row, c, a.D, du, a.stream);
    }
}

// Sum over the rows that a wavefront works on side by side, L lanes each; lane by lane.
template <int L>
__device__ __forceinline__ float other_rows_sum(float v) {
    if constexpr (L <= 8) v += dpp<0x128>(v);  // the eight lanes beside
    if constexpr (L <= 16) {
        const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    if constexpr (L <= 32) {
        const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    return v;
}
// Eight floats in LDS.
struct OctInLds {
    static __device__ __forceinline__ void store(float* p, const float* v) {
        v4f* to = reinterpret_cast<v4f*>(p);
        to[0] = v4f{v[0], v[1], v[2], v[3]};
        to[1] = v4f{v[4], v[5], v[6], v[7]};
    }
    static __device__ __forceinline__ void add(const float* p, float* v) {
        const v4f* from = reinterpret_cast<const v4f*>(p);
        const v4f a = from[0], b = from[1];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[j] += a[j];
            v[4 + j] += b[j];
        }
    }
};

// Eight columns of a weight's gradient.
template <typename P>
__device__ __forceinline__ void put_weights(float* g, int32_t c, int32_t D, bool accumulate, float* v) {
    if (accumulate) {
        float had[kOct];
        piece_read<kOct, P>(g, c, D, had);
#pragma unroll
        for (int j = 0; j < kOct; ++j) v[j] += had[j];
    }
    piece_put<kOct, P>(g, c, D, v);
}

// L lanes a row.  A workgroup takes the rows t = strip, strip + strips, ... of a node kRows at a time, keeps its sums for
// dgamma and dbeta in registers, and leaves them in `partial`.  A row's loads are issued while the one before it is worked on:
// the registers (209 for three pieces of bf16; 255 and 24 more for fp32 with `more`, which leaves one) leave two wavefronts a SIMD,
// and without that 8 x 4096 rows of 768 bf16 took 50 to 54 us against 43, all in (4.7 TB/s; traced one by one 42.5 here and 4.7
// in the join of 512 partial sums).
template <typename E, int L, int N, bool kSide>
__global__ __launch_bounds__(L > kThreads ? L : kThreads) void k_norm_grad(NormArgs<E> a) {
    typedef Elem<float, E::kNarrow> P;
    constexpr int kBlock = L > kThreads ? L : kThreads, kRows = kBlock / L;
    __shared__ float s_sum[2][L > kWave ? 2 * L / kWave : 1];
    __shared__ __align__(16) float s_part[kRows > 1 ? 2 * L * N * kOct : 4];
    const uint32_t block = a.first_block + blockIdx.x, node = block / a.per_node, strip = block - node * a.per_node;
    const int32_t lane = threadIdx.x & (L - 1), sub = threadIdx.x / L;
    const uint32_t octs = ((uint32_t)a.D + kOct - 1) / kOct;
    const DropNode mask(a.drop, node);
    const float inv = 1.f / (float)a.D;
    const int64_t first_row = (int64_t)node * a.T, stride = (int64_t)a.per_node * kRows;
    int64_t t = (int64_t)strip * kRows + sub;
    GradRow<E, N, kSide> next;
    if (t < a.T) grad_load<L, N, E, kSide>(a, first_row + t, lane, next);
    float gm[N][kOct], dg[N][kOct], db[N][kOct];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int32_t c = (lane + k * L) * kOct;
        piece_read<kOct, P>(a.gamma + (int64_t)node * a.ldx, c, a.D, gm[k]);
#pragma unroll
        for (int j = 0; j < kOct; ++j) dg[k][j] = db[k][j] = 0.f;
    }
    int turn = 0;
    for (; t < a.T; t += stride, turn ^= 1) {  // all lanes of a row alike
        const int64_t row = (first_row + t) * a.ld;
        const GradRow<E, N, kSide> in = next;
        if (t + stride < a.T) grad_load<L, N, E, kSide>(a, first_row + t + stride, lane, next);
        float h[N][kOct], xh[N][kOct], s[2] = {0.f, 0.f};
#pragma unroll
        for (int k = 0; k < N; ++k) {
            grad_input<E>(in.dy[k], in.u[k], (lane + k * L) * kOct, a.D, in.mean, in.rstd, h[k], xh[k]);
#pragma unroll
            for (int j = 0; j < kOct; ++j) {
                dg[k][j] += h[k][j] * xh[k][j];
                db[k][j] += h[k][j];
                h[k][j] *= gm[k][j];
                s[0] += h[k][j];
                s[1] += h[k][j] * xh[k][j];
            }
        }
        lanes_sum<L>(s, s_sum[turn]);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int32_t q = lane + k * L, c = q * kOct;
            if (c < a.D) grad_output<kSide, E>(a, mask, in.more[kSide ? k : 0], row, (uint32_t)t * octs + (uint32_t)q, c, in.rstd, s[0] * inv, s[1] * inv, h[k], xh[k]);
        }
    }
    if constexpr (kRows > 1) {
        // rows of one wavefront by the swaps of lanes, the wavefronts one after another through LDS
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int j = 0; j < kOct; ++j) {
                dg[k][j] = other_rows_sum<L>(dg[k][j]);
                db[k][j] = other_rows_sum<L>(db[k][j]);
            }
        const int wave = threadIdx.x / kWave;
        float* mine = s_part + (threadIdx.x & (L - 1)) * kOct;
        for (int w = 1; w < kBlock / kWave; ++w) {
            if (wave == w && (threadIdx.x & (kWave - 1)) < L) {
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    OctInLds::store(mine + (2 * k) * L * kOct, dg[k]);
                    OctInLds::store(mine + (2 * k + 1) * L * kOct, db[k]);
                }
            }
            __syncthreads();
            if (sub == 0) {
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    OctInLds::add(mine + (2 * k) * L * kOct, dg[k]);
                    OctInLds::add(mine + (2 * k + 1) * L * kOct, db[k]);
                }
            }
            __syncthreads();
        }
    }
    if (sub == 0) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int32_t c = (lane + k * L) * kOct;
            if (c >= a.D) continue;
            if (a.partial) {
                float* out = a.partial + (int64_t)block * 2 * a.D;
                piece_put<kOct, P>(out, c, a.D, dg[k]);
                piece_put<kOct, P>(out + a.D, c, a.D, db[k]);
            } else {
                put_weights<P>(a.g_gamma + (int64_t)node * a.ldx, c, a.D, a.accumulate, dg[k]);
                put_weights<P>(a.g_beta + (int64_t)node * a.ldx, c, a.D, a.accumulate, db[k]);
            }
        }
    }
}

// Longer rows: sums over the tokens first (a lane a column, the tokens dealt to strips), since du may take dy's place; then du
// and dx, one workgroup a row.
template <typename E>
__global__ __launch_bounds__(kThreads) void k_norm_grad_columns(NormArgs<E> a, uint32_t column_blocks) {
    const uint32_t block = a.first_block + blockIdx.x, node = block / (a.per_node * column_blocks), in_node = block - node * a.per_node * column_blocks;
    const uint32_t strip = in_node / column_blocks;
    const int64_t c = (int64_t)(in_node - strip * column_blocks) * kThreads + threadIdx.x;
    if (c >= a.D) return;
    float dg = 0.f, db = 0.f;
    for (int64_t t = strip; t < a.T; t += a.per_node) {
        const int64_t r = (int64_t)node * a.T + t;
        const float dy = E::get(a.x[r * a.ld + c]);
        dg += dy * ((E::get(a.u_in[r * a.ld + c]) - a.stats[2 * r]) * a.stats[2 * r + 1]);
        db += dy;
    }
    float* out = a.partial + ((int64_t)node * a.per_node + strip) * 2 * a.D;
    out[c] = dg;
    out[a.D + c] = db;
}
template <typename E, bool kSide>
__global__ __launch_bounds__(kLongThreads) void k_norm_grad_long(NormArgs<E> a) {
    __shared__ float s_sum[2 * kLongThreads / kWave];
    const uint32_t block = a.first_block + blockIdx.x, node = block / (uint32_t)a.T;
    const uint32_t t = block - node * (uint32_t)a.T;
    const int64_t r = (int64_t)node * a.T + t;
    const uint32_t octs = ((uint32_t)a.D + kOct - 1) / kOct;
    const DropNode mask(a.drop, node);
    const float* gamma = a.gamma + (int64_t)node * a.ldx;
    float s[2] = {0.f, 0.f}, h[kOct], xh[kOct];
    GradRow<E, 1, kSide> in;
    auto input = [&](uint32_t q) {
        const int32_t c = (int32_t)q * kOct;
        float gm[kOct];
        grad_load<kLongThreads, 1, E, kSide>(a, r, (int32_t)q, in);
        piece_read<kOct, ElemF32>(gamma, c, a.D, gm);
        grad_input<E>(in.dy[0], in.u[0], c, a.D, in.mean, in.rstd, h, xh);
#pragma unroll
        for (int j = 0; j < kOct; ++j) h[j] *= gm[j];
    };
    for (uint32_t q = threadIdx.x; q < octs; q += kLongThreads) {
        input(q);
#pragma unroll
        for (int j = 0; j < kOct; ++j) {
            s[0] += h[j];
            s[1] += h[j] * xh[j];
        }
    }
    lanes_sum<kLongThreads>(s, s_sum);
    const float inv = 1.f / (float)a.D;
    for (uint32_t q = threadIdx.x; q < octs; q += kLongThreads) {
        input(q);
        grad_output<kSide, E>(a, mask, in.more[0], r * a.ld, t * octs + q, (int32_t)q * kOct, in.rstd, s[0] * inv, s[1] * inv, h, xh);
    }
}

// Adds the strips of a node: 64 columns a workgroup, its wavefronts share the strips, eight loads under way; a fixed order.  4 us, a chain
// of two trips to memory.
__global__ __launch_bounds__(kThreads) void k_norm_grad_join(const float* __restrict__ partial, uint32_t strips, int32_t D, uint32_t blocks_per_node,
                                                             bool accumulate, float* __restrict__ g_gamma, float* __restrict__ g_beta, int64_t ldg, uint32_t first_block) {
    constexpr int kWaves = kThreads / kWave;
    __shared__ float s_part[kWaves][kWave];
    const uint32_t block = first_block + blockIdx.x, node = block / blocks_per_node;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int64_t c = (int64_t)(block - node * blocks_per_node) * kWave + lane;  // 0 .. 2D-1: gamma's columns, then beta's
    const float* from = partial + (int64_t)node * strips * 2 * D + c;
    float sum = 0.f;
    if (c < 2 * (int64_t)D) {
#pragma unroll 8
        for (uint32_t k = wave; k < strips; k += kWaves) sum += from[(int64_t)k * 2 * D];
    }
    s_part[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && c < 2 * (int64_t)D) {
#pragma unroll
        for (int w = 1; w < kWaves; ++w) sum += s_part[w][lane];
        float* out = (c < D ? g_gamma + c : g_beta + (c - D)) + (int64_t)node * ldg;
        *out = accumulate ? *out + sum : sum;
    }
}

constexpr int32_t kHeldColumns = 8192;  // longest rows that registers hold

// Lanes a row and pieces a lane by the number of eights in it: the smallest that hold it.  f gets both as constants.
template <int V>
struct Const {
    static constexpr int value = V;
};
template <typename E, typename F>
bool with_row_shape(int32_t octs, F&& f) {
    if constexpr (E::kNarrow) f(Const<8>(), Const<1>());
    else if (octs <= 8) f(Const<8>(), Const<1>());
    else if (octs <= 16) f(Const<16>(), Const<1>());
    else if (octs <= 32) f(Const<32>(), Const<1>());
    else if (octs <= 64) f(Const<32>(), Const<2>());
    else if (octs <= 96) f(Const<32>(), Const<3>());
    else if (octs <= 128) f(Const<64>(), Const<2>());
    else if (octs <= 192) f(Const<64>(), Const<3>());
    else if (octs <= 256) f(Const<256>(), Const<1>());
    else if (octs <= 512) f(Const<256>(), Const<2>());
    else if (octs <= 1024) f(Const<512>(), Const<2>());
    else return false;
    return true;
}

// Strips of a node: two workgroups a compute unit over all nodes, no more than there are rows (where a workgroup takes several rows
// side by side some strips have none and add zeros: 512 rows of 768 on one node 16.9 us); a single one for few rows, whose sums
// then need no launch of their own.  us a call, bf16, one strip and as many as rows: 8 x 16 x 768 14.0 and 15.7, 64 x 4 x 8192
// 13.7 and 18.2, 64 x 16 x 8192 25.8 and 32.6; but 64 x 16 x 2048 16.3 and 15.5, 8 x 16 x 8192 22.6 and 15.3, where a workgroup
// takes its rows one after another and few nodes leave the card empty.
constexpr int32_t kFewRows = 16;
uint32_t norm_grad_strips(const RowsShape& s) {
    if (s.T <= kFewRows && s.D <= kHeldColumns) return 1;
    const int64_t most = 512 / s.n > 1 ? 512 / s.n : 1;
    return (uint32_t)(s.T < most ? (s.T > 0 ? s.T : 1) : most);
}

}  // namespace

hipError_t launch_dropout(const gpga_ctx* c, const RowsShape& s, const DropArgs& drop, const void* x, const void* residual, void* y) {
    auto launch = [&](auto e) {
        typedef decltype(e) E;
        typedef typename E::mem M;
        NormArgs<E> a = {};
        a.T = s.T;
        a.D = s.D;
        a.ld = s.ld;
        a.drop = drop;
        a.stream = stream_rows(s, x, residual, y);
        a.x = static_cast<const M*>(x);
        a.side = static_cast<const M*>(residual);
        a.y = static_cast<M*>(y);
        const int32_t octs = (s.D + kOct - 1) / kOct;
        int lanes_log2 = 0;
        while (lanes_log2 < 8 && (1 << lanes_log2) < octs) ++lanes_log2;
        a.per_node = blocks_for(s.T, kThreads >> lanes_log2);
        return launch_blocks((uint64_t)a.per_node * s.n, kThreads, [&](uint32_t first, dim3 grid) {
            a.first_block = first;
            if (residual) k_dropout<E, true><<<grid, dim3(kThreads), 0, c->stream>>>(a, lanes_log2);
            else k_dropout<E, false><<<grid, dim3(kThreads), 0, c->stream>>>(a, lanes_log2);
        });
    };
    return s.D < kOct ? with_narrow_elem(s.dtype, launch) : with_elem(s.dtype, launch);
}

hipError_t launch_norm(const gpga_ctx* c, const RowsShape& s, const DropArgs& drop, const void* x, const void* residual, int64_t gamma_off,
                       int64_t beta_off, float eps, void* u, void* y, float* stats) {
    auto launch = [&](auto el) {
        typedef decltype(el) E;
        typedef typename E::mem M;
        NormArgs<E> a = {};
        a.T = s.T;
        a.D = s.D;
        a.ld = s.ld;
        a.ldx = c->ld;
        a.drop = drop;
        a.stream = stream_rows(s, x, residual, u, y);
        a.eps = eps;
        a.x = static_cast<const M*>(x);
        a.side = static_cast<const M*>(residual);
        a.u = static_cast<M*>(u);
        a.y = static_cast<M*>(y);
        a.stats = stats;
        a.gamma = c->x + gamma_off;
        a.beta = c->x + beta_off;
        hipError_t e = hipSuccess;
        const bool held = with_row_shape<E>((s.D + kOct - 1) / kOct, [&](auto l, auto k) {
            constexpr int L = decltype(l)::value, N = decltype(k)::value, kBlock = L > kThreads ? L : kThreads;
            a.per_node = blocks_for(s.T, kBlock / L);
            e = launch_blocks((uint64_t)a.per_node * s.n, kBlock, [&](uint32_t first, dim3 grid) {
                a.first_block = first;
                k_norm<E, L, N><<<grid, dim3(kBlock), 0, c->stream>>>(a);
            });
        });
        if constexpr (!E::kNarrow) {
            if (!held) {
                a.per_node = (uint32_t)s.T;
                e = launch_blocks((uint64_t)a.per_node * s.n, kLongThreads, [&](uint32_t first, dim3 grid) {
                    a.first_block = first;
                    k_norm_long<E><<<grid, dim3(kLongThreads), 0, c->stream>>>(a);
                });
            }
        }
        return e;
    };
    return s.D < kOct ? with_narrow_elem(s.dtype, launch) : with_elem(s.dtype, launch);
}

size_t norm_grad_scratch(const RowsShape& s) { return (size_t)s.n * norm_grad_strips(s) * 2 * (size_t)s.D * sizeof(float); }

hipError_t launch_norm_grad(const gpga_ctx* c, const RowsShape& s, const DropArgs& drop, const void* dy, const void* u, const float* stats,
                            const void* more, int64_t gamma_off, int64_t beta_off, void* du, void* dx, bool accumulate, void* scratch) {
    const uint32_t strips = norm_grad_strips(s);
    const bool direct = strips == 1 && s.D <= kHeldColumns;
    auto launch = [&](auto el) {
        typedef decltype(el) E;
        typedef typename E::mem M;
        NormArgs<E> a = {};
        a.T = s.T;
        a.D = s.D;
        a.ld = s.ld;
        a.ldx = c->ld;
        a.drop = drop;
        a.stream = stream_rows(s, du, dx);
        a.x = static_cast<const M*>(dy);
        a.side = static_cast<const M*>(more);
        a.u_in = static_cast<const M*>(u);
        a.u = static_cast<M*>(du);
        a.y = static_cast<M*>(dx);
        a.stats = const_cast<float*>(stats);
        a.gamma = c->x + gamma_off;
        a.partial = direct ? nullptr : static_cast<float*>(scratch);
        a.g_gamma = c->g + gamma_off;
        a.g_beta = c->g + beta_off;
        a.accumulate = accumulate;
        a.per_node = strips;
        hipError_t e = hipSuccess;
        const bool held = with_row_shape<E>((s.D + kOct - 1) / kOct, [&](auto l, auto k) {
            constexpr int L = decltype(l)::value, N = decltype(k)::value, kBlock = L > kThreads ? L : kThreads;
            e = launch_blocks((uint64_t)strips * s.n, kBlock, [&](uint32_t first, dim3 grid) {
                a.first_block = first;
                if (more) k_norm_grad<E, L, N, true><<<grid, dim3(kBlock), 0, c->stream>>>(a);
                else k_norm_grad<E, L, N, false><<<grid, dim3(kBlock), 0, c->stream>>>(a);
            });
        });
        if constexpr (!E::kNarrow) {
            if (!held) {
                const uint32_t column_blocks = blocks_for(s.D, kThreads);
                e = launch_blocks((uint64_t)strips * column_blocks * s.n, kThreads, [&](uint32_t first, dim3 grid) {
                    a.first_block = first;
                    k_norm_grad_columns<E><<<grid, dim3(kThreads), 0, c->stream>>>(a, column_blocks);
                });
                if (e != hipSuccess) return e;
                e = launch_blocks((uint64_t)s.T * s.n, kLongThreads, [&](uint32_t first, dim3 grid) {
                    a.first_block = first;
                    if (more) k_norm_grad_long<E, true><<<grid, dim3(kLongThreads), 0, c->stream>>>(a);
                    else k_norm_grad_long<E, false><<<grid, dim3(kLongThreads), 0, c->stream>>>(a);
                });
            }
        }
        return e;
    };
    const hipError_t e = s.D < kOct ? with_narrow_elem(s.dtype, launch) : with_elem(s.dtype, launch);
    if (e != hipSuccess || direct) return e;
    const uint32_t blocks = blocks_for(2 * (int64_t)s.D, kWave);
    return launch_blocks((uint64_t)blocks * s.n, kThreads, [&](uint32_t first, dim3 grid) {
        k_norm_grad_join<<<grid, dim3(kThreads), 0, c->stream>>>(static_cast<const float*>(scratch), strips, s.D, blocks, accumulate, c->g + gamma_off,
                                                                 c->g + beta_off, c->ld, first);
    });
}
