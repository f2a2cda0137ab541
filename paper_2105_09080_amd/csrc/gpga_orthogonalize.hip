// Orthogonalised updates of the nodes' matrices (include/gpga.h): the gradient of a matrix, or its running sum, is brought near the closest
// matrix with orthonormal rows (or columns) by a few steps of Newton-Schulz iteration,
//
//   X0 = U / (|U|_F + eps),  X <- p X + (q A + r A^2) X  with A = X X^T  (or, tall, X <- p X + X (q A + r A^2) with A = X^T X),
//
// which maps every singular value s to p s + q s^3 + r s^5 and leaves the singular vectors.  A has the shorter side's size.  Small singular
// values grow by p a step, and so do errors in them: everything is held in two halves (22 bits), fp32's precision, three matrix
// instructions a step (gpga_product.hpp).  Singular values are at most |U|_F / (|U|_F + eps) to begin with; the largest that a step can make of them is
// followed, so all scales are known constants, whether values grow or shrink.
#include "gpga_pack.hpp"

#include <cmath>
#include <cstddef>

namespace {

constexpr int kThreads = 256;
constexpr int kParts = 64;  // parts of a matrix's sum of squares

// ---- scales ------------------------------------------------------------------------------------------------------------------
// Largest |a s + b s^3 + c s^5| over 0 <= s <= most.
__host__ __device__ double odd_max(double a, double b, double c, double most) {
    auto f = [&](double s) { return fabs(s * (a + s * s * (b + s * s * c))); };
    double best = f(most);
    // a + 3 b z + 5 c z^2 = 0, z = s^2
    const double d = 9.0 * b * b - 20.0 * a * c;
    double z[2] = {-1.0, -1.0};
    if (c != 0.0 && d >= 0.0) {
        z[0] = (-3.0 * b + sqrt(d)) / (10.0 * c);
        z[1] = (-3.0 * b - sqrt(d)) / (10.0 * c);
    } else if (c == 0.0 && b != 0.0) {
        z[0] = -a / (3.0 * b);
    }
    for (double v : z)
        if (v > 0.0 && v < most * most) best = fmax(best, f(sqrt(v)));
    return best;
}
// Largest |b z + c z^2| over 0 <= z <= most.
__host__ __device__ double even_max(double b, double c, double most) {
    double best = fabs(b * most + c * most * most);
    if (c != 0.0) {
        const double z = -b / (2.0 * c);
        if (z > 0.0 && z < most) best = fmax(best, fabs(b * z + c * z * z));
    }
    return best;
}
// The exponent of the power of two that brings values of at most `bound` to 2^14 or below; of `none` where the bound is 0.
__host__ __device__ int up_exponent(double bound, int none) {
    int e;
    frexp(bound, &e);
    return bound == 0.0 ? none : 14 - e;
}

// What the products of a step are multiplied by, with X, A and B = q A + r A^2 held as 2^x, 2^g and 2^b times their values.  Each of these exponents
// may be far beyond a float's; the factors, in which they meet, are about 2^-14 (or nothing, where a term is nothing beside another).
struct OrthStep {
    float gram;                   // A from X X^T
    float poly_keep, poly_times;  // B from A and A^2
    float keep, times;            // X from X and B X
};
constexpr int kMaxSteps = 64;
struct OrthScales {
    OrthStep step[kMaxSteps];     // first: the products count floats from here
    float finish[2];              // `scale` and what the last X is held in
};

struct OrthPolynomial {
    double p, q, r, scale;
    int32_t steps;
};

// The first X is held in 2^(13 - k) for singular values of at most 2^k.
constexpr int kFirst = 13;
__host__ __device__ void follow_steps(const OrthPolynomial& c, int k, OrthScales* out) {
    const double p = c.p, q = c.q, r = c.r;
    const int32_t steps = c.steps;
    int x = kFirst - k;
    double most = ldexp(1.0, k);
    for (int32_t i = 0; i < steps; ++i) {
        const double z = most * most;
        const int g = up_exponent(z * 1.001, 0), b = up_exponent(even_max(q, r, z) * 1.001, 0);
        most = odd_max(p, q, r, most) * 1.001;
        const int next = up_exponent(most, x);
        out->step[i] = {(float)ldexp(1.0, g - 2 * x), (float)ldexp(q, b - g), (float)ldexp(r, b - 2 * g), (float)ldexp(p, next - x), (float)ldexp(1.0, next - x - b)};
        x = next;
    }
    const int half = x > 120 ? -120 : x < -120 ? 120 : -x;
    out->finish[0] = (float)ldexp(1.0, half);
    out->finish[1] = (float)ldexp(c.scale, -x - half);
}

struct OrthArgs {
    float* g;              // the first matrix of node 0
    float* v;              // running sum of node 0, or NULL
    int64_t ld, v_ld;      // floats between nodes
    int32_t R, C, count;   // matrices of R x C, count in a row of each node
    int32_t first;         // number of the chunk's first matrix
    float mu;
    int nesterov;
    float eps;
    double* squares;       // kParts a matrix
    half_t* x;             // (matrices, R', C') in two planes
    int64_t plane;
    OrthScales* scales;    // one a matrix
    uint32_t per_matrix, first_block;
};

__device__ __forceinline__ float* block_of(float* base, int64_t ld, int32_t b, int32_t count, int64_t size) {
    return base + (int64_t)(b / count) * ld + (int64_t)(b % count) * size;
}

// v <- mu v + g and the sum of squares of u = g + mu v, v or g, in fp64: neither overflows nor loses small gradients.
__global__ __launch_bounds__(kThreads) void k_orth_norm(OrthArgs a) {
    typedef float vec __attribute__((ext_vector_type(4), aligned(4)));
    const uint32_t block = a.first_block + blockIdx.x, part = block % kParts;
    const int32_t b = a.first + (int32_t)(block / kParts);
    const int64_t size = (int64_t)a.R * a.C;
    const float* g = block_of(a.g, a.ld, b, a.count, size);
    float* v = a.v ? block_of(a.v, a.v_ld, b, a.count, size) : nullptr;
    double sum = 0.0;
    auto one = [&](float u, float old, float* w) {
        *w = a.mu * old + u;
        if (v) u = a.nesterov ? u + a.mu * *w : *w;
        sum += (double)u * u;
    };
    const int64_t fours = size / 4, at = (int64_t)part * kThreads + threadIdx.x;
#pragma unroll 2
    for (int64_t e = at; e < fours; e += (int64_t)kParts * kThreads) {
        const vec u = *(reinterpret_cast<const vec*>(g) + e);
        vec old = {0.f, 0.f, 0.f, 0.f};
        if (v) old = *(reinterpret_cast<const vec*>(v) + e);
        float w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) one(u[k], old[k], &w[k]);
        if (v) *(reinterpret_cast<vec*>(v) + e) = vec{w[0], w[1], w[2], w[3]};
    }
    if (at < size % 4) {
        const int64_t e = fours * 4 + at;
        float w;
        one(g[e], v ? v[e] : 0.f, &w);
        if (v) v[e] = w;
    }
    __shared__ double s[kThreads];
    s[threadIdx.x] = sum;
    for (int h = kThreads / 2; h > 0; h >>= 1) {
        __syncthreads();
        if ((int)threadIdx.x < h) s[threadIdx.x] += s[threadIdx.x + h];
    }
    if (threadIdx.x == 0) a.squares[block] = s[0];
}

// What turns U into the first X: 2^(13 - k) / (|U| + eps), a product of two floats since it may be beyond one, with |U| / (|U| + eps) at most 2^k,
// k = 0 unless eps is above |U|.  0 for a matrix of zeros, NaN for one with an infinity or NaN.
struct OrthStart {
    float first, second;
    int k;
};
__device__ __forceinline__ OrthStart orth_start(double squares, float eps) {
    if (squares == 0.0) return {0.f, 0.f, 0};
    const double norm = sqrt(squares), whole = norm + (double)eps;
    if (!(whole < INFINITY)) return {NAN, NAN, 0};
    const double inv = 1.0 / whole;
    int k = 0, e;
    if (norm * 2.0 < whole) frexp(norm * inv, &k);
    const double f = frexp(ldexp(inv, kFirst - k), &e);
    return {ldexpf(1.f, e / 2), (float)ldexp(f, e - e / 2), k};
}

// u / (|u| + eps) as halves, a wavefront a row.
template <typename E>
__global__ __launch_bounds__(kThreads) void k_orth_pack(OrthArgs a, OrthPolynomial c0, OrthScales usual) {
    const uint32_t block = a.first_block + blockIdx.x;
    const int32_t m = (int32_t)(block / a.per_matrix), b = a.first + m, lane = threadIdx.x & (kWave - 1);
    const int32_t row = (int32_t)(block % a.per_matrix) * (kThreads / kWave) + threadIdx.x / kWave, R2 = padded(a.R), C2 = padded(a.C);
    double total = a.squares[m * kParts + lane];
    for (int h = kWave / 2; h > 0; h >>= 1) total += __shfl_xor(total, h);
    const OrthStart start = orth_start(total, a.eps);
    if (block % a.per_matrix == 0 && threadIdx.x < kWave) {
        if (start.k != 0) {
            if (lane == 0) follow_steps(c0, start.k, a.scales + m);
        } else {
            constexpr int kWords = (int)(sizeof(OrthScales) / sizeof(float));
            for (int i = lane; i < kWords; i += kWave) reinterpret_cast<float*>(a.scales + m)[i] = reinterpret_cast<const float*>(&usual)[i];
        }
    }
    const int64_t size = (int64_t)a.R * a.C;
    const float* g = block_of(a.g, a.ld, b, a.count, size) + (int64_t)row * a.C;
    const float* v = a.v ? block_of(a.v, a.v_ld, b, a.count, size) + (int64_t)row * a.C : nullptr;
    half_t* to = a.x + ((int64_t)m * R2 + row) * C2;
    const int32_t cols = row < a.R ? a.C : 0;
    for (int32_t c = lane * kOct; c < C2; c += kWave * kOct) {
        float u[kOct];
#pragma unroll
        for (int j = 0; j < kOct; ++j) u[j] = 0.f;
        if (c < cols) {
            piece_read<kOct, E>(v && !a.nesterov ? v : g, c, cols, u);
            if (a.nesterov) {
                float w[kOct];
                piece_read<kOct, E>(v, c, cols, w);
#pragma unroll
                for (int j = 0; j < kOct; ++j) u[j] += a.mu * w[j];
            }
        }
        half8 hi, lo;
#pragma unroll
        for (int j = 0; j < kOct; ++j) {
            const float w = u[j] * start.first * start.second;
            half_t h, l;
            split(w, &h, &l);
            hi[j] = h;
            lo[j] = l;
        }
        *reinterpret_cast<half8*>(to + c) = hi;
        *reinterpret_cast<half8*>(to + a.plane + c) = lo;
    }
}

struct OrthProduct {
    Operand A, B;
    TileGrid grid;
    uint32_t first_block;
    int32_t K;
    const half_t* add;        // planes as the result's: result = keep * add + times * product, or NULL
    half_t* out;
    int64_t plane;
    int32_t rows2, cols2;     // of the result, padded
    const OrthScales* scales; // one a matrix
    int32_t keep_at, times_at; // which of its floats are keep and times
    float* g;                 // last step: fp32 into the gradient's place
    int64_t ld;
    int32_t R, C, count, first;
};

template <typename S, bool Last>
__global__ __launch_bounds__(S::Threads, 2) void k_orth_product(OrthProduct a) {
    __shared__ __align__(16) char lds[2 * S::Stage];
    int32_t m, ti, tj;
    if (!a.grid.at(a.first_block + blockIdx.x, &m, &ti, &tj)) return;
    const int32_t m0 = ti * S::BM, n0 = tj * S::BN;
    float keep, times, finish[2];
    acc16 acc[S::NI][S::MI];
    product_tile<S>(
        a.A, a.B, m, m0, n0, a.K, lds, acc, [&](int row) { return min(n0 + row, a.B.rows - 1); }, NoMiddle{},
        [&] {
            // a matrix's own factors; 5 x 257 x 1023 in 15 launches 180 us with the call's in their arguments, 189 so, 192 to 194 with these loads before
            // the tiles' or after the sums
            const float* factors = reinterpret_cast<const float*>(a.scales + m);
            keep = factors[a.keep_at];
            times = factors[a.times_at];
            finish[0] = a.scales[m].finish[0];
            finish[1] = a.scales[m].finish[1];
        });
    const bool mirror = a.grid.tn == 0 && ti != tj;
    each_octet<S>(acc, lds, m0, n0, mirror, [&](int32_t row, int32_t col, float* v) {
        if (row >= a.rows2 || col >= a.cols2) return;
        const int64_t at = ((int64_t)m * a.rows2 + row) * a.cols2 + col;
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= times;
        if (a.add) {
            const half8 hi = *reinterpret_cast<const half8*>(a.add + at), lo = *reinterpret_cast<const half8*>(a.add + a.plane + at);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] += keep * ((float)hi[k] + (float)lo[k]);
        }
        if constexpr (Last) {
            if (row >= a.R || col >= a.C) return;
            float* to = block_of(a.g, a.ld, a.first + m, a.count, (int64_t)a.R * a.C) + (int64_t)row * a.C;
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = v[k] * finish[0] * finish[1];
            if (a.C < kOct) piece_put<kOct, Elem<float, true>>(to, col, a.C, v);
            else piece_put<kOct, Elem<float, false>>(to, col, a.C, v);
        } else {
            store_planes<2>(a.out + at, a.plane, v);
        }
    });
}

// steps = 0: u / (|u| + eps) itself
__global__ __launch_bounds__(kThreads) void k_orth_scaled(OrthArgs a, float scale) {
    const uint32_t block = a.first_block + blockIdx.x;
    const int32_t m = (int32_t)(block / a.per_matrix);
    const int64_t size = (int64_t)a.R * a.C, e = (int64_t)(block % a.per_matrix) * kThreads + threadIdx.x;
    double total = a.squares[m * kParts + (threadIdx.x & (kWave - 1))];
    for (int h = kWave / 2; h > 0; h >>= 1) total += __shfl_xor(total, h);
    const double norm = sqrt(total) + (double)a.eps;
    if (e >= size) return;
    float* g = block_of(a.g, a.ld, a.first + m, a.count, size);
    float u = g[e];
    if (a.v) {
        const float w = block_of(a.v, a.v_ld, a.first + m, a.count, size)[e];
        u = a.nesterov ? u + a.mu * w : w;
    }
    g[e] = total == 0.0 ? 0.f : norm < INFINITY ? (float)((double)scale * u / norm) : NAN;
}

// ---- small matrices ----------------------------------------------------------------------------------------------------------
// One workgroup brings a matrix into LDS, in two halves a value, takes all steps there and writes the result: X (short side down the rows) and
// one matrix of the short side's size that holds A and then q A + r A^2.  Results stay in registers until everybody has read what they
// replace.  Pieces of 16 bytes lie within their row xored with fold(row), so that 16 lanes that read one piece of 16 rows, and 32 that read
// 8 bytes each of 4 rows for the transposing read, meet every bank once (rows are odd or even multiples of 128 bytes, and the banks repeat
// after 256).  20 matrices in five steps, here and as products with a launch each: 64 x 64 25 and 72 us; 64 x 256 48, where 64 x 320 takes
// 98 in launches; 128 x 128 72, 192 x 192 in launches 121.
struct SmallArgs {
    OrthArgs o;
    int32_t k2;             // long side, padded
    OrthPolynomial c;
    OrthScales usual;       // for k = 0
};

template <int M2, int KMax, int Waves>
__global__ __launch_bounds__(Waves * kWave) void k_orth_small(SmallArgs a) {
    constexpr int kBlocks = (M2 / 32) * (KMax / 32) / Waves, kGramBlocks = (M2 / 32) * (M2 / 32);
    static_assert(kBlocks * Waves == (M2 / 32) * (KMax / 32) && kGramBlocks <= 2 * Waves, "blocks");
    constexpr int kGramEach = (kGramBlocks + Waves - 1) / Waves, kUnroll = KMax == 64 ? 4 : 1;  // more spills registers
    __shared__ __align__(16) half_t sx[2][M2 * KMax];
    __shared__ __align__(16) half_t sg[2][M2 * M2];
    __shared__ double s_sum[Waves];
    __shared__ OrthScales s_scales;
    const int t = threadIdx.x, lane = t & (kWave - 1), wave = t / kWave, k2 = KMax == M2 ? KMax : a.k2;
    const int32_t m = (int32_t)(a.o.first_block + blockIdx.x), b = a.o.first + m;
    const int64_t size = (int64_t)a.o.R * a.o.C;
    float* g = block_of(a.o.g, a.o.ld, b, a.o.count, size);
    float* v = a.o.v ? block_of(a.o.v, a.o.v_ld, b, a.o.count, size) : nullptr;
    const bool tall = a.o.R > a.o.C;

    auto fold = [](int row, int width) { return (width / 64 & 1) ? ((row & 2) << 1 | (row >> 2 & 3)) : ((row & 3) << 2 | (row >> 2 & 3)); };
    auto at = [&](int row, int col, int width) { return row * width + ((col >> 3 ^ fold(row, width)) << 3) + (col & 7); };
    // 8 k's of row `first + lane % 32`, or of column `first + ..` of X
    auto rows8 = [&](const half_t* p, int first, int kk, int width) {
        return *reinterpret_cast<const half8*>(p + at(first + (lane & 31), kk * 16 + (lane >> 5) * 8, width));
    };
    auto cols8 = [&](const half_t* p, int first, int kk) {
        typedef __attribute__((address_space(3))) short4v lshort;
        const int group = lane >> 4, i = lane & 15, k = kk * 16 + (group >> 1) * 8 + i / 4, col = first + (group & 1) * 16 + (i & 3) * 4;
        const half4 lo = __builtin_bit_cast(half4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lshort*)(p + at(k, col, k2))));
        const half4 hi = __builtin_bit_cast(half4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lshort*)(p + at(k + 4, col, k2))));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    auto times = [](const half8 (&fb)[2], const half8 (&fa)[2], acc16 c) {
        c = __builtin_amdgcn_mfma_f32_32x32x16_f16(fb[0], fa[0], c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x16_f16(fb[0], fa[1], c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x16_f16(fb[1], fa[1], c, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(fb[1], fa[0], c, 0, 0, 0);
    };

    double sum = 0.0;
    for (int32_t r = wave; r < a.o.R; r += Waves)
        for (int32_t c = lane; c < a.o.C; c += kWave) {
            const int64_t e = (int64_t)r * a.o.C + c;
            float u = g[e];
            if (v) {
                const float w = a.o.mu * v[e] + u;
                v[e] = w;
                u = a.o.nesterov ? u + a.o.mu * w : w;
            }
            sum += (double)u * u;
        }
    for (int h = kWave / 2; h > 0; h >>= 1) sum += __shfl_xor(sum, h);
    if (lane == 0) s_sum[wave] = sum;
    for (int e = t * 8; e < M2 * k2; e += Waves * kWave * 8) {
        *reinterpret_cast<half8*>(sx[0] + e) = half8{};
        *reinterpret_cast<half8*>(sx[1] + e) = half8{};
    }
    __syncthreads();
    double total = 0.0;
    for (int w = 0; w < Waves; ++w) total += s_sum[w];
    const OrthStart start = orth_start(total, a.o.eps);
    if (start.k == 0) {
        constexpr int kWords = (int)(sizeof(OrthScales) / sizeof(float));
        for (int i = t; i < kWords; i += Waves * kWave) reinterpret_cast<float*>(&s_scales)[i] = reinterpret_cast<const float*>(&a.usual)[i];
    } else if (t == 0) {
        follow_steps(a.c, start.k, &s_scales);
    }
    for (int32_t r = wave; r < a.o.R; r += Waves)
        for (int32_t c = lane; c < a.o.C; c += kWave) {
            const int64_t e = (int64_t)r * a.o.C + c;
            float u = g[e];
            if (v) u = a.o.nesterov ? u + a.o.mu * v[e] : v[e];
            u = u * start.first * start.second;
            const int to = tall ? at(c, r, k2) : at(r, c, k2);
            split(u, &sx[0][to], &sx[1][to]);
        }
    __syncthreads();

    // p[row][col .. col + 3] <- keep * p + times * acc
    auto put = [&](half_t* p0, half_t* p1, int width, int row0, int col0, const acc16& c, float keep, float times) {
        const int row = row0 + (lane & 31);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int to = at(row, col0 + q * 8 + (lane >> 5) * 4, width);
            half4 hi = *reinterpret_cast<const half4*>(p0 + to), lo = *reinterpret_cast<const half4*>(p1 + to);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float o = times * c[q * 4 + k] + (keep != 0.f ? keep * ((float)hi[k] + (float)lo[k]) : 0.f);
                half_t h, l;
                split(o, &h, &l);
                hi[k] = h;
                lo[k] = l;
            }
            *reinterpret_cast<half4*>(p0 + to) = hi;
            *reinterpret_cast<half4*>(p1 + to) = lo;
        }
    };
    for (int step = 0; step < a.c.steps; ++step) {
        const OrthStep scale = s_scales.step[step];
#pragma unroll
        for (int turn = 0; turn < 2; ++turn) {  // A = X X^T, then q A + r A A
            const half_t *p0 = turn ? sg[0] : sx[0], *p1 = turn ? sg[1] : sx[1];
            const int width = turn ? M2 : k2;
            acc16 c[kGramEach];
#pragma unroll
            for (int n = 0; n < kGramEach; ++n) {
                c[n] = acc16{};
                const int block = wave + n * Waves;
                if (block >= kGramBlocks) continue;
                const int row0 = block / (M2 / 32) * 32, col0 = block % (M2 / 32) * 32;
#pragma unroll kUnroll
                for (int kk = 0; kk < width / 16; ++kk) {
                    const half8 fa[2] = {rows8(p0, row0, kk, width), rows8(p1, row0, kk, width)};
                    const half8 fb[2] = {rows8(p0, col0, kk, width), rows8(p1, col0, kk, width)};
                    c[n] = times(fb, fa, c[n]);
                }
            }
            __syncthreads();
#pragma unroll
            for (int n = 0; n < kGramEach; ++n) {
                const int block = wave + n * Waves;
                if (block >= kGramBlocks) continue;
                put(sg[0], sg[1], M2, block / (M2 / 32) * 32, block % (M2 / 32) * 32, c[n], turn ? scale.poly_keep : 0.f, turn ? scale.poly_times : scale.gram);
            }
            __syncthreads();
        }
        acc16 c[kBlocks];
        const int across = k2 / 32;
#pragma unroll
        for (int n = 0; n < kBlocks; ++n) {
            c[n] = acc16{};
            const int block = wave + n * Waves;
            if (block >= M2 / 32 * across) continue;
            const int row0 = block / across * 32, col0 = block % across * 32;
#pragma unroll kUnroll
            for (int kk = 0; kk < M2 / 16; ++kk) {
                const half8 fa[2] = {rows8(sg[0], row0, kk, M2), rows8(sg[1], row0, kk, M2)};
                const half8 fb[2] = {cols8(sx[0], col0, kk), cols8(sx[1], col0, kk)};
                c[n] = times(fb, fa, c[n]);
            }
        }
        const bool last = step + 1 == a.c.steps;
        const float finish[2] = {s_scales.finish[0], s_scales.finish[1]};
        if (!last) __syncthreads();
#pragma unroll
        for (int n = 0; n < kBlocks; ++n) {
            const int block = wave + n * Waves;
            if (block >= M2 / 32 * across) continue;
            const int row0 = block / across * 32, col0 = block % across * 32;
            if (!last) {
                put(sx[0], sx[1], k2, row0, col0, c[n], scale.keep, scale.times);
                continue;
            }
            const int row = row0 + (lane & 31);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int col = col0 + q * 8 + (lane >> 5) * 4, from = at(row, col, k2);
                const half4 hi = *reinterpret_cast<const half4*>(sx[0] + from), lo = *reinterpret_cast<const half4*>(sx[1] + from);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float o = (scale.times * c[n][q * 4 + k] + scale.keep * ((float)hi[k] + (float)lo[k])) * finish[0] * finish[1];
                    if (row < (tall ? a.o.C : a.o.R) && col + k < (tall ? a.o.R : a.o.C))
                        g[tall ? (int64_t)(col + k) * a.o.C + row : (int64_t)row * a.o.C + col + k] = o;
                }
            }
        }
        __syncthreads();
    }
}

// With a short side of up to 64 few roundings average out and fp32's own error is least: there the small terms are taken along, too
// (30 x 1500: off by 2.5e-6 without them, 2.2e-6 with them, 1.6e-6 in fp32).
template <bool CA, bool CB>
using TileFull = Tile<64, 64, 2, 1, 64, 2, 2, CA, CB, 2, true>;

template <bool CA, bool CB, bool Last>
hipError_t launch_product(const gpga_ctx* c, OrthProduct& a, int32_t matrices, bool lower) {
    const bool small_side = a.rows2 == 64 || a.cols2 == 64;
    const int side = small_side ? 64 : tile_side(c->num_cus, 4, a.rows2, a.cols2, a.K, matrices, lower);
    a.grid.set(a.rows2, a.cols2, side, matrices, lower);
    auto launch = [&](auto tile) {
        typedef decltype(tile) S;
        return launch_blocks(a.grid.blocks(), S::Threads, [&](uint32_t first, dim3 grid) {
            a.first_block = first;
            k_orth_product<S, Last><<<grid, dim3(S::Threads), 0, c->stream>>>(a);
        });
    };
    if (small_side) return launch(TileFull<CA, CB>());
    if (side == 256) return launch(Tile256<2, 2, CA, CB>());
    if (side == 128) return launch(Tile128<2, 2, CA, CB>());
    return launch(Tile64<2, 2, CA, CB>());
}

// Scratch of a call of up to `matrices` matrices at a time.
struct OrthScratch {
    int32_t chunk;
    half_t *x[2], *gram, *poly;
    double* squares;
    OrthScales* scales;
};
OrthScratch carve(const OrthShape& s, char* base, size_t* bytes) {
    const int64_t R2 = padded(s.R), C2 = padded(s.C), m2 = R2 < C2 ? R2 : C2, all = (int64_t)s.n * s.count;
    const int64_t halves = 4 * R2 * C2 + 4 * m2 * m2, most = ((int64_t)4 << 30) / (2 * halves);
    OrthScratch w = {};
    w.chunk = (int32_t)(most < 1 ? 1 : most < all ? most : all);
    size_t used = 0;
    auto take = [&](size_t size) {
        char* p = base ? base + used : nullptr;
        used += (size + 255) / 256 * 256;
        return p;
    };
    for (half_t*& x : w.x) x = reinterpret_cast<half_t*>(take((size_t)w.chunk * R2 * C2 * 4));
    w.gram = reinterpret_cast<half_t*>(take((size_t)w.chunk * m2 * m2 * 4));
    w.poly = reinterpret_cast<half_t*>(take((size_t)w.chunk * m2 * m2 * 4));
    w.squares = reinterpret_cast<double*>(take((size_t)w.chunk * kParts * sizeof(double)));
    w.scales = reinterpret_cast<OrthScales*>(take((size_t)w.chunk * sizeof(OrthScales)));
    *bytes = used;
    return w;
}

// Matrices that one workgroup holds.
bool small_fits(const OrthShape& s) {
    const int32_t R2 = padded(s.R), C2 = padded(s.C), m2 = R2 < C2 ? R2 : C2, k2 = R2 < C2 ? C2 : R2;
    return m2 == 64 ? k2 <= 256 : k2 == 128;
}

}  // namespace

size_t orthogonalize_scratch(const OrthShape& s) {
    size_t bytes;
    carve(s, nullptr, &bytes);
    return bytes;
}

double orthogonalize_bound(int32_t steps, const float* coefficients) {
    double most = 1.0, worst = 1.0;
    for (int32_t k = 0; k < steps; ++k) {
        most = odd_max(coefficients[0], coefficients[1], coefficients[2], most) * 1.001;
        worst = std::fmax(worst, most);
    }
    return worst;
}

hipError_t launch_orthogonalize(const gpga_ctx* c, const OrthShape& s, int64_t off, float* v, float mu, bool nesterov, int32_t steps,
                                const float* coefficients, float eps, float scale, void* scratch) {
    size_t bytes;
    const OrthScratch w = carve(s, static_cast<char*>(scratch), &bytes);
    const int32_t R2 = padded(s.R), C2 = padded(s.C), m2 = R2 < C2 ? R2 : C2;
    const bool tall = s.R > s.C;
    const int64_t all = (int64_t)s.n * s.count;
    const OrthPolynomial polynomial = {coefficients[0], coefficients[1], coefficients[2], scale, steps};
    OrthScales usual = {};
    follow_steps(polynomial, 0, &usual);
    for (int64_t b0 = 0; b0 < all; b0 += w.chunk) {
        const int32_t matrices = (int32_t)(all - b0 < w.chunk ? all - b0 : w.chunk);
        OrthArgs a = {};
        a.g = c->g + off;
        a.v = v;
        a.ld = c->ld;
        a.v_ld = (int64_t)s.count * s.R * s.C;
        a.R = s.R;
        a.C = s.C;
        a.count = s.count;
        a.first = (int32_t)b0;
        a.mu = mu;
        a.nesterov = nesterov && v;
        a.eps = eps;
        a.squares = w.squares;
        a.x = w.x[0];
        a.plane = (int64_t)matrices * R2 * C2;
        a.scales = w.scales;
        hipError_t e = hipSuccess;
        const bool small = steps > 0 && small_fits(s);
        if (!small) {
            e = launch_blocks((uint64_t)kParts * matrices, kThreads, [&](uint32_t first, dim3 grid) {
                a.first_block = first;
                k_orth_norm<<<grid, dim3(kThreads), 0, c->stream>>>(a);
            });
            if (e != hipSuccess) return e;
        }
        if (steps == 0) {
            a.per_matrix = (uint32_t)(((int64_t)s.R * s.C + kThreads - 1) / kThreads);
            e = launch_blocks((uint64_t)a.per_matrix * matrices, kThreads, [&](uint32_t first, dim3 grid) {
                a.first_block = first;
                k_orth_scaled<<<grid, dim3(kThreads), 0, c->stream>>>(a, scale);
            });
            if (e != hipSuccess) return e;
            continue;
        }
        if (small) {
            SmallArgs f = {a, R2 > C2 ? R2 : C2, polynomial, usual};
            const int32_t waves = f.k2 > 64 ? 8 : 4;
            e = launch_blocks((uint64_t)matrices, waves * kWave, [&](uint32_t first, dim3 grid) {
                f.o.first_block = first;
                if (f.k2 == 64) k_orth_small<64, 64, 4><<<grid, dim3(256), 0, c->stream>>>(f);
                else if (m2 == 64) k_orth_small<64, 256, 8><<<grid, dim3(512), 0, c->stream>>>(f);
                else k_orth_small<128, 128, 8><<<grid, dim3(512), 0, c->stream>>>(f);
            });
            if (e != hipSuccess) return e;
            continue;
        }
        a.per_matrix = (uint32_t)(R2 / (kThreads / kWave));
        e = launch_blocks((uint64_t)a.per_matrix * matrices, kThreads, [&](uint32_t first, dim3 grid) {
            a.first_block = first;
            if (s.C < kOct) k_orth_pack<Elem<float, true>><<<grid, dim3(kThreads), 0, c->stream>>>(a, polynomial, usual);
            else k_orth_pack<Elem<float, false>><<<grid, dim3(kThreads), 0, c->stream>>>(a, polynomial, usual);
        });
        if (e != hipSuccess) return e;
        for (int32_t k = 0; k < steps; ++k) {
            const Operand x = {w.x[k & 1], (int64_t)matrices * R2 * C2, (int64_t)R2 * C2, C2, R2};
            const Operand gram = {w.gram, (int64_t)matrices * m2 * m2, (int64_t)m2 * m2, m2, m2}, poly = {w.poly, gram.plane, gram.batch, m2, m2};
            OrthProduct o = {};
            o.A = o.B = x;
            o.K = tall ? R2 : C2;
            o.out = w.gram;
            o.plane = gram.plane;
            o.rows2 = o.cols2 = m2;
            constexpr int32_t kStep = (int32_t)(sizeof(OrthStep) / sizeof(float));
            auto factor = [&](size_t member) { return k * kStep + (int32_t)(member / sizeof(float)); };
            o.scales = w.scales;
            o.keep_at = o.times_at = factor(offsetof(OrthStep, gram));
            e = tall ? launch_product<true, true, false>(c, o, matrices, true) : launch_product<false, false, false>(c, o, matrices, true);
            if (e != hipSuccess) return e;
            // q A + r A A
            o.A = o.B = gram;
            o.K = m2;
            o.add = w.gram;
            o.out = w.poly;
            o.keep_at = factor(offsetof(OrthStep, poly_keep));
            o.times_at = factor(offsetof(OrthStep, poly_times));
            e = launch_product<false, false, false>(c, o, matrices, true);
            if (e != hipSuccess) return e;
            const bool last = k + 1 == steps;
            o = {};
            o.A = tall ? x : poly;
            o.B = tall ? poly : x;
            o.K = m2;
            o.add = w.x[k & 1];
            o.out = w.x[(k + 1) & 1];
            o.plane = x.plane;
            o.rows2 = R2;
            o.cols2 = C2;
            o.scales = w.scales;
            o.keep_at = factor(offsetof(OrthStep, keep));
            o.times_at = factor(offsetof(OrthStep, times));
            o.g = c->g + off;
            o.ld = c->ld;
            o.R = s.R;
            o.C = s.C;
            o.count = s.count;
            o.first = (int32_t)b0;
            if (last) e = tall ? launch_product<false, false, true>(c, o, matrices, false) : launch_product<false, true, true>(c, o, matrices, false);
            else e = tall ? launch_product<false, false, false>(c, o, matrices, false) : launch_product<false, true, false>(c, o, matrices, false);
            if (e != hipSuccess) return e;
        }
    }
    return hipSuccess;
}
