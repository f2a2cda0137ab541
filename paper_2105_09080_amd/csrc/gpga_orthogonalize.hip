// Orthogonalised updates of the nodes' matrices (include/gpga.h): the gradient of a matrix, or its running sum, is brought near the closest
// matrix with orthonormal rows (or columns) by a few steps of Newton-Schulz iteration,
//
//   X0 = U / (|U|_F + eps),  X <- p X + (q A + r A^2) X  with A = X X^T  (or, tall, X <- p X + X (q A + r A^2) with A = X^T X),
//
// which maps every singular value s to p s + q s^3 + r s^5 and leaves the singular vectors.  A has the shorter side's size.  Small singular
// values grow by p a step, and so do errors in them: everything is held in two halves (22 bits), fp32's precision, three matrix
// instructions a step (gpga_product.hpp).  Singular values are at most 1 to begin with; the host follows the largest that a step can make
// of them, so all scales are known constants.
#include "gpga_pack.hpp"

#include <cmath>

namespace {

constexpr int kThreads = 256;
constexpr int kParts = 64;  // parts of a matrix's sum of squares

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
    float x_up;
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

// u / (|u| + eps) as halves, a wavefront a row.
template <typename E>
__global__ __launch_bounds__(kThreads) void k_orth_pack(OrthArgs a) {
    const uint32_t block = a.first_block + blockIdx.x;
    const int32_t m = (int32_t)(block / a.per_matrix), b = a.first + m, lane = threadIdx.x & (kWave - 1);
    const int32_t row = (int32_t)(block % a.per_matrix) * (kThreads / kWave) + threadIdx.x / kWave, R2 = padded(a.R), C2 = padded(a.C);
    double total = a.squares[m * kParts + lane];
    for (int h = kWave / 2; h > 0; h >>= 1) total += __shfl_xor(total, h);
    const double norm = sqrt(total) + (double)a.eps;
    const float inv = total == 0.0 ? 0.f : norm < INFINITY ? (float)(1.0 / norm) : NAN;
    // the reciprocal of a norm below 2^-126 is no float: such a gradient is scaled up first
    const float first = total < 1e-60 ? 0x1p100f : 1.f, second = total < 1e-60 ? (total == 0.0 ? 0.f : (float)(0x1p-100 / norm)) : inv;
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
            const float w = u[j] * first * second * a.x_up;
            hi[j] = (half_t)w;
            lo[j] = (half_t)(w - (float)hi[j]);
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
    float keep, times;
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
    acc16 acc[S::NI][S::MI];
    product_tile<S>(a.A, a.B, m, m0, n0, a.K, lds, acc, [&](int row) { return min(n0 + row, a.B.rows - 1); });
    const bool mirror = a.grid.tn == 0 && ti != tj;
    each_octet<S>(acc, lds, m0, n0, mirror, [&](int32_t row, int32_t col, float* v) {
        if (row >= a.rows2 || col >= a.cols2) return;
        const int64_t at = ((int64_t)m * a.rows2 + row) * a.cols2 + col;
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= a.times;
        if (a.add) {
            const half8 hi = *reinterpret_cast<const half8*>(a.add + at), lo = *reinterpret_cast<const half8*>(a.add + a.plane + at);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] += a.keep * ((float)hi[k] + (float)lo[k]);
        }
        if constexpr (Last) {
            if (row >= a.R || col >= a.C) return;
            float* to = block_of(a.g, a.ld, a.first + m, a.count, (int64_t)a.R * a.C) + (int64_t)row * a.C;
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

template <bool CA, bool CB, bool Last>
hipError_t launch_product(const gpga_ctx* c, OrthProduct& a, int32_t matrices, bool lower) {
    const int side = tile_side(c->num_cus, 4, a.rows2, a.cols2, a.K, matrices, lower);
    a.grid.set(a.rows2, a.cols2, side, matrices, lower);
    auto launch = [&](auto tile) {
        typedef decltype(tile) S;
        return launch_blocks(a.grid.blocks(), S::Threads, [&](uint32_t first, dim3 grid) {
            a.first_block = first;
            k_orth_product<S, Last><<<grid, dim3(S::Threads), 0, c->stream>>>(a);
        });
    };
    if (side == 256) return launch(Tile256<2, 2, CA, CB>());
    if (side == 128) return launch(Tile128<2, 2, CA, CB>());
    return launch(Tile64<2, 2, CA, CB>());
}

// Scratch of a call of up to `matrices` matrices at a time.
struct OrthScratch {
    int32_t chunk;
    half_t *x[2], *gram, *poly;
    double* squares;
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
    *bytes = used;
    return w;
}

// Power of two that brings values of at most `bound` to 2^14 or below.
float up_for(double bound) {
    int e;
    std::frexp(bound, &e);
    return (float)std::ldexp(1.0, 14 - e);
}

// Largest |a s + b s^3 + c s^5| over 0 <= s <= most.
double odd_max(double a, double b, double c, double most) {
    auto f = [&](double s) { return std::fabs(s * (a + s * s * (b + s * s * c))); };
    double best = f(most);
    // a + 3 b z + 5 c z^2 = 0, z = s^2
    const double d = 9.0 * b * b - 20.0 * a * c;
    double z[2] = {-1.0, -1.0};
    if (c != 0.0 && d >= 0.0) {
        z[0] = (-3.0 * b + std::sqrt(d)) / (10.0 * c);
        z[1] = (-3.0 * b - std::sqrt(d)) / (10.0 * c);
    } else if (c == 0.0 && b != 0.0) {
        z[0] = -a / (3.0 * b);
    }
    for (double v : z)
        if (v > 0.0 && v < most * most) best = std::fmax(best, f(std::sqrt(v)));
    return best;
}
// Largest |b z + c z^2| over 0 <= z <= most.
double even_max(double b, double c, double most) {
    double best = std::fabs(b * most + c * most * most);
    if (c != 0.0) {
        const double z = -b / (2.0 * c);
        if (z > 0.0 && z < most) best = std::fmax(best, std::fabs(b * z + c * z * z));
    }
    return best;
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
    const double p = coefficients[0], q = coefficients[1], r = coefficients[2];
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
        double most = 1.0;
        float x_up = up_for(1.0);
        a.x_up = x_up;
        hipError_t e = launch_blocks((uint64_t)kParts * matrices, kThreads, [&](uint32_t first, dim3 grid) {
            a.first_block = first;
            k_orth_norm<<<grid, dim3(kThreads), 0, c->stream>>>(a);
        });
        if (e != hipSuccess) return e;
        if (steps == 0) {
            a.per_matrix = (uint32_t)(((int64_t)s.R * s.C + kThreads - 1) / kThreads);
            e = launch_blocks((uint64_t)a.per_matrix * matrices, kThreads, [&](uint32_t first, dim3 grid) {
                a.first_block = first;
                k_orth_scaled<<<grid, dim3(kThreads), 0, c->stream>>>(a, scale);
            });
            if (e != hipSuccess) return e;
            continue;
        }
        a.per_matrix = (uint32_t)(R2 / (kThreads / kWave));
        e = launch_blocks((uint64_t)a.per_matrix * matrices, kThreads, [&](uint32_t first, dim3 grid) {
            a.first_block = first;
            if (s.C < kOct) k_orth_pack<Elem<float, true>><<<grid, dim3(kThreads), 0, c->stream>>>(a);
            else k_orth_pack<Elem<float, false>><<<grid, dim3(kThreads), 0, c->stream>>>(a);
        });
        if (e != hipSuccess) return e;
        for (int32_t k = 0; k < steps; ++k) {
            const Operand x = {w.x[k & 1], (int64_t)matrices * R2 * C2, (int64_t)R2 * C2, C2, R2};
            const Operand gram = {w.gram, (int64_t)matrices * m2 * m2, (int64_t)m2 * m2, m2, m2}, poly = {w.poly, gram.plane, gram.batch, m2, m2};
            const float gram_up = up_for(most * most * 1.001), poly_up = up_for(even_max(q, r, most * most) * 1.001 + 1e-30);
            OrthProduct o = {};
            o.A = o.B = x;
            o.K = tall ? R2 : C2;
            o.out = w.gram;
            o.plane = gram.plane;
            o.rows2 = o.cols2 = m2;
            o.times = (float)((double)gram_up / x_up / x_up);
            e = tall ? launch_product<true, true, false>(c, o, matrices, true) : launch_product<false, false, false>(c, o, matrices, true);
            if (e != hipSuccess) return e;
            // q A + r A A
            o.A = o.B = gram;
            o.K = m2;
            o.add = w.gram;
            o.out = w.poly;
            o.keep = (float)(q * poly_up / gram_up);
            o.times = (float)(r * poly_up / gram_up / gram_up);
            e = launch_product<false, false, false>(c, o, matrices, true);
            if (e != hipSuccess) return e;
            const bool last = k + 1 == steps;
            most = odd_max(p, q, r, most) * 1.001;
            const double out_up = last ? (double)scale : (double)up_for(most);
            o = {};
            o.A = tall ? x : poly;
            o.B = tall ? poly : x;
            o.K = m2;
            o.add = w.x[k & 1];
            o.out = w.x[(k + 1) & 1];
            o.plane = x.plane;
            o.rows2 = R2;
            o.cols2 = C2;
            o.keep = (float)(p * out_up / x_up);
            o.times = (float)(out_up / x_up / poly_up);
            o.g = c->g + off;
            o.ld = c->ld;
            o.R = s.R;
            o.C = s.C;
            o.count = s.count;
            o.first = (int32_t)b0;
            if (last) e = tall ? launch_product<false, false, true>(c, o, matrices, false) : launch_product<false, true, true>(c, o, matrices, false);
            else e = tall ? launch_product<false, false, false>(c, o, matrices, false) : launch_product<false, true, false>(c, o, matrices, false);
            if (e != hipSuccess) return e;
            x_up = (float)out_up;
        }
    }
    return hipSuccess;
}
