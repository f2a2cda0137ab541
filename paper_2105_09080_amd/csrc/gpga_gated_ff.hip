// Gated feed-forward block on the nodes' own matrices (include/gpga.h), forward and backward.
//
//   a = x Wg^T, b = x Wu^T, h = act(a) b, y = h Wd^T                     x, y: T x D a node; a, b, h: T x F
//   dh = dy Wd, da = dh b act'(a), db = dh act(a), dx = da Wg + db Wu,
//   dWg = da^T x, dWu = db^T x, dWd = dy^T h
//
// The products run on the matrix units (gpga_product.hpp) from halves with power-of-two scales.  Which operands get two halves follows
// from the result: what is fp32 in the end (gradients of parameters; everything with fp32 activations) gets two wherever an operand is
// not exact in one; what is rounded to fp16 gets two for one operand of each product and one (2^-11) for the other, and is off by up to root 2
// of its own rounding (dx 2.9e-4 in the 2-norm, 2.1e-4 with two everywhere, which took 1693 us in place of 1402 for 2 x 2048 tokens, 2048 x
// 5632; forward 1012 in place of 881 for 8 x 4096, 768 x 2048); what is rounded to bf16 (by up to 2^-8) gets one everywhere, and is off by
// 1.02 to 1.03 of its rounding.  Up to 64 tokens: bf16 pieces, see there.  Callers who want fp32's bits hand over fp32 activations.
// Scales: rows of x and of the matrices by their largest value; h, da and db, which are rounded in the epilogue that makes them, by
// bounds that are known before (forward Cauchy-Schwarz for a and b, element by element; backward the largest |act(a)| and |b| of the token and
// the sum of |dy| for dh, each of the three by its own): some 2^8 .. 2^14 above typical values, which halves' 29 binades below 2^15 have room for.
#include "gpga_pack.hpp"

namespace {

constexpr int kThreads = 256;
constexpr int kPackRows = kThreads / kWave;  // a wavefront a row

// ---- activation functions -------------------------------------------------------------------------------------------------
// silu(v) = v s, s = 1 / (1 + exp(-v)); silu' = s + v s (1 - s).  gelu(v) = v P, P = (1 + erf(v / sqrt 2)) / 2; gelu' = P + v exp(-v^2/2) /
// sqrt(2 pi).  |act(v)| <= |v|, |act'| <= 1.13.  erf by Abramowitz and Stegun, Handbook of Mathematical Functions, 7.1.26: with t = 1 /
// (1 + 0.3275911 z), z >= 0, 1 - erf(z) = (a1 t + .. + a5 t^5) exp(-z^2) to 1.5e-7, what a rounding of 1 + erf to fp32 costs, and its
// exponential is the slope's; the library's erff took a third of the product's time (8 x 8192 tokens, F = 4096).
template <int Act>
__device__ __forceinline__ void act_both(float v, float* value, float* slope) {
    if constexpr (Act == GPGA_SILU) {
        const float e = __expf(-v), s = __builtin_amdgcn_rcpf(1.f + e);
        *value = v * s;
        *slope = s + *value * (e > 1e30f ? 1.f : e * s);
    } else {
        const float t = __builtin_amdgcn_rcpf(1.f + 0.231641888f * fabsf(v)), e = __expf(-0.5f * v * v);  // 0.3275911 / sqrt 2
        const float tail = 0.5f * e * t * (0.254829592f + t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f))));
        const float p = v < 0.f ? tail : 1.f - tail;
        *value = v * p;
        *slope = p + v * (e * 0.39894228040143268f);
    }
}
template <int Act>
__device__ __forceinline__ float act_value(float v) {
    float value, slope;
    act_both<Act>(v, &value, &slope);
    return value;
}

// Another Slot for another maximum without a barrier between.
template <int Slot = 0>
__device__ __forceinline__ float block_max(float m) {
    __shared__ float s[kPackRows];
    m = wave_all<kWave>(m, max_nan);
    if ((threadIdx.x & (kWave - 1)) == 0) s[threadIdx.x / kWave] = m;
    __syncthreads();
    return max_nan(max_nan(s[0], s[1]), max_nan(s[2], s[3]));
}

// ---- rows as halves -------------------------------------------------------------------------------------------------------
// The three matrices of every node: rows of gate, up (D long) and down (F long), each with a scale of its own, or gate and up
// with one scale a node.
//
// Forward, what h is scaled by: |a_f| <= |x| |wg_f| < 2^(ex + eg_f), |b_f| < 2^(ex + eu_f) by Cauchy-Schwarz, with the exponents of the 2-norms of
// the token and of the matrices' rows f.  2^-(2 ex + eg_f + eu_f) h_f is below 1 whatever the rows' sizes are beside each other's; what depends on f goes
// into column f of the down matrix before that gets scales of its own.
struct PackMatrices {
    const float* gate;
    const float* up;
    const float* down;
    int64_t ldx;
    int32_t D, F;
    half_t *gu, *wd;              // planes: (n, 2 F', D') and (n, D', F'), ' padded
    int64_t gu_plane, wd_plane;
    float *gu_inv, *wd_inv;       // n x 2F', n x D'
    float* gu_up;                 // forward: n x 2F', 2^-eg and 2^(15-eu); 0 for a row of zeros
    float* fold;                  // forward: n x F', 2^(eg + eu)
    const float* node_max;        // backward: largest |gate| and largest |up| of a node, n x 2 x kMaxParts parts
    uint32_t gu_blocks, per_node, first_block;
};
constexpr int kMaxParts = 256;

// Forward: workgroup by workgroup two rows of gate and the same two of up, with scales by row.
template <typename E, int P>
__device__ __forceinline__ void pack_gate_up_rows(const PackMatrices& a, uint32_t block) {
    static_assert(kPackRows == 4, "two rows of each");
    __shared__ float s[kPackRows];
    const int64_t node = block / a.gu_blocks;
    const int32_t D2 = padded(a.D), F2 = padded(a.F), wave = threadIdx.x / kWave, f = (int32_t)(block % a.gu_blocks) * 2 + (wave & 1);
    const int64_t row = node * 2 * F2 + (wave < 2 ? f : F2 + f);
    const float* from = (wave < 2 ? a.gate : a.up) + node * a.ldx + (int64_t)f * a.D;
    const RowStat r = pack_row<E, P>(from, f < a.F ? a.D : 0, D2, true, {}, a.gu + row * D2, a.gu_plane);
    if ((threadIdx.x & (kWave - 1)) == 0) {
        a.gu_inv[row] = r.down;
        s[wave] = norm_exponent(r);
    }
    __syncthreads();
    if (threadIdx.x >= 2) return;
    const int64_t first = (int64_t)(block % a.gu_blocks) * 2 + threadIdx.x;
    const float eg = s[threadIdx.x], eu = s[threadIdx.x + 2], both = eg + eu;
    // a float's range, and room in it for the down matrix's values: beyond it up's part is what is left
    const float e = both != both || both == -INFINITY ? both : fminf(fmaxf(both, -112.f), 120.f);
    a.fold[node * F2 + first] = power_of_two(e);
    a.gu_up[node * 2 * F2 + first] = power_of_two(-eg);
    a.gu_up[node * 2 * F2 + F2 + first] = e == -INFINITY ? 0.f : ldexpf(power_of_two(eg), (int)(e != e ? 0.f : 15.f - e));
}

// Backward: the scale of a node's gate (0) or up (1) matrix.
__device__ __forceinline__ Scale matrix_scale(const float* node_max, int64_t node, int which) {
    const float* part = node_max + (node * 2 + which) * kMaxParts + (threadIdx.x & (kWave - 1));
    return scale_for(wave_all<kWave>(max_nan(max_nan(part[0], part[64]), max_nan(part[128], part[192])), max_nan));
}

// Workgroup `in` of a node's for gate and up, with one scale each.
template <typename E, int P>
__device__ __forceinline__ void pack_gate_up(const PackMatrices& a, int64_t node, int32_t in) {
    const int32_t D2 = padded(a.D), F2 = padded(a.F), row = in * kPackRows + threadIdx.x / kWave, f = row < F2 ? row : row - F2;
    const float* from = (row < F2 ? a.gate : a.up) + node * a.ldx + (int64_t)f * a.D;
    pack_row<E, P>(from, f < a.F ? a.D : 0, D2, false, matrix_scale(a.node_max, node, row >= F2), a.gu + (node * 2 * F2 + row) * D2, a.gu_plane);
}
// And for the down matrix, with scales by row.
template <typename E, int P, typename Fold = NoFold>
__device__ __forceinline__ void pack_down(const PackMatrices& a, int64_t node, int32_t in, Fold&& fold = {}) {
    const int32_t D2 = padded(a.D), F2 = padded(a.F), row = in * kPackRows + threadIdx.x / kWave;
    const RowStat r = pack_row<E, P>(a.down + node * a.ldx + (int64_t)row * a.F, row < a.D ? a.F : 0, F2, true, {}, a.wd + (node * D2 + row) * F2,
                                     a.wd_plane, fold);
    if ((threadIdx.x & (kWave - 1)) == 0) a.wd_inv[node * D2 + row] = r.down;
}
// Forward, second: with 2^(eg + eu) in its columns.
template <typename E, int P>
__global__ __launch_bounds__(kThreads) void k_ff_pack_down_folded(PackMatrices a) {
    const uint32_t block = a.first_block + blockIdx.x;
    const int64_t node = block / a.per_node;
    const float* fold = a.fold + node * padded(a.F);
    pack_down<E, P>(a, node, (int32_t)(block % a.per_node), [&](int32_t c, float* v) {
#pragma unroll
        for (int j = 0; j < kOct; ++j) v[j] *= fold[c + j];
    });
}

// Backward, first: the down matrix, and the largest |gate| and the largest |up| of a node in kMaxParts parts each.
template <typename E>
__global__ __launch_bounds__(kThreads) void k_ff_pack_down(PackMatrices a, float* parts) {
    typedef float vec __attribute__((ext_vector_type(4), aligned(4)));
    const uint32_t block = a.first_block + blockIdx.x;
    const int64_t node = block / a.per_node;
    const int32_t p = (int32_t)(block % a.per_node);
    if (p >= kMaxParts) {
        pack_down<E, 2>(a, node, p - kMaxParts);
        return;
    }
    const float* from[2] = {a.gate + node * a.ldx, a.up + node * a.ldx};
    float m[2] = {0.f, 0.f};
    const int64_t count = (int64_t)a.F * a.D, fours = count / 4, at = (int64_t)p * kThreads + threadIdx.x;
#pragma unroll 2
    for (int64_t e = at; e < fours; e += (int64_t)kMaxParts * kThreads)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const vec v = *(reinterpret_cast<const vec*>(from[k]) + e);
            m[k] = max_nan(m[k], max_nan(max_nan(fabsf(v[0]), fabsf(v[1])), max_nan(fabsf(v[2]), fabsf(v[3]))));
        }
    if (at < count % 4) {
        m[0] = max_nan(m[0], fabsf(from[0][fours * 4 + at]));
        m[1] = max_nan(m[1], fabsf(from[1][fours * 4 + at]));
    }
    m[0] = block_max<0>(m[0]);
    m[1] = block_max<1>(m[1]);
    if (threadIdx.x == 0) {
        parts[node * 2 * kMaxParts + p] = m[0];
        parts[(node * 2 + 1) * kMaxParts + p] = m[1];
    }
}

// Rows of activations of a chunk of tokens: kRowsEach for each of a workgroup's wavefronts.
constexpr int kRowsEach = 4;
struct PackRows {
    const void* src;
    int64_t ld, node;          // elements between rows, between nodes
    int32_t rows, cols;        // real ones of a node
    half_t* dst;               // (n, rows', cols')
    int64_t plane;
    float* inv;                // n x rows'
    uint32_t per_node, first_block;
};

// Forward, first: gate and up (the first `matrix_blocks` workgroups), and x as halves with 2^-ex and 2^ex of its rows.
template <typename E, int P, int PW>
__global__ __launch_bounds__(kThreads) void k_ff_pack_x(PackMatrices w, uint32_t matrix_blocks, PackRows a, float* h_up, float* h_inv) {
    const int32_t cols2 = padded(a.cols), lane = threadIdx.x & (kWave - 1), rows2 = padded(a.rows);
    uint32_t block = a.first_block + blockIdx.x;
    if (block < matrix_blocks) {
        pack_gate_up_rows<Elem<float, E::kNarrow>, PW>(w, block);
        return;
    }
    block -= matrix_blocks;
    const int64_t node = block / a.per_node;
    for (int k = 0; k < kRowsEach; ++k) {
        const int32_t row = ((int32_t)(block % a.per_node) * kRowsEach + k) * kPackRows + threadIdx.x / kWave;
        const int64_t at = node * rows2 + row;
        const typename E::mem* from = static_cast<const typename E::mem*>(a.src) + node * a.node + (int64_t)row * a.ld;
        const RowStat r = pack_row<E, P>(from, row < a.rows ? a.cols : 0, cols2, true, {}, a.dst + at * cols2, a.plane);
        if (lane == 0) {
            const float e = norm_exponent(r);
            a.inv[at] = r.down;
            h_up[at] = power_of_two(-e);
            h_inv[at] = power_of_two(e);
        }
    }
}

// The largest |a| of a row, and the largest a: |act(a)| is at most a where a > 0 and min(|a| / 2, 0.28) where not.
struct RowRange {
    float size, most;
    __device__ __forceinline__ float act_bound() const { return size < INFINITY ? fmaxf(most, fminf(size * 0.5f, 0.28f)) : size; }
};
template <typename E>
__device__ __forceinline__ RowRange row_range(const typename E::mem* row, int32_t cols) {
    RowRange r = {0.f, 0.f};
    for (int32_t c = (int32_t)(threadIdx.x & (kWave - 1)) * kOct; c < cols; c += kWave * kOct) {
        float v[kOct];
        piece_read<kOct, E>(row, c, cols, v);
#pragma unroll
        for (int j = 0; j < kOct; ++j) {
            r.size = max_nan(r.size, fabsf(v[j]));
            r.most = fmaxf(r.most, v[j]);
        }
    }
    return {wave_all<kWave>(r.size, max_nan), wave_max<kWave>(r.most)};
}

// Backward, what a token's rows of da, db and h are scaled by, each by a bound of its own: |dh| <= sum |dy| |w|, |da| <= 1.14 |dh| max |b|,
// |db| <= |dh| max |act(a)|, |h| <= max |act(a)| max |b|.  dx adds da Wg and db Wu in one sum: after the first the sums are brought to the second's
// scale, by 2^-120 to 2^70: sums of up to 2^51 stay in fp32's range.  Of scales further apart the finer one is made coarser.
struct TokenScales {
    float *da_up, *da_inv, *db_up, *db_inv, *h_up, *h_inv;  // a power of two, its inverse (0: the row is zeros)
    float* dx_middle;                                      // factor of the sums of da Wg
    int32_t* dx_exp;                                       // dx = 2^dx_exp times the sums
    float* part;                                           // n x 3 x workgroups of a node: largest |x| da_inv, |x| db_inv, |dy| h_inv
};
__device__ __forceinline__ int exponent_of(float power) { return (int)(__float_as_uint(power) >> 23) - 127; }

// Backward, second: gate and up by their largest values; dy times the scales of the down matrix's rows as halves, and its tokens' scales.
// For the products over tokens da = da' / up and so on leaves factors that go into the other operand (k_ff_pack_tokens).
template <typename E, int P>
__global__ __launch_bounds__(kThreads) void k_ff_pack_dy(PackMatrices w, uint32_t matrix_blocks, PackRows a, const void* x, const void* hidden, int64_t hidden_node,
                                                         TokenScales t) {
    typedef typename E::mem M;
    const int32_t cols2 = padded(a.cols), lane = threadIdx.x & (kWave - 1), rows2 = padded(a.rows);
    uint32_t block = a.first_block + blockIdx.x;
    if (block < matrix_blocks) {
        pack_gate_up<Elem<float, E::kNarrow>, P>(w, block / w.gu_blocks, (int32_t)(block % w.gu_blocks));
        return;
    }
    block -= matrix_blocks;
    const int64_t node = block / a.per_node;
    float p[3] = {0.f, 0.f, 0.f};
    {
        const int32_t row = (int32_t)(block % a.per_node) * kPackRows + threadIdx.x / kWave;
        const bool real = row < a.rows;
        const int64_t from = node * a.node + (int64_t)row * a.ld, at = node * rows2 + row;
        const Scale gate = matrix_scale(w.node_max, node, 0), up = matrix_scale(w.node_max, node, 1);
        float xm = 0.f, ym = 0.f, vm = 0.f, bm = 0.f;
        if (real) {
            const M* h = static_cast<const M*>(hidden) + node * hidden_node + (int64_t)row * 2 * w.F;
            vm = row_range<E>(h, w.F).act_bound();
            bm = row_max<E>(h + w.F, w.F);
            if (!(fmaxf(vm, bm) < INFINITY) || vm != vm || bm != bm) vm = bm = NAN;  // the token has no gradient then
            xm = row_max<E>(static_cast<const M*>(x) + from, a.cols);
            ym = row_max<E>(static_cast<const M*>(a.src) + from, a.cols);
        }
        const float* inv = w.wd_inv + node * cols2;
        const RowStat r = pack_row<E, P>(static_cast<const M*>(a.src) + from, real ? a.cols : 0, cols2, true, {}, a.dst + at * cols2, a.plane,
                                         [&](int32_t c, float* v) {
#pragma unroll
                                             for (int j = 0; j < kOct; ++j) v[j] *= inv[c + j];
                                         });
        const float dh = r.sum * r.down * 32768.f * 1.0001f;
        Scale sa = scale_for(dh * (1.14f * bm)), sb = scale_for(dh * vm);
        const Scale sh = scale_for(vm * bm);
        const bool no_a = sa.down == 0.f || gate.down == 0.f, no_b = sb.down == 0.f || up.down == 0.f;
        const bool bad = sa.up != sa.up || sb.up != sb.up || gate.up != gate.up || up.up != up.up;
        int ea = exponent_of(sa.up), eb = exponent_of(sb.up), apart = eb + exponent_of(up.up) - ea - exponent_of(gate.up);
        if (!bad && !no_a && !no_b) {
            constexpr int kMost = 70, kLeast = -120;
            if (apart > kMost) eb = max(eb - (apart - kMost), -126);
            if (apart < kLeast) ea = max(ea - (kLeast - apart), -126);
            apart = min(max(apart, kLeast), kMost);
            sa = {ldexpf(1.f, ea), ldexpf(1.f, -ea)};
            sb = {ldexpf(1.f, eb), ldexpf(1.f, -eb)};
        }
        if (lane == 0) {
            a.inv[at] = r.down;
            t.da_up[at] = sa.up;
            t.da_inv[at] = sa.down;
            t.db_up[at] = sb.up;
            t.db_inv[at] = sb.down;
            t.h_up[at] = sh.up;
            t.h_inv[at] = sh.down;
            t.dx_middle[at] = bad ? NAN : no_a ? 0.f : no_b ? 1.f : ldexpf(1.f, apart);
            t.dx_exp[at] = bad ? 0 : no_b ? -ea - exponent_of(gate.up) : -eb - exponent_of(up.up);
        }
        p[0] = xm * sa.down;
        p[1] = xm * sb.down;
        p[2] = ym * sh.down;
    }
    __shared__ float s[3][kPackRows];
    if (lane == 0) {
#pragma unroll
        for (int k = 0; k < 3; ++k) s[k][threadIdx.x / kWave] = p[k];
    }
    __syncthreads();
    if (threadIdx.x < 3) {
        const float* q = s[threadIdx.x];
        t.part[(node * 3 + threadIdx.x) * a.per_node + block % a.per_node] = max_nan(max_nan(q[0], q[1]), max_nan(q[2], q[3]));
    }
}

// x / up of da, x / up of db or dy / up of h of every token as halves with one scale a node, a third of the workgroups each.
struct PackTokens {
    PackRows of[3];            // inv: one a node
    const float* row_inv[3];
    const float* part;
    uint32_t parts, each, first_block;
};
template <typename E, int P>
__global__ __launch_bounds__(kThreads) void k_ff_pack_tokens(PackTokens t) {
    uint32_t block = t.first_block + blockIdx.x;
    const uint32_t which = block / t.each;
    block -= which * t.each;
    const PackRows a = t.of[which];
    const int32_t cols2 = padded(a.cols), rows2 = padded(a.rows);
    const int64_t node = block / a.per_node;
    const float* from = t.part + (node * 3 + which) * t.parts;
    float w = 0.f;
    for (uint32_t p = threadIdx.x; p < t.parts; p += kThreads) w = max_nan(w, from[p]);
    const Scale node_scale = scale_for(block_max(w));
    for (int k = 0; k < kRowsEach; ++k) {
        const int32_t row = ((int32_t)(block % a.per_node) * kRowsEach + k) * kPackRows + threadIdx.x / kWave;
        const int64_t at = node * rows2 + row;
        const float inv = row < a.rows ? t.row_inv[which][at] : 0.f;
        const Scale s = {inv * node_scale.up, 0.f};
        const typename E::mem* src = static_cast<const typename E::mem*>(a.src) + node * a.node + (int64_t)row * a.ld;
        pack_row<E, P>(src, row < a.rows ? a.cols : 0, cols2, false, s, a.dst + at * cols2, a.plane);
        if (row == 0 && (threadIdx.x & (kWave - 1)) == 0) a.inv[node] = node_scale.down;
    }
}

// ---- products ---------------------------------------------------------------------------------------------------------------
struct FfProduct {
    Operand A, B;
    TileGrid grid;
    uint32_t first_block;
    int32_t M, N, K;          // real rows and columns, padded terms
    const float* row_inv;     // scales of A's rows, n x rows of A's memory (or of k_ff_pack_tokens, one a node)
    const float* col_inv;     // of B's rows
    const float* gu_up;
    int32_t F, nodes;
    // activations in or out
    void* out;
    int64_t out_ld, out_node;
    void* hidden;
    int64_t hidden_node;
    int stream;               // hidden passes by the L2 caches
    // planes out
    half_t *h, *da;
    int64_t h_plane, da_plane;
    const float *h_up, *da_up, *db_up;
    // dx: TokenScales
    const float* middle;
    const int32_t* exp;
    // gradients out
    float* g;
    int64_t g_ld, off0, off1;  // columns of the blocks of gate and up, or down's
    int64_t second;            // halves from the B that gate's takes to up's, or 0: a single matrix
    int accumulate;
};

// h = act(x Wg^T) (x Wu^T): a wavefront's blocks of 32 columns are gate and up of the same 32 f's in turn.
template <typename S, typename E, int Act, int PH>
__global__ __launch_bounds__(S::Threads, 2) void k_ff_up(FfProduct a) {
    __shared__ __align__(16) char lds[2 * S::Stage];
    static_assert(S::NI == 2, "gate and up");
    int32_t node, ti, tj;
    if (!a.grid.at(a.first_block + blockIdx.x, &node, &ti, &tj)) return;
    const int32_t F2 = padded(a.F), m0 = ti * S::BM, f0 = tj * (S::BN / 2);
    acc16 acc[S::NI][S::MI];
    product_tile<S>(a.A, a.B, node, m0, 0, a.K, lds, acc,
                    [&](int row) { return (row >> 5 & 1) * F2 + min(f0 + (row >> 6) * 32 + (row & 31), F2 - 1); });
    typedef typename E::mem M;
    const int32_t f1 = wave_col<S>(2 * f0) / 2;
    const int64_t T2 = a.A.rows;
    each_octet_pair<S>(acc, lds, m0, [&](int32_t row, int32_t col, float* va, float* vb) {
        const int32_t f = f1 + col;
        if (row >= a.M || f >= F2) return;
        const int64_t at = node * T2 + row;
        const float xi = a.row_inv[at], up = a.h_up[at];
        const float *wi = a.col_inv + (int64_t)node * 2 * F2 + f, *wu = a.gu_up + (int64_t)node * 2 * F2 + f;
        float h[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            va[k] *= xi * wi[k];
            vb[k] *= xi * wi[F2 + k];
            h[k] = act_value<Act>(va[k]) * up * wu[k] * (vb[k] * up * wu[F2 + k]);  // neither factor passes its bound on the way
        }
        store_planes<PH>(a.h + at * F2 + f, a.h_plane, h);
        if (a.hidden && f < a.F) {
            M* hid = static_cast<M*>(a.hidden) + (int64_t)node * a.hidden_node + (int64_t)row * 2 * a.F;
            piece_put<kOct, E>(hid, f, a.F, va, a.stream);
            piece_put<kOct, E>(hid + a.F, f, a.F, vb, a.stream);
        }
    });
}

// Activations out.  Forward: a scale of the column and twice the row's, and the 2^15 that h is held in; backward (B by columns): da Wg and db Wu, each
// half of the terms, with the row's power of two (TokenScales).
template <typename S, typename E>
__device__ __forceinline__ void rows_product(const FfProduct& a, uint32_t block, char* lds) {
    int32_t node, ti, tj;
    if (!a.grid.at(block, &node, &ti, &tj)) return;
    const int32_t m0 = ti * S::BM, n0 = tj * S::BN;
    acc16 acc[S::NI][S::MI];
    const int64_t rows = (int64_t)node * a.A.rows;
    if constexpr (S::ColsB)
        product_tile<S>(a.A, a.B, node, m0, n0, a.K, lds, acc, [](int row) { return row; },
                        [&](int32_t row) { return a.middle[rows + min(row, a.A.rows - 1)]; });
    else
        product_tile<S>(a.A, a.B, node, m0, n0, a.K, lds, acc, [&](int row) { return min(n0 + row, a.B.rows - 1); });
    typedef typename E::mem M;
    each_octet<S>(acc, lds, m0, n0, false, [&](int32_t row, int32_t col, float* v) {
        if (row >= a.M || col >= a.N) return;
        if constexpr (S::ColsB) {
            const int e = a.exp[rows + row];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = ldexpf(v[k], e);
        } else {
            const float r = a.row_inv[rows + row];
            const float* c = a.col_inv + (int64_t)node * a.B.rows;
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = v[k] * (c[col + k] * 0x1p-15f) * r * r;
        }
        piece_put<kOct, E>(static_cast<M*>(a.out) + node * a.out_node + (int64_t)row * a.out_ld, col, a.N, v);
    });
}

template <typename S, typename E>
__global__ __launch_bounds__(S::Threads, 2) void k_ff_rows(FfProduct a) {
    __shared__ __align__(16) char lds[2 * S::Stage];
    rows_product<S, E>(a, a.first_block + blockIdx.x, lds);
}

// dh = dy Wd, and from it and the kept [a | b] the rows of [da | db] and h as halves.  Rows behind the last token are zeros: the
// products over tokens take them along.
template <typename S, typename E, int Act, int PA, int PH>
__global__ __launch_bounds__(S::Threads, 2) void k_ff_down_grad(FfProduct a) {
    __shared__ __align__(16) char lds[2 * S::Stage];
    int32_t node, ti, tj;
    if (!a.grid.at(a.first_block + blockIdx.x, &node, &ti, &tj)) return;
    const int32_t F2 = padded(a.F), T2 = a.A.rows, m0 = ti * S::BM, n0 = tj * S::BN;
    acc16 acc[S::NI][S::MI];
    product_tile<S>(a.A, a.B, node, m0, n0, a.K, lds, acc, [&](int row) { return row; });
    typedef typename E::mem M;
    each_octet<S>(acc, lds, m0, n0, false, [&](int32_t row, int32_t f, float* da) {
        if (row >= T2 || f >= F2) return;
        const int64_t at = (int64_t)node * T2 + row;
        float db[8] = {0.f}, h[8] = {0.f};
        if (row < a.M && f < a.F) {
            const M* hid = static_cast<const M*>(a.hidden) + (int64_t)node * a.hidden_node + (int64_t)row * 2 * a.F;
            float va[8], vb[8];
            piece_read<kOct, E>(hid, f, a.F, va);
            piece_read<kOct, E>(hid + a.F, f, a.F, vb);
            const float inv = a.row_inv[at], da_up = inv * a.da_up[at], db_up = inv * a.db_up[at], h_up = a.h_up[at];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                float value, slope;
                act_both<Act>(va[k], &value, &slope);
                db[k] = da[k] * db_up * value;
                da[k] = da[k] * da_up * vb[k] * slope;
                h[k] = value * vb[k] * h_up;
            }
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) da[k] = 0.f;
        }
        store_planes<PA>(a.da + at * 2 * F2 + f, a.da_plane, da);
        store_planes<PA>(a.da + at * 2 * F2 + F2 + f, a.da_plane, db);
        store_planes<PH>(a.h + at * F2 + f, a.h_plane, h);
    });
}

// Gradients of matrices: of gate and of up, two to a node, which are the first and the second half of A's columns; or of the down matrix's.
// G: fp32, narrow where a row of the matrix is.
template <typename S, typename G>
__device__ __forceinline__ void matrix_grad(const FfProduct& a, uint32_t block, char* lds) {
    int32_t node, ti, tj;
    if (!a.grid.at(block, &node, &ti, &tj)) return;
    const int32_t up = a.second ? node & 1 : 0, base = up * (a.A.ld / 2);
    if (a.second) node >>= 1;
    Operand B = a.B;
    B.p += up * a.second;
    const int32_t m0 = base + ti * S::BM, n0 = tj * S::BN;
    acc16 acc[S::NI][S::MI];
    product_tile<S>(a.A, B, node, m0, n0, a.K, lds, acc, [&](int row) { return row; });
    const float inv = a.row_inv[up * a.nodes + node];
    const int64_t off = up ? a.off1 : a.off0;
    each_octet<S>(acc, lds, m0, n0, false, [&](int32_t row, int32_t col, float* v) {
        row -= base;
        if (row >= a.M || col >= a.N) return;
        float* to = a.g + (int64_t)node * a.g_ld + off + (int64_t)row * a.N;
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= inv;
        if (a.accumulate) {
            float had[8];
            piece_read<kOct, G>(to, col, a.N, had);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] += had[k];
        }
        piece_put<kOct, G>(to, col, a.N, v);
    });
}

// dx, the gradients of gate and up and that of down wait for the same things only, and are one launch: 7 x 333 tokens, 511 x 1021, fp32, took 37
// and twice 28 us by themselves.
template <bool WithX, typename SX, typename SG, typename SD, typename E>
__global__ __launch_bounds__(SG::Threads, 2) void k_ff_grads(FfProduct x, FfProduct g, FfProduct d) {
    constexpr int kG = SG::Stage > SD::Stage ? SG::Stage : SD::Stage, kLds = WithX && SX::Stage > kG ? SX::Stage : kG;
    static_assert(SX::Threads == SG::Threads && SX::Threads == SD::Threads, "one shape of workgroup");
    __shared__ __align__(16) char lds[2 * kLds];
    typedef Elem<float, E::kNarrow> G;
    uint32_t block = g.first_block + blockIdx.x;
    if constexpr (WithX) {
        if (block < x.grid.blocks()) {
            rows_product<SX, E>(x, block, lds);
            return;
        }
        block -= x.grid.blocks();
    }
    if (block < g.grid.blocks()) matrix_grad<SG, G>(g, block, lds);
    else matrix_grad<SD, G>(d, block - g.grid.blocks(), lds);
}

__global__ __launch_bounds__(kThreads) void k_ff_zero(float* g, int64_t g_ld, int64_t off0, int64_t off1, int64_t off2, int64_t count, uint32_t per_node,
                                                      uint32_t first) {
    const uint32_t block = first + blockIdx.x, node = block / per_node;
    const int64_t e = (int64_t)(block % per_node) * kThreads + threadIdx.x;
    if (e >= count) return;
    float* row = g + (int64_t)node * g_ld;
    row[off0 + e] = row[off1 + e] = row[off2 + e] = 0.f;
}

// ---- few tokens ---------------------------------------------------------------------------------------------------------------
// Up to kFewTokens tokens a node: every matrix is read once, as it lies in X, and that is what takes the time (4 nodes, 1024 x 4096, fp16,
// 1, 16, 32 and 64 tokens: 42, 47, 63 and 87 us, the tiles' way 180 to 187; 20 nodes, 128 x 512: 10, 10, 13 and 18, the tiles' way 30 to
// 35).  A wavefront takes 16 rows of a matrix (16 of gate and the same 16 of up), 64 columns at a time, as bf16 pieces made in registers,
// which need no scale: three of them hold fp32; two (2^-17) go with bf16 activations, and hold h where y is rounded to 16 bits.  The wavefronts of a workgroup share a row's columns and
// add their sums in LDS.
// A lane holds 16 neighbouring columns of a row, 64 bytes, four lanes a row; which of a matrix instruction's k's they are does not
// matter as long as both operands agree.
constexpr int32_t kFewTokens = 64;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// Columns c .. c+15 of a row of `cols`; zeros behind the end.
template <typename M>
struct Sixteen {
    typedef M vec __attribute__((ext_vector_type(8), aligned(alignof(M))));
    M v[16];
    __device__ __forceinline__ void load(const M* row, int32_t c, int32_t cols) {
        if (c + 16 <= cols) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const vec p = *(reinterpret_cast<const vec*>(row + c) + k);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[8 * k + j] = p[j];
            }
        } else {
#pragma unroll
            for (int k = 0; k < 16; ++k) v[k] = c + k < cols ? row[c + k] : (M)0.f;
        }
    }
    // as P pieces, eight a matrix instruction
    template <int P>
    __device__ __forceinline__ void pieces(bf16x8 (&out)[P][2]) const {
        typedef __bf16 two __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int k = 0; k < 16; k += 2) {
            v2f r = {(float)v[k], (float)v[k + 1]};
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const two b = __builtin_convertvector(r, two);
                out[p][k / 8][k % 8] = b[0];
                out[p][k / 8][k % 8 + 1] = b[1];
                if (p + 1 < P) {
                    const uint32_t w = __builtin_bit_cast(uint32_t, b);
                    r[0] -= __uint_as_float(w << 16);
                    r[1] -= __uint_as_float(w & 0xffff0000u);
                }
            }
        }
    }
};

struct FewArgs {
    const void* x;             // activations, or h
    int64_t x_ld, x_node;
    const float* w[2];         // gate and up, or down
    int64_t ldx;
    int32_t T, K, rows;        // columns and rows of a matrix
    uint32_t per_node, first_block;
    void* hidden;              // up: n * T rows of 2 F, or NULL
    float* h;                  // up: n * T rows of F in fp32
    void* y;                   // down
    int64_t ld;
};

// EX: type of the operand that is read, E: of the result; Mats = 2: gate and up, 1: down.  NB: blocks of 16 tokens.
template <typename EX, typename E, int Mats, int Act, int PW, int PX, int NB, int Waves>
__global__ __launch_bounds__(Waves * kWave, (NB == 1 ? 4 : NB == 2 ? 3 : 2) - (PX == 3 && NB < 4 ? 1 : 0)) void k_ff_few(FewArgs a) {
    const uint32_t block = a.first_block + blockIdx.x;
    const int64_t node = block / a.per_node;
    const int32_t row0 = (int32_t)(block % a.per_node) * 16, lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int32_t row = min(row0 + (lane & 15), a.rows - 1), inner = (lane >> 4) * 16;
    const float* w[Mats];
#pragma unroll
    for (int m = 0; m < Mats; ++m) w[m] = a.w[m] + node * a.ldx + (int64_t)row * a.K;
    const typename EX::mem* x[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) x[b] = static_cast<const typename EX::mem*>(a.x) + node * a.x_node + (int64_t)min(b * 16 + (lane & 15), a.T - 1) * a.x_ld;
    v4f acc[Mats][NB];
#pragma unroll
    for (int m = 0; m < Mats; ++m)
#pragma unroll
        for (int b = 0; b < NB; ++b) acc[m][b] = v4f{0.f, 0.f, 0.f, 0.f};
    // the next chunk of the matrices and, as far as registers go, of the tokens is under way while one is multiplied
    constexpr bool kAhead = NB <= 2;
    struct Chunk {
        Sixteen<float> w[Mats];
        Sixteen<typename EX::mem> x[kAhead ? NB : 1];
    } now, next;
    // Each workgroup begins at another chunk: rows that lie a power of two apart would all be read from the same few channels of memory
    // at a time (24 tokens on 4 nodes, 1024 x 4096: 63.2 and 59.5 us)
    const int32_t chunks = (a.K + 63) / 64, begin = (int32_t)(block * Waves % (uint32_t)chunks);
    auto column = [&](int32_t k) { return (k + begin < chunks ? k + begin : k + begin - chunks) * 64 + inner; };
    auto load = [&](Chunk& to, int32_t k) {
        const int32_t c = column(k);
#pragma unroll
        for (int m = 0; m < Mats; ++m) to.w[m].load(w[m], c, a.K);
        if constexpr (kAhead) {
#pragma unroll
            for (int b = 0; b < NB; ++b) to.x[b].load(x[b], c, a.K);
        }
    };
    int32_t k = wave;
    if (k < chunks) load(now, k);
    for (; k < chunks; k += Waves) {
        if (k + Waves < chunks) load(next, k + Waves);
        bf16x8 px[NB][PX][2];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            if constexpr (!kAhead) now.x[0].load(x[b], column(k), a.K);
            now.x[kAhead ? b : 0].template pieces<PX>(px[b]);
        }
#pragma unroll
        for (int m = 0; m < Mats; ++m) {
            bf16x8 pw[PW][2];
            now.w[m].template pieces<PW>(pw);
#pragma unroll
            for (int i = 0; i < PW; ++i)
#pragma unroll
                for (int j = 0; j < PX && i + j < PW; ++j)
#pragma unroll
                    for (int half = 0; half < 2; ++half)
#pragma unroll
                        for (int b = 0; b < NB; ++b)
                            acc[m][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pw[i][half], px[b][j][half], acc[m][b], 0, 0, 0);
        }
        now = next;
    }
    __shared__ v4f s[Waves][Mats][NB][kWave];
#pragma unroll
    for (int m = 0; m < Mats; ++m)
#pragma unroll
        for (int b = 0; b < NB; ++b) s[wave][m][b][lane] = acc[m][b];
    __syncthreads();
    // lane l: token l % 16, rows 4 (l / 16) .. + 3
    for (int b = wave; b < NB; b += Waves) {
        v4f sum[Mats];
#pragma unroll
        for (int m = 0; m < Mats; ++m) {
            sum[m] = s[0][m][b][lane];
#pragma unroll
            for (int v = 1; v < Waves; ++v) sum[m] += s[v][m][b][lane];
        }
        const int32_t t = b * 16 + (lane & 15), r = row0 + (lane >> 4) * 4;
        if (t >= a.T) continue;
        const int64_t token = node * a.T + t;
        typedef typename E::mem M;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (r + j >= a.rows) continue;
            if constexpr (Mats == 2) {
                a.h[token * a.rows + r + j] = act_value<Act>(sum[0][j]) * sum[1][j];
                if (a.hidden) {
                    M* hid = static_cast<M*>(a.hidden) + token * 2 * a.rows + r + j;
                    hid[0] = E::put(sum[0][j]);
                    hid[a.rows] = E::put(sum[1][j]);
                }
            } else {
                static_cast<M*>(a.y)[token * a.ld + r + j] = E::put(sum[0][j]);
            }
        }
    }
}

// ---- launches ----------------------------------------------------------------------------------------------------------------
// Scratch of a call: blocks of a multiple of 256 bytes, handed out in order; without memory it counts.
struct Carve {
    char* base;
    size_t used = 0;
    template <typename P>
    P* take(int64_t count) {
        P* p = base ? reinterpret_cast<P*>(base + used) : nullptr;
        used += ((size_t)count * sizeof(P) + 255) / 256 * 256;
        return p;
    }
};

// Tokens of a node that go through together: scratch stays below some 4 GiB (and the least of a tile, whatever the width), and every
// workgroup of k_ff_pack_tokens reads a number of every four of them.
int32_t chunk_tokens(const FfShape& s, int64_t halves) {
    constexpr int64_t kMost = 1 << 16;
    const int64_t bytes = 2 * halves * s.n;
    const int64_t most = ((int64_t)4 << 30) / bytes / 256 * 256;
    const int64_t want = most < 256 ? 256 : most < kMost ? most : kMost;
    return s.T < want ? s.T : (int32_t)want;
}

struct FfScratch {
    int32_t chunk;
    int px, pgu, pd, ph, pa;  // planes
    half_t *gu, *wd, *x, *h, *dy, *da, *tokens[3];
    float *gu_inv, *wd_inv, *gu_up, *fold, *node_max, *x_inv, *h_up, *h_inv, *node_inv;
    TokenScales t;
};

FfScratch carve_ff(const FfShape& s, bool grad, char* base, size_t* bytes) {
    FfScratch w = {};
    const bool f32 = s.dtype == GPGA_F32;
    const int32_t D2 = padded(s.D), F2 = padded(s.F);
    Carve c = {base};
    w.px = f32 ? 2 : 1;
    if (!grad) {
        w.pgu = w.pd = s.dtype == GPGA_BF16 ? 1 : 2;
        w.ph = f32 ? 2 : 1;
        w.chunk = chunk_tokens(s, (int64_t)w.px * D2 + (int64_t)w.ph * F2);
    } else {
        w.pgu = f32 ? 2 : 1;
        w.pd = w.ph = w.pa = 2;
        w.chunk = chunk_tokens(s, (int64_t)4 * w.px * D2 + (int64_t)6 * F2);
    }
    const int64_t n = s.n, T2 = padded(w.chunk);
    w.gu = c.take<half_t>(n * 2 * F2 * D2 * w.pgu);
    w.wd = c.take<half_t>(n * F2 * D2 * w.pd);
    w.gu_inv = c.take<float>(n * 2 * F2);
    w.wd_inv = c.take<float>(n * D2);
    w.h = c.take<half_t>(n * T2 * F2 * w.ph);
    w.x_inv = c.take<float>(n * T2);
    w.h_up = c.take<float>(n * T2);
    w.h_inv = c.take<float>(n * T2);
    if (!grad) {
        w.gu_up = c.take<float>(n * 2 * F2);
        w.fold = c.take<float>(n * F2);
        w.x = c.take<half_t>(n * T2 * D2 * w.px);
    } else {
        w.node_max = c.take<float>(n * 2 * kMaxParts);
        w.dy = c.take<half_t>(n * T2 * D2 * w.px);
        for (half_t*& p : w.tokens) p = c.take<half_t>(n * T2 * D2 * w.px);
        w.da = c.take<half_t>(n * T2 * 2 * F2 * w.pa);
        w.t.da_up = c.take<float>(n * T2);
        w.t.da_inv = c.take<float>(n * T2);
        w.t.db_up = c.take<float>(n * T2);
        w.t.db_inv = c.take<float>(n * T2);
        w.t.h_up = w.h_up;
        w.t.h_inv = w.h_inv;
        w.t.dx_middle = c.take<float>(n * T2);
        w.t.dx_exp = c.take<int32_t>(n * T2);
        w.t.part = c.take<float>(n * 3 * (T2 / kPackRows));
        w.node_inv = c.take<float>(3 * n);
    }
    *bytes = c.used;
    return w;
}

Operand rows_operand(const half_t* p, int64_t n, int32_t rows, int32_t cols) { return {p, n * rows * cols, (int64_t)rows * cols, cols, rows}; }

// f(tile, grid) on the tiles that suit rows x cols with K terms.
template <int PA, int PB, bool CA, bool CB, typename F>
hipError_t launch_product(const gpga_ctx* c, FfProduct& a, int32_t rows, int32_t cols, F&& f) {
    const int side = tile_side(c->num_cus, PA + PB, rows, cols, a.K, c->n, false);
    a.grid.set(rows, cols, side, c->n, false);
    auto launch = [&](auto tile) {
        typedef decltype(tile) S;
        return launch_blocks(a.grid.blocks(), S::Threads, [&](uint32_t first, dim3 grid) {
            a.first_block = first;
            f(tile, grid);
        });
    };
    if (side == 256) return launch(Tile256<PA, PB, CA, CB>());
    if (side == 128) return launch(Tile128<PA, PB, CA, CB>());
    return launch(Tile64<PA, PB, CA, CB>());
}

// f(a constant) for the kind of activation.
template <int V>
struct Const {
    static constexpr int value = V;
};
template <typename F>
void with_act(int32_t act, F&& f) {
    if (act == GPGA_SILU) f(Const<GPGA_SILU>());
    else f(Const<GPGA_GELU>());
}

PackMatrices pack_matrices(const gpga_ctx* c, const FfShape& s, const FfScratch& w) {
    const int32_t D2 = padded(s.D), F2 = padded(s.F);
    PackMatrices a = {};
    a.gate = c->x + s.gate_off;
    a.up = c->x + s.up_off;
    a.down = c->x + s.down_off;
    a.ldx = c->ld;
    a.D = s.D;
    a.F = s.F;
    a.gu = w.gu;
    a.wd = w.wd;
    a.gu_plane = (int64_t)s.n * 2 * F2 * D2;
    a.wd_plane = (int64_t)s.n * F2 * D2;
    a.gu_inv = w.gu_inv;
    a.wd_inv = w.wd_inv;
    a.gu_up = w.gu_up;
    a.fold = w.fold;
    a.node_max = w.node_max;
    a.gu_blocks = (uint32_t)(2 * F2 / kPackRows);
    a.per_node = (uint32_t)(D2 / kPackRows);
    return a;
}

#define GPGA_LAUNCH(call)                        \
    do {                                         \
        const hipError_t e_ = (call);            \
        if (e_ != hipSuccess) return e_;         \
    } while (0)

// The three products of the backward pass on tiles of one side: what all tiles take on all compute units and, for the end, half of the
// longest one.
template <int PDX, int PGU, int PX, typename E>
hipError_t launch_grads(const gpga_ctx* c, FfProduct& x, FfProduct& g, FfProduct& d, int32_t T, int32_t D2, int32_t F2) {
    // one plane of each operand makes tiles whose steps are longer: with them two workgroups of 128 x 128 fit a compute unit in place of
    // three (8 x 4096 tokens, 768 x 2048, bf16: 1110 us together, 302 and 667 apart)
    constexpr bool kWithX = PDX + PGU > 2;
    if constexpr (!kWithX)
        GPGA_LAUNCH((launch_product<PDX, PGU, false, true>(c, x, T, D2, [&](auto tile, dim3 grid) {
            typedef decltype(tile) S;
            k_ff_rows<S, E><<<grid, dim3(S::Threads), 0, c->stream>>>(x);
        })));
    int side = 0;
    double best = 0.;
    for (int t = 0; t < 3; ++t) {
        const TileTime a(t, PDX + PGU, T, D2, x.K, c->n, false), b(t, 2 + PX, F2, D2, g.K, 2 * c->n, false), e(t, PX + 2, D2, F2, d.K, c->n, false);
        double us = ((kWithX ? a.tiles * a.us : 0.) + b.tiles * b.us + e.tiles * e.us) / c->num_cus + 0.5 * (kWithX ? fmax(a.us, b.us) : b.us);
        if (t == 0) us = fmax(us, fmax(kWithX ? TileTime::alone(PDX + PGU, x.K) : 0., TileTime::alone(2 + PX, g.K)));
        if (t == 0 || us < best) {
            best = us;
            side = 64 << t;
        }
    }
    if (kWithX) x.grid.set(T, D2, side, c->n, false);
    g.grid.set(F2, D2, side, 2 * c->n, false);
    d.grid.set(D2, F2, side, c->n, false);
    auto launch = [&](auto sx, auto sg, auto sd) {
        typedef decltype(sx) SX;
        const uint64_t blocks = (uint64_t)(kWithX ? x.grid.blocks() : 0) + g.grid.blocks() + d.grid.blocks();
        return launch_blocks(blocks, SX::Threads, [&](uint32_t first, dim3 grid) {
            g.first_block = first;
            k_ff_grads<kWithX, SX, decltype(sg), decltype(sd), E><<<grid, dim3(SX::Threads), 0, c->stream>>>(x, g, d);
        });
    };
    if (side == 256) return launch(Tile256<PDX, PGU, false, true>(), Tile256<2, PX, true, true>(), Tile256<PX, 2, true, true>());
    if (side == 128) return launch(Tile128<PDX, PGU, false, true>(), Tile128<2, PX, true, true>(), Tile128<PX, 2, true, true>());
    return launch(Tile64<PDX, PGU, false, true>(), Tile64<2, PX, true, true>(), Tile64<PX, 2, true, true>());
}

template <typename E, int NB>
hipError_t few(const gpga_ctx* c, const FfShape& s, const void* x, void* hidden, void* y, float* h) {
    typedef typename E::mem M;
    constexpr int PW = __is_same(M, __bf16) ? 2 : 3, PX = sizeof(M) == 4 ? 3 : __is_same(M, __bf16) ? 1 : 2, PH = sizeof(M) == 4 ? 3 : 2;
    FewArgs a = {};
    a.x = x;
    a.x_ld = s.ld;
    a.x_node = (int64_t)s.T * s.ld;
    a.w[0] = c->x + s.gate_off;
    a.w[1] = c->x + s.up_off;
    a.ldx = c->ld;
    a.T = s.T;
    a.K = s.D;
    a.rows = s.F;
    a.per_node = (uint32_t)((s.F + 15) / 16);
    a.hidden = hidden;
    a.h = h;
    GPGA_LAUNCH(launch_blocks((uint64_t)a.per_node * s.n, 4 * kWave, [&](uint32_t first, dim3 grid) {
        a.first_block = first;
        with_act(s.act, [&](auto act) {
            k_ff_few<E, E, 2, decltype(act)::value, PW, PX, NB, 4><<<grid, dim3(4 * kWave), 0, c->stream>>>(a);
        });
    }));
    a.x = h;
    a.x_ld = s.F;
    a.x_node = (int64_t)s.T * s.F;
    a.w[0] = c->x + s.down_off;
    a.K = s.F;
    a.rows = s.D;
    a.per_node = (uint32_t)((s.D + 15) / 16);
    a.y = y;
    a.ld = s.ld;
    return launch_blocks((uint64_t)a.per_node * s.n, 8 * kWave, [&](uint32_t first, dim3 grid) {
        a.first_block = first;
        k_ff_few<ElemF32, E, 1, GPGA_SILU, PW, PH, NB, 8><<<grid, dim3(8 * kWave), 0, c->stream>>>(a);
    });
}

template <typename E>
hipError_t forward(const gpga_ctx* c, const FfShape& s, const void* x, void* hidden, void* y, char* scratch) {
    typedef typename E::mem M;
    if (s.T <= kFewTokens) {
        typedef Elem<M, false> Wide;  // 16 columns at a time, or one by one
        float* h = reinterpret_cast<float*>(scratch);
        if (s.T <= 16) return few<Wide, 1>(c, s, x, hidden, y, h);
        if (s.T <= 32) return few<Wide, 2>(c, s, x, hidden, y, h);
        return few<Wide, 4>(c, s, x, hidden, y, h);
    }
    constexpr bool kF32 = sizeof(M) == 4, kBf16 = __is_same(M, __bf16);
    constexpr int PX = kF32 ? 2 : 1, PW = kBf16 ? 1 : 2, PH = PX;
    size_t bytes;
    const FfScratch w = carve_ff(s, false, scratch, &bytes);
    const int32_t D2 = padded(s.D), F2 = padded(s.F);
    PackMatrices m = pack_matrices(c, s, w);
    for (int32_t t0 = 0; t0 < s.T; t0 += w.chunk) {
        const int32_t T = s.T - t0 < w.chunk ? s.T - t0 : w.chunk, T2 = padded(T);
        PackRows p = {static_cast<const M*>(x) + (int64_t)t0 * s.ld, s.ld, (int64_t)s.T * s.ld, T, s.D, w.x, (int64_t)s.n * T2 * D2, w.x_inv,
                      (uint32_t)(T2 / (kPackRows * kRowsEach)), 0};
        const uint32_t matrix_blocks = t0 ? 0 : m.gu_blocks * (uint32_t)s.n;
        GPGA_LAUNCH(launch_blocks((uint64_t)p.per_node * s.n + matrix_blocks, kThreads, [&](uint32_t first, dim3 grid) {
            p.first_block = first;
            k_ff_pack_x<E, PX, PW><<<grid, dim3(kThreads), 0, c->stream>>>(m, matrix_blocks, p, w.h_up, w.h_inv);
        }));
        if (t0 == 0)
            GPGA_LAUNCH(launch_blocks((uint64_t)m.per_node * s.n, kThreads, [&](uint32_t first, dim3 grid) {
                m.first_block = first;
                k_ff_pack_down_folded<Elem<float, E::kNarrow>, PW><<<grid, dim3(kThreads), 0, c->stream>>>(m);
            }));
        FfProduct a = {};
        a.A = rows_operand(w.x, s.n, T2, D2);
        a.B = rows_operand(w.gu, s.n, 2 * F2, D2);
        a.M = T;
        a.K = D2;
        a.F = s.F;
        a.row_inv = w.x_inv;
        a.col_inv = w.gu_inv;
        a.gu_up = w.gu_up;
        a.hidden = hidden ? static_cast<M*>(hidden) + (int64_t)t0 * 2 * s.F : nullptr;
        a.hidden_node = (int64_t)s.T * 2 * s.F;
        // 8 x 4096 tokens, 768 x 2048, bf16: 530 us without, 494 with
        a.stream = s.F % 8 == 0 && stream_rows({s.n, s.T, 2 * s.F, 2 * s.F, s.dtype}, hidden);
        a.h = w.h;
        a.h_plane = (int64_t)s.n * T2 * F2;
        a.h_up = w.h_up;
        GPGA_LAUNCH((launch_product<PX, PW, false, false>(c, a, T, 2 * F2, [&](auto tile, dim3 grid) {
            with_act(s.act, [&](auto act) {
                typedef decltype(tile) S;
                k_ff_up<S, E, decltype(act)::value, PH><<<grid, dim3(S::Threads), 0, c->stream>>>(a);
            });
        })));
        FfProduct b = {};
        b.A = rows_operand(w.h, s.n, T2, F2);
        b.B = rows_operand(w.wd, s.n, D2, F2);
        b.M = T;
        b.N = s.D;
        b.K = F2;
        b.row_inv = w.h_inv;
        b.col_inv = w.wd_inv;
        b.out = static_cast<M*>(y) + (int64_t)t0 * s.ld;
        b.out_ld = s.ld;
        b.out_node = (int64_t)s.T * s.ld;
        GPGA_LAUNCH((launch_product<PH, PW, false, false>(c, b, T, D2, [&](auto tile, dim3 grid) {
            typedef decltype(tile) S;
            k_ff_rows<S, E><<<grid, dim3(S::Threads), 0, c->stream>>>(b);
        })));
    }
    return hipSuccess;
}

template <typename E>
hipError_t backward(const gpga_ctx* c, const FfShape& s, const void* dy, const void* x, const void* hidden, void* dx, bool accumulate, char* scratch) {
    typedef typename E::mem M;
    constexpr bool kF32 = sizeof(M) == 4, kBf16 = __is_same(M, __bf16);
    constexpr int PX = kF32 ? 2 : 1, PGU = kF32 ? 2 : 1, PDX = kBf16 ? 1 : 2;
    size_t bytes;
    const FfScratch w = carve_ff(s, true, scratch, &bytes);
    const int32_t D2 = padded(s.D), F2 = padded(s.F);
    const int64_t n = s.n;
    PackMatrices m = pack_matrices(c, s, w);
    m.per_node += kMaxParts;
    GPGA_LAUNCH(launch_blocks((uint64_t)m.per_node * s.n, kThreads, [&](uint32_t first, dim3 grid) {
        m.first_block = first;
        k_ff_pack_down<Elem<float, E::kNarrow>><<<grid, dim3(kThreads), 0, c->stream>>>(m, w.node_max);
    }));
    for (int32_t t0 = 0; t0 < s.T; t0 += w.chunk) {
        const int32_t T = s.T - t0 < w.chunk ? s.T - t0 : w.chunk, T2 = padded(T);
        const int64_t skip = (int64_t)t0 * s.ld;
        const M* hid = static_cast<const M*>(hidden) + (int64_t)t0 * 2 * s.F;
        const int64_t hidden_node = (int64_t)s.T * 2 * s.F;
        PackRows p = {static_cast<const M*>(dy) + skip, s.ld, (int64_t)s.T * s.ld, T, s.D, w.dy, n * T2 * D2, w.x_inv, (uint32_t)(T2 / kPackRows), 0};
        const uint32_t matrix_blocks = t0 ? 0 : m.gu_blocks * (uint32_t)s.n;
        GPGA_LAUNCH(launch_blocks((uint64_t)p.per_node * s.n + matrix_blocks, kThreads, [&](uint32_t first, dim3 grid) {
            p.first_block = first;
            k_ff_pack_dy<E, PX><<<grid, dim3(kThreads), 0, c->stream>>>(m, matrix_blocks, p, static_cast<const M*>(x) + skip, hid, hidden_node, w.t);
        }));
        p.per_node /= kRowsEach;
        PackTokens tokens = {{p, p, p}, {w.t.da_inv, w.t.db_inv, w.h_inv}, w.t.part, (uint32_t)(T2 / kPackRows), p.per_node * (uint32_t)s.n, 0};
        for (int k = 0; k < 3; ++k) {
            if (k < 2) tokens.of[k].src = static_cast<const M*>(x) + skip;
            tokens.of[k].dst = w.tokens[k];
            tokens.of[k].inv = w.node_inv + k * n;
        }
        GPGA_LAUNCH(launch_blocks((uint64_t)3 * tokens.each, kThreads, [&](uint32_t first, dim3 grid) {
            tokens.first_block = first;
            k_ff_pack_tokens<E, PX><<<grid, dim3(kThreads), 0, c->stream>>>(tokens);
        }));
        FfProduct a = {};
        a.A = rows_operand(w.dy, n, T2, D2);
        a.B = rows_operand(w.wd, n, D2, F2);
        a.M = T;
        a.K = D2;
        a.F = s.F;
        a.row_inv = w.x_inv;
        a.hidden = const_cast<M*>(hid);
        a.hidden_node = hidden_node;
        a.h = w.h;
        a.h_plane = n * T2 * F2;
        a.h_up = w.h_up;
        a.da = w.da;
        a.da_plane = n * T2 * 2 * F2;
        a.da_up = w.t.da_up;
        a.db_up = w.t.db_up;
        GPGA_LAUNCH((launch_product<PX, 2, false, true>(c, a, T2, F2, [&](auto tile, dim3 grid) {
            with_act(s.act, [&](auto act) {
                typedef decltype(tile) S;
                k_ff_down_grad<S, E, decltype(act)::value, 2, 2><<<grid, dim3(S::Threads), 0, c->stream>>>(a);
            });
        })));
        FfProduct b = {};
        b.A = rows_operand(w.da, n, T2, 2 * F2);
        b.B = rows_operand(w.gu, n, 2 * F2, D2);
        b.M = T;
        b.N = s.D;
        b.K = 2 * F2;
        b.middle = w.t.dx_middle;
        b.exp = w.t.dx_exp;
        b.out = static_cast<M*>(dx) + skip;
        b.out_ld = s.ld;
        b.out_node = (int64_t)s.T * s.ld;
        FfProduct g = {};
        g.A = rows_operand(w.da, n, T2, 2 * F2);
        g.B = rows_operand(w.tokens[0], n, T2, D2);
        g.second = w.tokens[1] - w.tokens[0];
        g.nodes = s.n;
        g.M = s.F;
        g.N = s.D;
        g.K = T2;
        g.row_inv = w.node_inv;
        g.g = c->g;
        g.g_ld = c->ld;
        g.off0 = s.gate_off;
        g.off1 = s.up_off;
        g.accumulate = accumulate || t0 > 0;
        FfProduct d = g;
        d.A = rows_operand(w.tokens[2], n, T2, D2);
        d.second = 0;
        d.B = rows_operand(w.h, n, T2, F2);
        d.M = s.D;
        d.N = s.F;
        d.row_inv = w.node_inv + 2 * n;
        d.off0 = s.down_off;
        GPGA_LAUNCH((launch_grads<PDX, PGU, PX, E>(c, b, g, d, T, D2, F2)));
    }
    return hipSuccess;
}

}  // namespace

size_t gated_ff_scratch(const FfShape& s, bool grad) {
    if (s.T == 0) return 0;
    if (!grad && s.T <= kFewTokens) return (size_t)s.n * s.T * s.F * sizeof(float);
    size_t bytes;
    carve_ff(s, grad, nullptr, &bytes);
    return bytes;
}

hipError_t launch_gated_ff(const gpga_ctx* c, const FfShape& s, const void* x, void* hidden, void* y, void* scratch) {
    auto launch = [&](auto e) { return forward<decltype(e)>(c, s, x, hidden, y, static_cast<char*>(scratch)); };
    return s.D < kOct || s.F < kOct ? with_narrow_elem(s.dtype, launch) : with_elem(s.dtype, launch);
}

hipError_t launch_gated_ff_grad(const gpga_ctx* c, const FfShape& s, const void* dy, const void* x, const void* hidden, void* dx, bool accumulate,
                                void* scratch) {
    if (s.T == 0) {
        if (accumulate) return hipSuccess;
        const int64_t count = (int64_t)s.F * s.D;
        const uint32_t per_node = (uint32_t)((count + kThreads - 1) / kThreads);
        return launch_blocks((uint64_t)per_node * s.n, kThreads, [&](uint32_t first, dim3 grid) {
            k_ff_zero<<<grid, dim3(kThreads), 0, c->stream>>>(c->g, c->ld, s.gate_off, s.up_off, s.down_off, count, per_node, first);
        });
    }
    auto launch = [&](auto e) { return backward<decltype(e)>(c, s, dy, x, hidden, dx, accumulate, static_cast<char*>(scratch)); };
    return s.D < kOct || s.F < kOct ? with_narrow_elem(s.dtype, launch) : with_elem(s.dtype, launch);
}
