// Cross-entropy of softmax(z) over a vocabulary, averaged over a node's counted tokens (label >= 0), and its gradient.
//
//   loss_i = (1/N_i) * sum over counted t of log sum_v exp(z_v - m) + (m - z_label),  m = max_v z_v
//   dz_v   = (a/N_i) * (exp(z_v - m) / sum - [v = label])                              rows that are not counted: 0
//
// The loss is a sum of two terms that are both at least 0: m is never added to the logarithm, so large logits cost no
// digits.  A label of V or more is never an address: the loss of its node and its row of dz are NaN.  A node without a
// counted token has loss 0 (NaN would spread to every node with the next gossip step).
//
// Three forms.  Rows of up to 32768 columns are read once: L lanes hold a row as exp(z - m_lane) in fp32, m_lane the largest value
// of the lane, and one pass over the lanes joins maxima and sums; the gradient is what is held times exp(m_lane - m) a / (N sum).
// Longer ones are swept twice by a workgroup, the second time out of the cache.  Where there are fewer rows than compute units,
// long ones are cut into pieces for a workgroup each, and a second launch reads them again for the gradient.
//
// Bound by the logits' bytes: 8 x 512 rows of 32000 bf16 with the gradient in 90 us (5.5 TB/s; three readings of a row took 164).  A
// compute unit holds two such rows, so loads, sums and stores of two rows overlap and no more; holding rows as they lie in
// memory and taking exp twice was slower at every number of lanes (130 to 180 us, registers).  One row of 128000 fp32 a node: 5 us.
#include "gpga_rows.hpp"

namespace {

constexpr int kThreads = 256;
constexpr int kNodeThreads = 1024;  // of the launches that take a node a workgroup
constexpr float kLowest = -3.402823466e38f;  // stands for -inf as a maximum: -inf - kLowest is -inf and not NaN

uint32_t blocks_for(int64_t items, int64_t per_block) { return (uint32_t)((items + per_block - 1) / per_block); }

template <typename E>
struct LossArgs {
    typedef typename E::mem mem;
    int32_t T, V;
    int64_t ld;
    uint32_t per_node;     // workgroups of a node
    uint32_t first_block;  // of the launch
    const mem* z;
    const int32_t* labels;
    mem* dz;               // may be NULL
    float* row_loss;       // n*T
    const int32_t* count;  // n: counted tokens; NULL: a workgroup counts the labels of its node itself
    float grad_scale;
    bool stream;           // rows pass by the caches
    uint32_t* left;        // counters, one a node, kLossLeftStride apart; NULL: k_loss_mean follows
    float* loss;           // n
    // rows in pieces
    uint32_t pieces;       // of a row
    int32_t piece;         // columns of one, a multiple of kOct * kThreads
    float* parts;          // n*T x pieces pairs (maximum, sum)
};

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1) v += __shfl_xor(v, off, kWave);
    return v;
}

// Counted tokens among labels[0 .. T), by a workgroup of `threads`; `lds` one word a wavefront.  Holds a barrier.
__device__ __forceinline__ int32_t count_labels(const int32_t* __restrict__ labels, int32_t T, int32_t threads, int32_t* lds) {
    int32_t mine = 0;
#pragma unroll 4
    for (int32_t t = threadIdx.x; t < T; t += threads) mine += labels[t] >= 0 ? 1 : 0;
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1) mine += __shfl_xor(mine, off, kWave);
    if ((threadIdx.x & (kWave - 1)) == 0) lds[threadIdx.x / kWave] = mine;
    __syncthreads();
    mine = 0;
    for (int32_t w = 0; w < threads / kWave; ++w) mine += lds[w];
    return mine;
}

// loss = sum over the node's rows / counted tokens, by a workgroup of `threads`; double, a fixed order.  row(t) is the loss of row t.
template <typename F>
__device__ __forceinline__ void node_loss(int32_t T, int32_t threads, int32_t counted, double* lds, float* loss, F&& row) {
    double mine = 0.0;
    for (int64_t t = threadIdx.x; t < T; t += 4 * threads) {  // four loads under way
        float v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = t + k * threads < T ? row((int32_t)(t + k * threads)) : 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) mine += (double)v[k];
    }
    mine = wave_sum64(mine);
    if ((threadIdx.x & (kWave - 1)) == 0) lds[threadIdx.x / kWave] = mine;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int32_t w = 1; w < threads / kWave; ++w) mine += lds[w];
        *loss = counted > 0 ? (float)(mine / counted) : 0.f;
    }
}

// Whether this workgroup is the last of its node, once what thread 0 stored for the others has arrived; said in *last, for after a
// barrier.  The counter is 0 again for the next launch.
__device__ __forceinline__ void note_end(uint32_t* left, uint32_t workgroups, int32_t* last) {
    asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
    const bool is = __hip_atomic_fetch_add(left, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == workgroups - 1;
    if (is) __hip_atomic_store(left, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *last = is;
}

__global__ __launch_bounds__(kNodeThreads) void k_count(const int32_t* __restrict__ labels, int32_t T, int32_t* __restrict__ count,
                                                    uint32_t first_block) {
    __shared__ int32_t s_count[kNodeThreads / kWave];
    const uint32_t node = first_block + blockIdx.x;
    const int32_t n = count_labels(labels + (int64_t)node * T, T, kNodeThreads, s_count);
    if (threadIdx.x == 0) count[node] = n;
}

// Where the losses of a node are not added up by the last workgroup of the launch that makes them.
__global__ __launch_bounds__(kNodeThreads) void k_loss_mean(const float* __restrict__ row_loss, const int32_t* __restrict__ labels, int32_t T,
                                                        float* __restrict__ loss, uint32_t first_block) {
    __shared__ int32_t s_count[kNodeThreads / kWave];
    __shared__ double s_sum[kNodeThreads / kWave];
    const uint32_t node = first_block + blockIdx.x;
    const float* rows = row_loss + (int64_t)node * T;
    const int32_t counted = count_labels(labels + (int64_t)node * T, T, kNodeThreads, s_count);
    node_loss(T, kNodeThreads, counted, s_sum, loss + node, [&](int32_t t) { return rows[t]; });
}

// Columns past the end of the row take no part.
__device__ __forceinline__ void past_end(float* v, int32_t c, int32_t V) {
#pragma unroll
    for (int j = 0; j < kOct; ++j) v[j] = c + j < V ? v[j] : -INFINITY;
}
// v[at] -= by
__device__ __forceinline__ void less_at(float* v, int32_t at, float by) {
#pragma unroll
    for (int j = 0; j < kOct; ++j) v[j] -= j == at ? by : 0.f;
}

// ---- rows held in registers: L lanes a row, N pieces of eight columns a lane ------------------------------------------------
template <typename E, int L, int N>
__global__ __launch_bounds__(L > kThreads ? L : kThreads) void k_loss_held(LossArgs<E> a) {
    constexpr int kBlock = L > kThreads ? L : kThreads, kRows = kBlock / L, kWaves = kBlock / kWave, kRowWaves = L / kWave, kLanes = L < kWave ? L : kWave;
    __shared__ float s_max[kWaves], s_sum[kWaves];
    __shared__ int32_t s_count[kWaves], s_last;
    __shared__ double s_total[kWaves];
    const uint32_t block = a.first_block + blockIdx.x, node = block / a.per_node;
    const int32_t t = (int32_t)((block - node * a.per_node) * kRows + threadIdx.x / L);
    const int64_t r = (int64_t)node * a.T + t;
    const int32_t lane = threadIdx.x & (L - 1);
    const int32_t* labels = a.labels + (int64_t)node * a.T;
    const int32_t label = t < a.T ? labels[t] : -1;
    const typename E::mem* z = a.z + r * a.ld;
    Piece<E, kOct> in[N];
    float picked = 0.f;
    const bool bad = label >= a.V;
    if (label >= 0) {
#pragma unroll
        for (int k = 0; k < N; ++k) in[k] = piece_load<kOct, E>(z, (lane + k * L) * kOct, a.V, a.stream);
        picked = E::get(z[bad ? 0 : label]);
    }
    const int32_t counted = a.count ? a.count[node] : count_labels(labels, a.T, kBlock, s_count);
    float e[N][kOct], mine = kLowest, sum = 0.f, top = 0.f, share = 1.f;
    if (label >= 0) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int32_t c = (lane + k * L) * kOct;
            piece_get<kOct, E>(in[k], c, a.V, e[k]);
            if (c + kOct > a.V) past_end(e[k], c, a.V);
#pragma unroll
            for (int j = 0; j < kOct; ++j) mine = fmaxf(mine, e[k][j]);
        }
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int j = 0; j < kOct; ++j) {
                e[k][j] = __expf(e[k][j] - mine);
                sum += e[k][j];
            }
        top = wave_max<kLanes>(mine);
        sum = wave_sum<kLanes>(sum * __expf(mine - top));
    }
    if constexpr (L > kWave) {
        if ((threadIdx.x & (kWave - 1)) == 0) {
            s_max[threadIdx.x / kWave] = top;
            s_sum[threadIdx.x / kWave] = sum;
        }
        __syncthreads();  // from here on dz may take the place of z
        top = s_max[0];
#pragma unroll
        for (int w = 1; w < kRowWaves; ++w) top = fmaxf(top, s_max[w]);
        sum = 0.f;
#pragma unroll
        for (int w = 0; w < kRowWaves; ++w) sum += s_sum[w] * __expf(s_max[w] - top);
    }
    if (lane == 0 && t < a.T) {
        const float loss = label < 0 ? 0.f : bad ? __builtin_nanf("") : logf(sum) + (top - picked);
        __hip_atomic_store(a.row_loss + r, loss, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (a.left) {
        if (kRows > 1) {
            asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
            __syncthreads();
        }
        if (threadIdx.x == 0) note_end(a.left + (int64_t)node * kLossLeftStride, a.per_node, &s_last);
    }
    if (a.dz && t < a.T) {
        typename E::mem* dz = a.dz + r * a.ld;
        if (label < 0) {
            const float zero[kOct] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const int32_t c = (lane + k * L) * kOct;
                if (c < a.V) piece_put<kOct, E>(dz, c, a.V, zero, a.stream);
            }
        } else {
            const float scale = bad ? __builtin_nanf("") : a.grad_scale / (float)counted;
            share = __expf(mine - top) * (scale / sum);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const int32_t c = (lane + k * L) * kOct;
                if (c < a.V) {
#pragma unroll
                    for (int j = 0; j < kOct; ++j) e[k][j] *= share;
                    if ((uint32_t)(label - c) < kOct) less_at(e[k], label - c, scale);
                    piece_put<kOct, E>(dz, c, a.V, e[k], a.stream);
                }
            }
        }
    }
    if (a.left) {
        __syncthreads();
        if (s_last)
            node_loss(a.T, kBlock, counted, s_total, a.loss + node, [&](int32_t k) {
                return __hip_atomic_load(a.row_loss + (int64_t)node * a.T + k, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            });
    }
}

// ---- rows that registers do not hold: columns from .. to of a row, by kLanes lanes ------------------------------------------
constexpr int kPiecesAhead = 4;  // of a lane, whose loads are under way together

// Running maximum and sum of exp(z - maximum) of a lane.
template <typename E, int kLanes>
__device__ __forceinline__ void sweep_sum(const typename E::mem* z, int32_t from, int32_t to, int32_t V, float* top_out, float* sum_out) {
    float top = kLowest, sum = 0.f;
    for (int32_t c0 = from + (int32_t)threadIdx.x * kOct; c0 < to; c0 += kPiecesAhead * kLanes * kOct) {
        Piece<E, kOct> in[kPiecesAhead];
#pragma unroll
        for (int k = 0; k < kPiecesAhead; ++k) in[k] = piece_load<kOct, E>(z, c0 + k * kLanes * kOct, V);
#pragma unroll
        for (int k = 0; k < kPiecesAhead; ++k) {
            const int32_t c = c0 + k * kLanes * kOct;
            if (c >= to) break;
            float v[kOct], most = top;
            piece_get<kOct, E>(in[k], c, V, v);
            if (c + kOct > V) past_end(v, c, V);
#pragma unroll
            for (int j = 0; j < kOct; ++j) most = fmaxf(most, v[j]);
            sum *= __expf(top - most);
            top = most;
#pragma unroll
            for (int j = 0; j < kOct; ++j) sum += __expf(v[j] - top);
        }
    }
    *top_out = top;
    *sum_out = sum;
}
// The gradient, exp(z - top) * share less scale at the label.
template <typename E, int kLanes>
__device__ __forceinline__ void sweep_grad(const typename E::mem* z, typename E::mem* dz, int32_t from, int32_t to, int32_t V, int32_t label, float top,
                                           float share, float scale, bool stream) {
    for (int32_t c0 = from + (int32_t)threadIdx.x * kOct; c0 < to; c0 += kPiecesAhead * kLanes * kOct) {
        Piece<E, kOct> in[kPiecesAhead];
#pragma unroll
        for (int k = 0; k < kPiecesAhead; ++k) in[k] = piece_load<kOct, E>(z, c0 + k * kLanes * kOct, V);
#pragma unroll
        for (int k = 0; k < kPiecesAhead; ++k) {
            const int32_t c = c0 + k * kLanes * kOct;
            if (c >= to) break;
            float v[kOct];
            piece_get<kOct, E>(in[k], c, V, v);
#pragma unroll
            for (int j = 0; j < kOct; ++j) v[j] = __expf(v[j] - top) * share;
            if ((uint32_t)(label - c) < kOct) less_at(v, label - c, scale);
            piece_put<kOct, E>(dz, c, V, v, stream);
        }
    }
}

// A workgroup a row, read twice for the gradient: the second time from the cache in front of memory, which holds the rows of the 512 workgroups that
// are under way (8 x 256 rows of 100000 bf16: 179 us; in two launches, between which it loses them, 247).
template <typename E, int kLanes>
__global__ __launch_bounds__(kLanes) void k_loss_swept(LossArgs<E> a) {
    constexpr int kWaves = kLanes / kWave;
    __shared__ float s_max[kWaves], s_sum[kWaves];
    __shared__ int32_t s_count[kWaves];
    const uint32_t block = a.first_block + blockIdx.x, node = block / a.per_node;
    const int64_t r = block;
    const int32_t* labels = a.labels + (int64_t)node * a.T;
    const int32_t label = a.labels[r];
    const typename E::mem* z = a.z + r * a.ld;
    typename E::mem* dz = a.dz ? a.dz + r * a.ld : nullptr;
    if (label < 0) {
        if (threadIdx.x == 0) a.row_loss[r] = 0.f;
        const float zero[kOct] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        for (int32_t c = threadIdx.x * kOct; dz && c < a.V; c += kLanes * kOct) piece_put<kOct, E>(dz, c, a.V, zero, a.stream);
        return;
    }
    const bool bad = label >= a.V;
    const float picked = E::get(z[bad ? 0 : label]);
    const int32_t counted = !dz ? 0 : a.count ? a.count[node] : count_labels(labels, a.T, kLanes, s_count);
    float top, sum;
    sweep_sum<E, kLanes>(z, 0, a.V, a.V, &top, &sum);
    const float most = wave_max<kWave>(top);
    sum = wave_sum<kWave>(sum * __expf(top - most));
    if ((threadIdx.x & (kWave - 1)) == 0) {
        s_max[threadIdx.x / kWave] = most;
        s_sum[threadIdx.x / kWave] = sum;
    }
    __syncthreads();  // from here on dz may take the place of z
    top = s_max[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) top = fmaxf(top, s_max[w]);
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sum += s_sum[w] * __expf(s_max[w] - top);
    if (threadIdx.x == 0) a.row_loss[r] = bad ? __builtin_nanf("") : logf(sum) + (top - picked);
    if (!dz) return;
    const float scale = bad ? __builtin_nanf("") : a.grad_scale / (float)counted;
    sweep_grad<E, kLanes>(z, dz, 0, a.V, a.V, label, top, scale / sum, scale, a.stream);
}

// ---- rows in pieces: a workgroup for each ------------------------------------------------------------------------------------
// Maximum and sum of exp(z - maximum) of a row from those of its pieces, by an aligned group of lanes (a power of two up to 64); all
// of them get both.
struct MaxSum {
    float top, sum;
};
__device__ __forceinline__ MaxSum join_parts(const float* parts, uint32_t pieces, uint32_t lanes) {
    auto part = [&](uint32_t k) { return __hip_atomic_load(parts + k, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
    MaxSum all = {kLowest, 0.f};
    for (uint32_t k = threadIdx.x & (lanes - 1); k < pieces; k += lanes) {
        const float top = part(2 * k), sum = part(2 * k + 1), most = fmaxf(all.top, top);
        all.sum = all.sum * __expf(all.top - most) + sum * __expf(top - most);
        all.top = most;
    }
    for (uint32_t off = lanes / 2; off > 0; off >>= 1) {
        const float top = __shfl_xor(all.top, off, kWave), sum = __shfl_xor(all.sum, off, kWave), most = fmaxf(all.top, top);
        all.sum = all.sum * __expf(all.top - most) + sum * __expf(top - most);
        all.top = most;
    }
    return all;
}
__device__ __forceinline__ uint32_t join_lanes(uint32_t pieces) {
    uint32_t lanes = 1;
    while (lanes < pieces && lanes < kWave) lanes *= 2;
    return lanes;
}

// Loss of a node whose rows are in pieces, by a workgroup: a group of lanes a row in turn.
template <typename E>
__device__ __forceinline__ void node_loss_parts(const LossArgs<E>& a, uint32_t node, int32_t* s_count, double* s_total) {
    const int64_t first = (int64_t)node * a.T;
    const int32_t counted = count_labels(a.labels + first, a.T, kThreads, s_count);
    const uint32_t lanes = join_lanes(a.pieces);
    double mine = 0.0;
    for (int64_t t = threadIdx.x / lanes; t < a.T; t += kThreads / lanes) {
        const int64_t r = first + t;
        const int32_t label = a.labels[r];
        const float picked = label >= 0 && label < a.V ? E::get(a.z[r * a.ld + label]) : __builtin_nanf("");
        if (label < 0) continue;
        const MaxSum all = join_parts(a.parts + r * 2 * a.pieces, a.pieces, lanes);
        if ((threadIdx.x & (lanes - 1)) == 0) mine += (double)(logf(all.sum) + (all.top - picked));
    }
    mine = wave_sum64(mine);
    if ((threadIdx.x & (kWave - 1)) == 0) s_total[threadIdx.x / kWave] = mine;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kThreads / kWave; ++w) mine += s_total[w];
        a.loss[node] = counted > 0 ? (float)(mine / counted) : 0.f;
    }
}

template <typename E>
__global__ __launch_bounds__(kThreads) void k_loss_parts(LossArgs<E> a) {
    constexpr int kWaves = kThreads / kWave;
    __shared__ float s_max[kWaves], s_sum[kWaves];
    __shared__ int32_t s_count[kWaves], s_last;
    __shared__ double s_total[kWaves];
    const int64_t r = blockIdx.x / a.pieces;
    const uint32_t node = (uint32_t)(r / a.T), piece = blockIdx.x - (uint32_t)r * a.pieces;
    if (a.labels[r] >= 0) {
        const int32_t from = (int32_t)piece * a.piece, to = a.V - from < a.piece ? a.V : from + a.piece;
        const typename E::mem* z = a.z + r * a.ld;
        float top, sum;
        sweep_sum<E, kThreads>(z, from, to, a.V, &top, &sum);
        float all = wave_max<kWave>(top);
        sum = wave_sum<kWave>(sum * __expf(top - all));
        if ((threadIdx.x & (kWave - 1)) == 0) {
            s_max[threadIdx.x / kWave] = all;
            s_sum[threadIdx.x / kWave] = sum;
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < kWaves; ++w) all = fmaxf(all, s_max[w]);
            sum = 0.f;
            for (int w = 0; w < kWaves; ++w) sum += s_sum[w] * __expf(s_max[w] - all);
            float* part = a.parts + (r * a.pieces + piece) * 2;
            __hip_atomic_store(part, all, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __hip_atomic_store(part + 1, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    }
    if (!a.left) return;  // k_loss_join follows
    if (threadIdx.x == 0) note_end(a.left + (int64_t)node * kLossLeftStride, a.per_node, &s_last);
    __syncthreads();
    if (!s_last) return;
    node_loss_parts<E>(a, node, s_count, s_total);
}

template <typename E>
__global__ __launch_bounds__(kThreads) void k_loss_join(LossArgs<E> a) {
    __shared__ int32_t s_count[kThreads / kWave];
    __shared__ double s_total[kThreads / kWave];
    node_loss_parts<E>(a, blockIdx.x, s_count, s_total);
}

template <typename E>
__global__ __launch_bounds__(kThreads) void k_loss_parts_grad(LossArgs<E> a) {
    __shared__ int32_t s_count[kThreads / kWave];
    const int64_t r = blockIdx.x / a.pieces;
    const uint32_t node = (uint32_t)(r / a.T), piece = blockIdx.x - (uint32_t)r * a.pieces;
    const int32_t label = a.labels[r];
    const int32_t from = (int32_t)piece * a.piece, to = a.V - from < a.piece ? a.V : from + a.piece;
    const typename E::mem* z = a.z + r * a.ld;
    typename E::mem* dz = a.dz + r * a.ld;
    if (label < 0) {
        const float zero[kOct] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        for (int32_t c = from + (int32_t)threadIdx.x * kOct; c < to; c += kThreads * kOct) piece_put<kOct, E>(dz, c, a.V, zero);
        return;
    }
    const int32_t counted = count_labels(a.labels + (int64_t)node * a.T, a.T, kThreads, s_count);
    const MaxSum all = join_parts(a.parts + r * 2 * a.pieces, a.pieces, kWave);
    const float scale = label >= a.V ? __builtin_nanf("") : a.grad_scale / (float)counted, share = scale / all.sum;
    sweep_grad<E, kThreads>(z, dz, from, to, a.V, label, all.top, share, scale, a.stream);
}

template <int V>
struct Const {
    static constexpr int value = V;
};
// Lanes a row and pieces a lane by the number of eights in it: the smallest that hold it.  Up to 16384 columns at most 512 lanes, so that
// a compute unit has room for several rows (8 x 512 rows of 12000 bf16: 41 us with 3 x 512, 51 with 2 x 1024); above, it has two
// whatever their length (8 x 512 rows of 20000 bf16 take 70 us, of 32000 91).
template <typename E, typename F>
bool with_row_shape(int32_t octs, F&& f) {
    if constexpr (E::kNarrow) f(Const<16>(), Const<1>());
    else if (octs <= 16) f(Const<16>(), Const<1>());
    else if (octs <= 32) f(Const<32>(), Const<1>());
    else if (octs <= 64) f(Const<64>(), Const<1>());
    else if (octs <= 128) f(Const<64>(), Const<2>());
    else if (octs <= 256) f(Const<64>(), Const<4>());
    else if (octs <= 512) f(Const<256>(), Const<2>());
    else if (octs <= 768) f(Const<256>(), Const<3>());
    else if (octs <= 1024) f(Const<256>(), Const<4>());
    else if (octs <= 1536) f(Const<512>(), Const<3>());
    else if (octs <= 2048) f(Const<512>(), Const<4>());
    else if (octs <= 3072) f(Const<1024>(), Const<3>());
    else if (octs <= 4096) f(Const<1024>(), Const<4>());
    else return false;
    return true;
}

constexpr int32_t kHeldAlone = 8192;  // longest rows that are held for the loss alone

// Long rows are cut into pieces where there are fewer of them than compute units.
constexpr int32_t kPieceUnit = kOct * kThreads;
struct Cut {
    uint32_t pieces = 0;  // 0: a row is one workgroup's or less
    int32_t piece = 0;
    Cut(const RowsShape& s, int num_cus) {
        const int64_t rows = (int64_t)s.n * s.T;
        if (s.D <= 8192 || rows == 0 || rows >= num_cus) return;
        const int64_t units = ((int64_t)s.D + kPieceUnit - 1) / kPieceUnit, wanted = 4 * num_cus / rows;
        const int64_t each = wanted < units ? units / wanted : 1;
        piece = (int32_t)(each * kPieceUnit < s.D ? each * kPieceUnit : s.D);
        pieces = (uint32_t)(((int64_t)s.D + piece - 1) / piece);
    }
};

}  // namespace

size_t token_loss_scratch(const RowsShape& s, int num_cus) {
    const Cut cut(s, num_cus);
    return ((size_t)s.n * (size_t)s.T * (cut.pieces ? 2 * cut.pieces : 1) + (size_t)s.n) * 4;
}

hipError_t launch_token_loss(const gpga_ctx* c, const RowsShape& s, const void* logits, const int32_t* labels, float grad_scale, float* loss,
                             void* dlogits, void* scratch) {
    const Cut cut(s, c->num_cus);
    int32_t* count = static_cast<int32_t*>(scratch);
    float* rows = reinterpret_cast<float*>(count + s.n);
    // the launch's last workgroup of a node adds up its losses, unless so many end there that they would queue for the counter
    // (1000 rows of 300 fp32 on one node: 9.1 us, with a launch for the sum 11.8; 700 workgroups a node: 28 us and 14)
    constexpr int64_t kMostAtCounter = 256;
    auto counter = [&](int64_t per_node) { return c->loss_left && s.n <= 65535 && per_node <= kMostAtCounter ? c->loss_left : nullptr; };
    auto count_launch = [&]() {
        return launch_blocks((uint64_t)s.n, kNodeThreads, [&](uint32_t first, dim3 grid) {
            k_count<<<grid, dim3(kNodeThreads), 0, c->stream>>>(labels, s.T, count, first);
        });
    };
    auto mean_launch = [&]() {
        return launch_blocks((uint64_t)s.n, kNodeThreads, [&](uint32_t first, dim3 grid) {
            k_loss_mean<<<grid, dim3(kNodeThreads), 0, c->stream>>>(rows, labels, s.T, loss, first);
        });
    };
    auto launch = [&](auto el) {
        typedef decltype(el) E;
        LossArgs<E> a = {};
        a.T = s.T;
        a.V = s.D;
        a.ld = s.ld;
        a.z = static_cast<const typename E::mem*>(logits);
        a.labels = labels;
        a.dz = static_cast<typename E::mem*>(dlogits);
        a.grad_scale = grad_scale;
        a.stream = stream_rows(s, logits, dlogits);
        a.loss = loss;
        const uint32_t all = (uint32_t)s.n * (uint32_t)s.T;
        if (cut.pieces) {
            if constexpr (!E::kNarrow) {
                a.pieces = cut.pieces;
                a.piece = cut.piece;
                a.parts = rows;
                a.per_node = (uint32_t)s.T * cut.pieces;
                a.left = counter((int64_t)s.T * cut.pieces);
                k_loss_parts<E><<<dim3(all * cut.pieces), dim3(kThreads), 0, c->stream>>>(a);
                hipError_t e = hipGetLastError();
                if (e == hipSuccess && !a.left) {
                    k_loss_join<E><<<dim3((uint32_t)s.n), dim3(kThreads), 0, c->stream>>>(a);
                    e = hipGetLastError();
                }
                if (e != hipSuccess || !a.dz) return e;
                k_loss_parts_grad<E><<<dim3(all * cut.pieces), dim3(kThreads), 0, c->stream>>>(a);
            }
            return hipGetLastError();
        }
        a.row_loss = rows;
        hipError_t e = hipSuccess;
        auto held_launch = [&](auto l, auto k) {
            constexpr int L = decltype(l)::value, N = decltype(k)::value, kBlock = L > kThreads ? L : kThreads;
            a.per_node = blocks_for(s.T, kBlock / L);
            a.left = counter(a.per_node);
            // few labels of a node are counted by the workgroup of a row itself, behind that row's loads
            if (s.T > 4 * kBlock) {
                a.count = count;
                e = count_launch();
            }
            if (e != hipSuccess) return;
            e = launch_blocks((uint64_t)a.per_node * s.n, kBlock, [&](uint32_t first, dim3 grid) {
                a.first_block = first;
                k_loss_held<E, L, N><<<grid, dim3(kBlock), 0, c->stream>>>(a);
            });
        };
        // the loss alone needs no row held: 8 x 512 rows of 32000 bf16 46 us, held 60
        const bool held = !(s.D > kHeldAlone && !dlogits) && with_row_shape<E>((s.D + kOct - 1) / kOct, held_launch);
        if constexpr (!E::kNarrow) {
            if (!held) {
                a.per_node = (uint32_t)s.T;
                if (dlogits && s.T > 4 * kNodeThreads) {
                    a.count = count;
                    e = count_launch();
                }
                if (e != hipSuccess) return e;
                e = launch_blocks(all, dlogits ? kNodeThreads : 512, [&](uint32_t first, dim3 grid) {
                    a.first_block = first;
                    if (dlogits) k_loss_swept<E, kNodeThreads><<<grid, dim3(kNodeThreads), 0, c->stream>>>(a);
                    else k_loss_swept<E, 512><<<grid, dim3(512), 0, c->stream>>>(a);
                });
            }
        }
        if (e != hipSuccess || a.left) return e;
        return mean_launch();
    };
    if (s.T == 0) return mean_launch();  // losses of 0
    return s.D < kOct ? with_narrow_elem(s.dtype, launch) : with_elem(s.dtype, launch);
}
