// Cross-entropy of softmax(z) over a vocabulary, averaged over a node's counted tokens (label >= 0), and its gradient.
//
//   loss_i = (1/N_i) * sum over counted t of log sum_v exp(z_v - m) + (m - z_label),  m = max_v z_v
//   dz_v   = (a/N_i) * (exp(z_v - m) / sum - [v = label])                              rows that are not counted: 0
//
// The loss is a sum of two terms that are both at least 0: m is never added to the logarithm, so large logits cost no
// digits.  A label of V or more is never an address: the loss of its node and its row of dz are NaN.  A node without a
// counted token has loss 0 (NaN would spread to every node with the next gossip step).
#include "gpga_rows.hpp"

namespace {

constexpr int kThreads = 256;
constexpr int kCountThreads = 256;

template <typename E>
struct LossArgs {
    typedef typename E::mem mem;
    int32_t T, V;
    int64_t ld;
    const mem* z;
    const int32_t* labels;
    mem* dz;            // may be NULL
    float* row_loss;    // n*T
    const int32_t* count;  // n: counted tokens
    float grad_scale;
};

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1) v += __shfl_xor(v, off, kWave);
    return v;
}

// Counted tokens of each node; a workgroup a node.
__global__ __launch_bounds__(kCountThreads) void k_count(const int32_t* __restrict__ labels, int32_t T, int32_t* __restrict__ count) {
    __shared__ int32_t s_count[kCountThreads / kWave];
    int32_t mine = 0;
    for (int32_t t = threadIdx.x; t < T; t += kCountThreads) mine += labels[(int64_t)blockIdx.x * T + t] >= 0;
    for (int off = kWave / 2; off > 0; off >>= 1) mine += __shfl_xor(mine, off, kWave);
    if ((threadIdx.x & (kWave - 1)) == 0) s_count[threadIdx.x / kWave] = mine;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kCountThreads / kWave; ++w) mine += s_count[w];
        count[blockIdx.x] = mine;
    }
}

template <typename E>
__global__ __launch_bounds__(kThreads) void k_token_loss(LossArgs<E> a) {
    __shared__ float s_max[kThreads / kWave], s_sum[kThreads / kWave];
    const int64_t r = blockIdx.x;
    const int32_t label = a.labels[r];
    const typename E::mem* z = a.z + r * a.ld;
    typename E::mem* dz = a.dz ? a.dz + r * a.ld : nullptr;
    if (label < 0) {
        if (threadIdx.x == 0) a.row_loss[r] = 0.f;
        if (dz) {
            const float zero[kOct] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            for (int32_t c = threadIdx.x * kOct; c < a.V; c += kThreads * kOct) row_store<E>(dz, c, a.V, zero);
        }
        return;
    }
    const int64_t node = r / a.T;
    float top = -INFINITY, v[kOct];
    bool nan = false;
    for (int32_t c = threadIdx.x * kOct; c < a.V; c += kThreads * kOct) {
        row_load<E>(z, c, a.V, v, -INFINITY);
#pragma unroll
        for (int j = 0; j < kOct; ++j) {
            top = fmaxf(top, v[j]);
            nan |= v[j] != v[j];
        }
    }
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, kWave));
    if ((threadIdx.x & (kWave - 1)) == 0) s_max[threadIdx.x / kWave] = top;
    __syncthreads();
    for (int w = 0; w < kThreads / kWave; ++w) top = fmaxf(top, s_max[w]);
    float sum = nan ? __builtin_nanf("") : 0.f;
    for (int32_t c = threadIdx.x * kOct; c < a.V; c += kThreads * kOct) {
        row_load<E>(z, c, a.V, v, -INFINITY);
#pragma unroll
        for (int j = 0; j < kOct; ++j) sum += c + j < a.V ? __expf(v[j] - top) : 0.f;
    }
    sum = lanes_sum<kThreads>(sum, s_sum);
    const bool bad = label >= a.V;
    const float picked = E::get(z[bad ? 0 : label]);
    __syncthreads();  // dz may take the place of z
    if (threadIdx.x == 0) a.row_loss[r] = bad ? __builtin_nanf("") : logf(sum) + (top - picked);
    if (!dz) return;
    const float scale = bad ? __builtin_nanf("") : a.grad_scale / (float)a.count[node];
    const float part = scale / sum;
    for (int32_t c = threadIdx.x * kOct; c < a.V; c += kThreads * kOct) {
        row_load<E>(z, c, a.V, v);
#pragma unroll
        for (int j = 0; j < kOct; ++j) v[j] = __expf(v[j] - top) * part - (c + j == label ? scale : 0.f);
        row_store<E>(dz, c, a.V, v);
    }
}

// Mean over the counted tokens of each node; sums in double, a fixed order.
__global__ __launch_bounds__(kCountThreads) void k_loss_mean(const float* __restrict__ row_loss, const int32_t* __restrict__ count, int32_t T,
                                                             float* __restrict__ loss) {
    __shared__ double s_sum[kCountThreads / kWave];
    double mine = 0.0;
    for (int32_t t = threadIdx.x; t < T; t += kCountThreads) mine += (double)row_loss[(int64_t)blockIdx.x * T + t];
    mine = wave_sum(mine);
    if ((threadIdx.x & (kWave - 1)) == 0) s_sum[threadIdx.x / kWave] = mine;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kCountThreads / kWave; ++w) mine += s_sum[w];
        const int32_t n = count[blockIdx.x];
        loss[blockIdx.x] = n > 0 ? (float)(mine / n) : 0.f;
    }
}

}  // namespace

size_t token_loss_scratch(const RowsShape& s) { return ((size_t)s.n * (size_t)s.T + (size_t)s.n) * 4; }

hipError_t launch_token_loss(const gpga_ctx* c, const RowsShape& s, const void* logits, const int32_t* labels, float grad_scale, float* loss,
                             void* dlogits, void* scratch) {
    int32_t* count = static_cast<int32_t*>(scratch);
    float* row_loss = reinterpret_cast<float*>(count + s.n);
    k_count<<<dim3((uint32_t)s.n), dim3(kCountThreads), 0, c->stream>>>(labels, s.T, count);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && s.T > 0) {
        e = with_elem(s.dtype, [&](auto el) {
            typedef decltype(el) E;
            LossArgs<E> a = {};
            a.T = s.T;
            a.V = s.D;
            a.ld = s.ld;
            a.z = static_cast<const typename E::mem*>(logits);
            a.labels = labels;
            a.dz = static_cast<typename E::mem*>(dlogits);
            a.row_loss = row_loss;
            a.count = count;
            a.grad_scale = grad_scale;
            k_token_loss<E><<<dim3((uint32_t)s.n * (uint32_t)s.T), dim3(kThreads), 0, c->stream>>>(a);
            return hipGetLastError();
        });
    }
    if (e != hipSuccess) return e;
    k_loss_mean<<<dim3((uint32_t)s.n), dim3(kCountThreads), 0, c->stream>>>(row_loss, count, s.T, loss);
    return hipGetLastError();
}
