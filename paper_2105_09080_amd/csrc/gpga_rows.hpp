// Shared by the language-model operators (embedding, dropout, layer norm, token loss): element types of activations,
// access to eight columns of a row, sums over the lanes of a row, the dropout mask, and the launchers.
//
// Activations are n * T rows, row i*T + t = token t of node i, of D elements (fp32, bf16 or fp16) with a common leading
// dimension ld >= D in elements.  Parameters are fp32 and lie in row i of X; their gradients go to the same columns of g.
// All arithmetic is fp32; a result is rounded to the activations' type once, where it is stored.
#pragma once

#include "gpga_internal.hpp"
#include "gpga_rng.hpp"

constexpr uint32_t TAG_DROPOUT = 4u;  // low byte of the fourth counter word, the layer above it

// ---- element types -------------------------------------------------------------------------------------------------
// Eight elements at a time.  Rows need only the alignment of an element: gfx950 takes 16-byte global accesses at any
// address, so a wide access is the same instruction for every leading dimension and column offset.

constexpr int kOct = 8;  // columns a lane owns in one piece (one Philox call gives the dropout lots of eight)

struct ElemF32 {
    typedef float mem;
    typedef float vec __attribute__((ext_vector_type(4), aligned(4)));
    static __device__ __forceinline__ float get(mem v) { return v; }
    static __device__ __forceinline__ mem put(float v) { return v; }
    static __device__ __forceinline__ void load8(const mem* p, float* v) {
        const vec a = *reinterpret_cast<const vec*>(p), b = *reinterpret_cast<const vec*>(p + 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[j] = a[j];
            v[4 + j] = b[j];
        }
    }
    static __device__ __forceinline__ void load4(const mem* p, float* v) {
        const vec a = *reinterpret_cast<const vec*>(p);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = a[j];
    }
    static __device__ __forceinline__ void store4(mem* p, const float* v) {
        vec a;
#pragma unroll
        for (int j = 0; j < 4; ++j) a[j] = v[j];
        *reinterpret_cast<vec*>(p) = a;
    }
    static __device__ __forceinline__ void store8(mem* p, const float* v) {
        vec a, b;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            a[j] = v[j];
            b[j] = v[4 + j];
        }
        *reinterpret_cast<vec*>(p) = a;
        *reinterpret_cast<vec*>(p + 4) = b;
    }
};

template <typename M>
struct Elem16 {
    typedef M mem;
    typedef M vec __attribute__((ext_vector_type(8), aligned(2)));
    typedef float wide __attribute__((ext_vector_type(8)));
    typedef M vec4 __attribute__((ext_vector_type(4), aligned(2)));
    static __device__ __forceinline__ float get(mem v) { return (float)v; }
    static __device__ __forceinline__ mem put(float v) { return (mem)v; }  // to nearest, ties to even
    static __device__ __forceinline__ void load8(const mem* p, float* v) {
        const wide w = __builtin_convertvector(*reinterpret_cast<const vec*>(p), wide);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = w[j];
    }
    static __device__ __forceinline__ void load4(const mem* p, float* v) {
        const v4f w = __builtin_convertvector(*reinterpret_cast<const vec4*>(p), v4f);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = w[j];
    }
    static __device__ __forceinline__ void store8(mem* p, const float* v) {
        wide w;
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = v[j];
        *reinterpret_cast<vec*>(p) = __builtin_convertvector(w, vec);
    }
};
typedef Elem16<__bf16> ElemBF16;
typedef Elem16<_Float16> ElemF16;

// Columns c .. c+7 of a row of D; columns past the end read as `fill` and are not stored.
template <typename E>
__device__ __forceinline__ void row_load(const typename E::mem* row, int32_t c, int32_t D, float* v, float fill = 0.f) {
    if (c + kOct <= D) {
        E::load8(row + c, v);
    } else {
#pragma unroll
        for (int j = 0; j < kOct; ++j) v[j] = c + j < D ? E::get(row[c + j]) : fill;
    }
}
template <typename E>
__device__ __forceinline__ void row_store(typename E::mem* row, int32_t c, int32_t D, const float* v) {
    if (c + kOct <= D) {
        E::store8(row + c, v);
    } else {
#pragma unroll
        for (int j = 0; j < kOct; ++j)
            if (c + j < D) row[c + j] = E::put(v[j]);
    }
}

// Columns c .. c+3 in the same way.
template <typename E>
__device__ __forceinline__ void row_load4(const typename E::mem* row, int32_t c, int32_t D, float* v) {
    if (c + 4 <= D) {
        E::load4(row + c, v);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = c + j < D ? E::get(row[c + j]) : 0.f;
    }
}
template <typename E>
__device__ __forceinline__ void row_store4(typename E::mem* row, int32_t c, int32_t D, const float* v) {
    if (c + 4 <= D) {
        E::store4(row + c, v);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (c + j < D) row[c + j] = E::put(v[j]);
    }
}

// ---- sums over the L lanes that share a row ---------------------------------------------------------------------------
// L <= 64: lanes of one wavefront; else the whole workgroup of L lanes, through `lds` (L / 64 floats).  Every lane gets the
// same bits.
template <int L>
__device__ __forceinline__ float lanes_sum(float v, float* lds) {
#pragma unroll
    for (int off = (L < kWave ? L : kWave) / 2; off > 0; off >>= 1) v += __shfl_xor(v, off, kWave);
    if (L > kWave) {
        __syncthreads();  // lds may still be read by the sum before this one
        if ((threadIdx.x & (kWave - 1)) == 0) lds[threadIdx.x / kWave] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int w = 0; w < L / kWave; ++w) v += lds[w];
    }
    return v;
}

// ---- dropout ---------------------------------------------------------------------------------------------------------
// Element (t, c) of node i in iteration k stays iff its 16-bit lot is at least `drop` = round(65536 p).  Lots 2j and 2j+1 of
// columns 8q .. 8q+7 are the lower and upper half of word j of Philox(t * ceil(D/8) + q, i, k, 4 + 256 layer) under the
// seed.  Sixteen bits a lot: p is kept to 2^-17 and one call of ten rounds serves eight elements; what stays is scaled by
// 65536 / (65536 - drop), so the expectation is exact for the p that is used.
struct DropArgs {
    uint32_t k0, k1;    // seed
    uint32_t iter, tag;
    uint32_t drop;      // 0: no dropout
    float factor;
};
struct DropNode {
    PhiloxPair pair;
    __device__ __forceinline__ DropNode(const DropArgs& a, uint32_t node) : pair(node, a.iter, a.k0, a.k1) {}
    __device__ __forceinline__ void apply(const DropArgs& a, uint32_t group, float* v) const {
        const u32x4 r = philox_rounds(PhiloxQuad(group, a.tag, a.k1), pair, a.k0, a.k1);
        const uint32_t w[4] = {r.a, r.b, r.c, r.d};
#pragma unroll
        for (int j = 0; j < 4; ++j) {  // selected, not multiplied by 0: what is dropped may be infinite
            v[2 * j] = (w[j] & 0xffffu) >= a.drop ? v[2 * j] * a.factor : 0.f;
            v[2 * j + 1] = (w[j] >> 16) >= a.drop ? v[2 * j + 1] * a.factor : 0.f;
        }
    }
};

// ---- launchers (gpga_embed.hip, gpga_norm.hip, gpga_token_loss.hip) ------------------------------------------------------
struct RowsShape {
    int32_t n, T, D;
    int64_t ld;
    int32_t dtype;  // gpga_dtype
};

hipError_t launch_embed(const gpga_ctx* c, const RowsShape& s, const int32_t* tokens, int64_t table_off, int32_t V, float scale, void* y);
size_t embed_grad_scratch(const RowsShape& s);
hipError_t launch_embed_grad(const gpga_ctx* c, const RowsShape& s, const int32_t* tokens, int64_t table_off, int32_t V, float scale,
                             const void* dy, bool accumulate, void* scratch);
hipError_t launch_dropout(const gpga_ctx* c, const RowsShape& s, const DropArgs& drop, const void* x, const void* residual, void* y);
hipError_t launch_norm(const gpga_ctx* c, const RowsShape& s, const DropArgs& drop, const void* x, const void* residual, int64_t gamma_off,
                       int64_t beta_off, float eps, void* u, void* y, float* stats);
size_t norm_grad_scratch(const RowsShape& s);
hipError_t launch_norm_grad(const gpga_ctx* c, const RowsShape& s, const DropArgs& drop, const void* dy, const void* u, const float* stats,
                            const void* more, int64_t gamma_off, int64_t beta_off, void* du, void* dx, bool accumulate, void* scratch);
size_t token_loss_scratch(const RowsShape& s);
hipError_t launch_token_loss(const gpga_ctx* c, const RowsShape& s, const void* logits, const int32_t* labels, float grad_scale, float* loss,
                             void* dlogits, void* scratch);

// Calls f with a value of the element type that `dtype` names.
template <typename F>
inline hipError_t with_elem(int32_t dtype, F&& f) {
    switch (dtype) {
        case GPGA_F32: return f(ElemF32());
        case GPGA_BF16: return f(ElemBF16());
        default: return f(ElemF16());
    }
}
