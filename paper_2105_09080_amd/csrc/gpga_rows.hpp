// Shared by the language-model operators (embedding, dropout, layer norm, token loss): element types of activations,
// access to eight columns of a row, sums over the lanes of a row, the dropout mask, and the launchers.
//
// Activations are n * T rows, row i*T + t = token t of node i, of D elements (fp32, bf16 or fp16) with a common leading
// dimension ld >= D in elements.  Parameters are fp32 and lie in row i of X; their gradients go to the same columns of g.
// All arithmetic is fp32, but for the products of the operators with matrices, whose operands are pieces of 11 to 24 bits with fp32 sums
// (gpga_product.hpp); a result is rounded to the activations' type once, where it is stored.
#pragma once

#include "gpga_internal.hpp"
#include "gpga_rng.hpp"
#include "gpga_spans.hpp"

constexpr uint32_t TAG_DROPOUT = 4u;  // low byte of the fourth counter word, the layer above it

// ---- element types and pieces of a row -------------------------------------------------------------------------------
// A lane owns W consecutive columns of a row at a time, a piece (8 where the rows are those of activations, 4 where fp32 rows of
// g are written).  Rows need only the alignment of an element: gfx950 takes 16-byte global accesses at any address, so a wide
// access is the same instruction for every leading dimension and column offset.
//
// The last piece of a row whose D no W divides, and pieces behind the row, are read at column D - W instead, so loads need no
// branch and many are under way together; piece_get then moves the columns to their places.  What a piece holds of other
// lanes' columns is dropped there, so an output may take the place of an input.  Kinds with kNarrow read element by element:
// they are for rows shorter than a piece.
constexpr int kOct = 8;

template <typename M, bool kNarrow_>
struct Elem {
    typedef M mem;
    static constexpr bool kNarrow = kNarrow_;
    static __device__ __forceinline__ float get(mem v) { return (float)v; }
    static __device__ __forceinline__ mem put(float v) { return (mem)v; }  // to nearest, ties to even
};
typedef Elem<float, false> ElemF32;

template <typename E, int W>
struct Piece {
    static constexpr int kWords = W * (int)sizeof(typename E::mem) / 4;
    uint32_t w[kWords];
};

// Keeps the compiler from merging the two kinds of access into one plain one.
__device__ __forceinline__ void own_branch() { asm volatile(""); }

// `stream` (uniform): the access leaves no copy behind in the L2 caches, for arrays that they could not hold until the next
// operator comes (stream_rows below).
template <int W, typename E>
__device__ __forceinline__ Piece<E, W> piece_load(const typename E::mem* row, int32_t c, int32_t D, bool stream = false) {
    typedef typename E::mem M;
    Piece<E, W> p;
    if constexpr (E::kNarrow) {
        M v[W];
#pragma unroll
        for (int j = 0; j < W; ++j) v[j] = c + j < D ? row[c + j] : (M)0.f;
        __builtin_memcpy(p.w, v, sizeof(p.w));
    } else {
        constexpr int kLoad = Piece<E, W>::kWords < 4 ? Piece<E, W>::kWords : 4;
        typedef uint32_t vec __attribute__((ext_vector_type(kLoad), aligned(alignof(M))));
        const M* at = row + (c + W <= D ? c : D - W);
#pragma unroll
        for (int k = 0; k < Piece<E, W>::kWords / kLoad; ++k) {
            const vec* from = reinterpret_cast<const vec*>(at) + k;
            vec v;
            if (stream) {
                own_branch();
                v = __builtin_nontemporal_load(from);
                own_branch();
            } else {
                v = *from;
            }
#pragma unroll
            for (int j = 0; j < kLoad; ++j) p.w[k * kLoad + j] = v[j];
        }
    }
    return p;
}

// Columns c .. c+W-1 in fp32; 0 past the end of the row.  Of no meaning for c >= D.
template <int W, typename E>
__device__ __forceinline__ void piece_get(Piece<E, W> p, int32_t c, int32_t D, float* v) {
    typedef typename E::mem M;
    constexpr int N = Piece<E, W>::kWords, kPerWord = 4 / (int)sizeof(M);
    if (!E::kNarrow && D % W) {
        const bool tail = c + W > D;
        const uint32_t gone = (uint32_t)(W - D % W);  // columns before c that a last piece holds
#pragma unroll
        for (int step = N / 2; step > 0; step >>= 1)
            if (gone / kPerWord & step) {
#pragma unroll
                for (int k = 0; k < N; ++k) p.w[k] = tail ? (k + step < N ? p.w[k + step] : 0u) : p.w[k];
            }
        if (kPerWord == 2 && (gone & 1)) {
#pragma unroll
            for (int k = 0; k < N; ++k) p.w[k] = tail ? (k + 1 < N ? p.w[k + 1] << 16 : 0u) | p.w[k] >> 16 : p.w[k];
        }
    }
    if constexpr (sizeof(M) == 4) {
#pragma unroll
        for (int j = 0; j < W; ++j) v[j] = __builtin_bit_cast(float, p.w[j]);
    } else {
        typedef M pair __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int k = 0; k < N; ++k) {
            if constexpr (__is_same(M, __bf16)) {
                v[2 * k] = __builtin_bit_cast(float, p.w[k] << 16);
                v[2 * k + 1] = __builtin_bit_cast(float, p.w[k] & 0xffff0000u);
            } else {
                const pair h = __builtin_bit_cast(pair, p.w[k]);
                v[2 * k] = (float)h[0];
                v[2 * k + 1] = (float)h[1];
            }
        }
    }
}

// Both for one piece.
template <int W, typename E>
__device__ __forceinline__ void piece_read(const typename E::mem* row, int32_t c, int32_t D, float* v) {
    piece_get<W, E>(piece_load<W, E>(row, c, D), c, D, v);
}

// Columns c .. of the row, as many as there are, c < D.
template <int W, typename E>
__device__ __forceinline__ void piece_put(typename E::mem* row, int32_t c, int32_t D, const float* v, bool stream = false) {
    typedef typename E::mem M;
    typedef M vec __attribute__((ext_vector_type(W), aligned(alignof(M))));
    typedef float wide __attribute__((ext_vector_type(W)));
    if (!E::kNarrow && c + W <= D) {
        wide f;
#pragma unroll
        for (int j = 0; j < W; ++j) f[j] = v[j];
        vec* to = reinterpret_cast<vec*>(row + c);
        const vec out = __builtin_convertvector(f, vec);
        if (stream) {
            own_branch();
            __builtin_nontemporal_store(out, to);
            own_branch();
        } else {
            *to = out;
        }
    } else {
#pragma unroll
        for (int j = 0; j < W; ++j)
            if (c + j < D) row[c + j] = E::put(v[j]);
    }
}

// ---- sums and maxima over the lanes that share a row -----------------------------------------------------------------------
// All of an aligned group of L lanes of a wavefront, L = 8, 16, 32 or 64; every lane gets the same bits.  Lanes of 16 by DPP
// (exchange with the neighbour, the pair, the mirrored eight, the mirrored sixteen), rows of 16 by the swaps of gfx950; no
// LDS.
template <int kCtrl>
__device__ __forceinline__ float dpp(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), kCtrl, 0xf, 0xf, true));
}
template <int L, typename F>
__device__ __forceinline__ float wave_all(float v, F&& f) {
    v = f(v, dpp<0xb1>(v));
    v = f(v, dpp<0x4e>(v));
    v = f(v, dpp<0x141>(v));
    if constexpr (L > 8) v = f(v, dpp<0x140>(v));
    if constexpr (L > 16) {
        const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = f(__uint_as_float(s[0]), __uint_as_float(s[1]));
    }
    if constexpr (L > 32) {
        const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = f(__uint_as_float(s[0]), __uint_as_float(s[1]));
    }
    return v;
}
template <int L>
__device__ __forceinline__ float wave_sum(float v) {
    return wave_all<L>(v, [](float a, float b) { return a + b; });
}
template <int L>
__device__ __forceinline__ float wave_max(float v) {
    return wave_all<L>(v, [](float a, float b) { return fmaxf(a, b); });
}

// Sums of K values over L lanes; for L > 64 over the whole workgroup of L lanes, through `lds` (K * L / 64 floats), which no
// lane may still be reading: two sums in a row need different ones.
template <int L, int K>
__device__ __forceinline__ void lanes_sum(float (&v)[K], float* lds) {
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = wave_sum<(L < kWave ? L : kWave)>(v[k]);
    if constexpr (L > kWave) {
        if ((threadIdx.x & (kWave - 1)) == 0) {
#pragma unroll
            for (int k = 0; k < K; ++k) lds[threadIdx.x / kWave * K + k] = v[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            v[k] = lds[k];
#pragma unroll
            for (int w = 1; w < L / kWave; ++w) v[k] += lds[w * K + k];
        }
    }
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
size_t token_loss_scratch(const RowsShape& s, int num_cus);
hipError_t launch_token_loss(const gpga_ctx* c, const RowsShape& s, const void* logits, const int32_t* labels, float grad_scale, float* loss,
                             void* dlogits, void* scratch);

// Gated feed-forward block (gpga_gated_ff.hip): T tokens a node, matrices at column offsets of X.
struct FfShape {
    int32_t n, T, D, F;
    int64_t ld;
    int32_t dtype, act;
    int64_t gate_off, up_off, down_off;
};
size_t gated_ff_scratch(const FfShape& s, bool grad);
hipError_t launch_gated_ff(const gpga_ctx* c, const FfShape& s, const void* x, void* hidden, void* y, void* scratch);
hipError_t launch_gated_ff_grad(const gpga_ctx* c, const FfShape& s, const void* dy, const void* x, const void* hidden, void* dx, bool accumulate,
                                void* scratch);

// Orthogonalised updates (gpga_orthogonalize.hip): `count` matrices of R x C a node, one after another.
struct OrthShape {
    int32_t n, R, C, count;
};
size_t orthogonalize_scratch(const OrthShape& s);
// Largest singular value that any of the steps can lead to.
double orthogonalize_bound(int32_t steps, const float* coefficients);
hipError_t launch_orthogonalize(const gpga_ctx* c, const OrthShape& s, int64_t off, float* v, float mu, bool nesterov, int32_t steps,
                                const float* coefficients, float eps, float scale, void* scratch);

// Whether accesses to activation arrays stream past the L2 caches (4 MiB for each of 8 XCDs): arrays of 32 MiB and more whose rows
// begin on 16-byte boundaries.  Streaming stores that end within a line are written by themselves: 8 x 1537 rows of 3642
// bf16 took 35 us with them and 25 without.
template <typename... P>
inline bool stream_rows(const RowsShape& s, P... arrays) {
    const int64_t size = s.dtype == GPGA_F32 ? 4 : 2;
    uintptr_t at = (uintptr_t)(s.ld * size);
    for (const void* p : {static_cast<const void*>(arrays)...}) at |= reinterpret_cast<uintptr_t>(p);
    return (at & 15u) == 0 && (int64_t)s.n * s.T * s.D * size >= 32ll << 20;
}

// Launches `blocks` workgroups of `threads`: f(first, grid) launches those from number `first` on.
template <typename F>
inline hipError_t launch_blocks(uint64_t blocks, uint32_t threads, F&& f) {
    return for_launches(blocks, threads, [&](uint32_t first, uint32_t count) {
        f(first, dim3(count));
        return hipGetLastError();
    });
}

// Calls f with a value of the kind of element that `dtype` names; the narrow kinds are for rows shorter than a piece.
template <typename F>
inline hipError_t with_elem(int32_t dtype, F&& f) {
    switch (dtype) {
        case GPGA_F32: return f(Elem<float, false>());
        case GPGA_BF16: return f(Elem<__bf16, false>());
        default: return f(Elem<_Float16, false>());
    }
}
template <typename F>
inline hipError_t with_narrow_elem(int32_t dtype, F&& f) {
    switch (dtype) {
        case GPGA_F32: return f(Elem<float, true>());
        case GPGA_BF16: return f(Elem<__bf16, true>());
        default: return f(Elem<_Float16, true>());
    }
}
