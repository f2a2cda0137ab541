// Embedding lookup with scaling, and its gradient by sorted tokens, for n nodes with a table each.
//
//   y[i,t,:]  = scale * E_i[tok[i,t],:]
//   dE_i[v,:] = scale * sum over t with tok[i,t] = v of dy[i,t,:]        (+ what g holds, if it is to be added to)
//
// tok < 0 is padding (a row of zeros, no gradient); a token of V or more is never an address: its row of y is NaN, and in
// the gradient the whole block of its node.
#include "gpga_rows.hpp"

namespace {

constexpr int kThreads = 256;

// ---- lookup ----------------------------------------------------------------------------------------------------------
// 2^lanes_log2 lanes a row, eight columns a lane and turn.  One workgroup for each kThreads >> lanes_log2 rows of a node.
template <typename E>
__global__ __launch_bounds__(kThreads) void k_embed(const int32_t* __restrict__ tokens, const float* __restrict__ table, int64_t ldx,
                                                    int32_t V, int32_t D, int32_t T, uint32_t blocks_per_node, int lanes_log2, float scale,
                                                    typename E::mem* __restrict__ y, int64_t ld) {
    const uint32_t node = blockIdx.x / blocks_per_node;
    const int32_t t = (int32_t)((blockIdx.x - node * blocks_per_node) * (uint32_t)(kThreads >> lanes_log2)) + (int32_t)(threadIdx.x >> lanes_log2);
    if (t >= T) return;
    const int64_t row = (int64_t)node * T + t;
    const int32_t tok = tokens[row];
    const bool real = tok >= 0 && tok < V;
    const float other = tok < 0 ? 0.f : __builtin_nanf("");
    const float* src = table + (int64_t)node * ldx + (int64_t)(real ? tok : 0) * D;
    typename E::mem* dst = y + row * ld;
    const int32_t step = kOct << lanes_log2;
#pragma unroll 2
    for (int32_t c = (int32_t)(threadIdx.x & ((1u << lanes_log2) - 1u)) * kOct; c < D; c += step) {
        float v[kOct];
        if (real) {
            row_load<ElemF32>(src, c, D, v);
#pragma unroll
            for (int j = 0; j < kOct; ++j) v[j] *= scale;
        } else {
#pragma unroll
            for (int j = 0; j < kOct; ++j) v[j] = other;
        }
        row_store<E>(dst, c, D, v);
    }
}

// ---- sorting the tokens of a node ---------------------------------------------------------------------------------------
// A workgroup sorts a tile of kTile (token, position) pairs in LDS, least significant digit first and stable, so equal
// tokens stay in the order of their positions; k_merge puts the tiles of a node together.  Keys: the token, V for padding,
// V + 1 for a token that is out of range.
constexpr int kSortThreads = 1024;
constexpr int kSortItems = 4;
constexpr int kTile = kSortThreads * kSortItems;
constexpr int kSortWaves = kSortThreads / kWave;
constexpr int kDigits = 256;

__global__ __launch_bounds__(kSortThreads) void k_sort_tile(const int32_t* __restrict__ tokens, int32_t T, int32_t V, uint32_t tiles, int bits,
                                                            uint32_t* __restrict__ keys, int32_t* __restrict__ pos) {
    __shared__ uint32_t s_key[kTile];
    __shared__ uint16_t s_pos[kTile];
    __shared__ uint32_t s_count[kSortWaves][kDigits];
    __shared__ uint32_t s_total[kDigits / kWave];
    const uint32_t node = blockIdx.x / tiles;
    const int32_t base = (int32_t)(blockIdx.x - node * tiles) * kTile;
    const int64_t from = (int64_t)node * T + base;
    const int32_t count = T - base < kTile ? T - base : kTile;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int32_t first = wave * kWave * kSortItems + lane;  // item j of a lane: first + j * 64

    uint32_t key[kSortItems];
    uint16_t at[kSortItems];
#pragma unroll
    for (int j = 0; j < kSortItems; ++j) {
        const int32_t e = first + j * kWave;
        at[j] = (uint16_t)e;
        key[j] = 0xffffffffu;  // past the end: behind everything
        if (e < count) {
            const int32_t tok = tokens[from + e];
            key[j] = tok < 0 ? (uint32_t)V : tok >= V ? (uint32_t)V + 1u : (uint32_t)tok;
        }
    }
    const int passes = (bits + 7) / 8, width = (bits + passes - 1) / passes;
    const uint32_t mask = (1u << width) - 1u;
    for (int pass = 0; pass < passes; ++pass) {
        for (int d = threadIdx.x; d < kSortWaves * kDigits; d += kSortThreads) (&s_count[0][0])[d] = 0u;
        __syncthreads();
        uint32_t rank[kSortItems];
#pragma unroll
        for (int j = 0; j < kSortItems; ++j) {
            const uint32_t digit = (key[j] >> (pass * width)) & mask;
            uint64_t peers = ~0ull;
            for (int b = 0; b < width; ++b) {
                const uint64_t set = __ballot((digit >> b) & 1u);
                peers &= ((digit >> b) & 1u) ? set : ~set;
            }
            const uint32_t before = __builtin_popcountll(peers & ((1ull << lane) - 1ull));
            // one lane a digit counts for all its peers; a wavefront's LDS accesses stay in order
            volatile uint32_t* counter = &s_count[wave][digit];
            const uint32_t had = *counter;
            __builtin_amdgcn_wave_barrier();
            if (before == 0) *counter = had + (uint32_t)__builtin_popcountll(peers);
            __builtin_amdgcn_wave_barrier();
            rank[j] = had + before;
        }
        __syncthreads();
        // where each wavefront's items of a digit begin: digits in order, wavefronts in order within a digit
        uint32_t total = 0, ahead = 0;
        if (threadIdx.x < kDigits) {
            for (int w = 0; w < kSortWaves; ++w) total += s_count[w][threadIdx.x];
            ahead = total;
            for (int off = 1; off < kWave; off <<= 1) {
                const uint32_t up = __shfl_up(ahead, off, kWave);
                if (lane >= off) ahead += up;
            }
            if (lane == kWave - 1) s_total[wave] = ahead;
        }
        __syncthreads();
        if (threadIdx.x < kDigits) {
            uint32_t at_digit = ahead - total;
            for (int w = 0; w < wave; ++w) at_digit += s_total[w];
            for (int w = 0; w < kSortWaves; ++w) {
                const uint32_t held = s_count[w][threadIdx.x];
                s_count[w][threadIdx.x] = at_digit;
                at_digit += held;
            }
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kSortItems; ++j) {
            const uint32_t to = s_count[wave][(key[j] >> (pass * width)) & mask] + rank[j];
            s_key[to] = key[j];
            s_pos[to] = at[j];
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kSortItems; ++j) {
            key[j] = s_key[first + j * kWave];
            at[j] = s_pos[first + j * kWave];
        }
    }
#pragma unroll
    for (int j = 0; j < kSortItems; ++j) {
        const int32_t e = first + j * kWave;
        if (e < count) {
            keys[from + e] = key[j];
            pos[from + e] = base + (int32_t)at[j];
        }
    }
}

// Number of the `count` sorted keys that are below `key`.
__device__ __forceinline__ int32_t keys_below(const uint32_t* __restrict__ keys, int32_t count, uint32_t key) {
    int32_t lo = 0, hi = count;
    while (lo < hi) {
        const int32_t mid = (int32_t)(((uint32_t)lo + (uint32_t)hi) >> 1);
        if (keys[mid] < key) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

// Merges the sorted tiles of every node by rank (an item's place is its place in its tile plus the items of the other tiles
// that come before it) and finds where each row of the table begins in the sorted order: start[v] = items with a key
// below v, v = 0 .. V.  The first `merge_blocks` workgroups of a node merge, the others find.
__global__ __launch_bounds__(kThreads) void k_merge(const uint32_t* __restrict__ tile_keys, const int32_t* __restrict__ tile_pos, int32_t T, int32_t V,
                                                    uint32_t tiles, uint32_t merge_blocks, uint32_t blocks_per_node, uint32_t* __restrict__ keys,
                                                    int32_t* __restrict__ pos, int32_t* __restrict__ start) {
    const uint32_t node = blockIdx.x / blocks_per_node, b = blockIdx.x - node * blocks_per_node;
    const uint32_t* mine = tile_keys + (int64_t)node * T;
    if (b < merge_blocks) {
        const int32_t e = (int32_t)(b * kThreads + threadIdx.x);
        if (e >= T) return;
        const uint32_t own = (uint32_t)e / kTile, key = mine[e];
        int32_t to = e - (int32_t)own * kTile;
        for (uint32_t k = 0; k < tiles; ++k) {
            if (k == own) continue;
            const int32_t base = (int32_t)k * kTile, count = T - base < kTile ? T - base : kTile;
            to += keys_below(mine + base, count, k < own ? key + 1u : key);  // equal tokens of earlier tiles come first
        }
        keys[(int64_t)node * T + to] = key;
        pos[(int64_t)node * T + to] = tile_pos[(int64_t)node * T + e];
    } else {
        const uint32_t v = (b - merge_blocks) * kThreads + threadIdx.x;
        if (v > (uint32_t)V) return;
        int32_t below = 0;
        for (uint32_t k = 0; k < tiles; ++k) {
            const int32_t base = (int32_t)k * kTile, count = T - base < kTile ? T - base : kTile;
            below += keys_below(mine + base, count, v);
        }
        start[(int64_t)node * (V + 1ll) + v] = below;
    }
}

// ---- gradient ----------------------------------------------------------------------------------------------------------
// A wavefront takes rows of the table in turn: the items of a row lie side by side in the sorted order, and their rows of dy
// are added in the order of their positions.
template <typename E>
__global__ __launch_bounds__(kThreads) void k_embed_grad(const uint32_t* __restrict__ keys, const int32_t* __restrict__ pos,
                                                         const int32_t* __restrict__ start, int32_t T, int32_t V, int32_t D,
                                                         const typename E::mem* __restrict__ dy, int64_t ld, float scale, bool accumulate,
                                                         uint32_t rows_per_block, uint32_t blocks_per_node, float* __restrict__ g, int64_t ldg) {
    const uint32_t node = blockIdx.x / blocks_per_node, b = blockIdx.x - node * blocks_per_node;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const bool bad = T > 0 && keys[(int64_t)node * T + T - 1] == (uint32_t)V + 1u;
    const int32_t* at = pos + (int64_t)node * T;
    const int32_t* begin = start + (int64_t)node * (V + 1ll);
    const typename E::mem* rows = dy + (int64_t)node * T * ld;
    const int64_t last = ((int64_t)b + 1) * rows_per_block < V ? ((int64_t)b + 1) * rows_per_block : V;
    for (int64_t v = (int64_t)b * rows_per_block + wave; v < last; v += kThreads / kWave) {
        const int32_t from = begin[v], to = begin[v + 1];
        if (accumulate && from == to && !bad) continue;
        float* out = g + (int64_t)node * ldg + v * D;
        for (int32_t c = lane * kOct; c < D; c += kWave * kOct) {
            float sum[kOct] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            for (int32_t e = from; e < to; ++e) {
                float v8[kOct];
                row_load<E>(rows + (int64_t)at[e] * ld, c, D, v8);
#pragma unroll
                for (int j = 0; j < kOct; ++j) sum[j] += v8[j];
            }
            float had[kOct] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (accumulate) row_load<ElemF32>(out, c, D, had);
#pragma unroll
            for (int j = 0; j < kOct; ++j) sum[j] = bad ? __builtin_nanf("") : had[j] + scale * sum[j];
            row_store<ElemF32>(out, c, D, sum);
        }
    }
}

uint32_t blocks_for(int64_t items, int64_t per_block) { return (uint32_t)((items + per_block - 1) / per_block); }

size_t padded(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

// Scratch of the gradient: sorted keys and positions (of the tiles, and merged where there are several), row starts.
struct GradSpace {
    size_t items, tile_keys, tile_pos, keys, pos, start, bytes;
    uint32_t tiles;
    GradSpace(const RowsShape& s, int32_t V) {
        items = (size_t)s.n * (size_t)s.T;
        tiles = s.T > 0 ? blocks_for(s.T, kTile) : 0;
        const size_t one = padded(items * 4);
        tile_keys = 0;
        tile_pos = one;
        keys = tiles > 1 ? 2 * one : tile_keys;
        pos = tiles > 1 ? 3 * one : tile_pos;
        start = (tiles > 1 ? 4 : 2) * one;
        bytes = start + padded((size_t)s.n * ((size_t)V + 1) * 4);
    }
};

}  // namespace

hipError_t launch_embed(const gpga_ctx* c, const RowsShape& s, const int32_t* tokens, int64_t table_off, int32_t V, float scale, void* y) {
    // 32 lanes a row or more, fewer only where the row has no work for them; as many as leave the fewest idle in the last turn
    const int32_t octs = (s.D + kOct - 1) / kOct;
    int lanes_log2 = 0, least = 0;
    while (least < 5 && (1 << least) < octs) ++least;
    int64_t idle = -1;
    for (int l = least; l <= 8; ++l) {
        const int64_t turns = (octs + (1 << l) - 1) >> l, lost = (turns << l) - octs;
        if (idle < 0 || lost <= idle) {
            idle = lost;
            lanes_log2 = l;
        }
    }
    const uint32_t per_node = blocks_for(s.T, kThreads >> lanes_log2);
    return with_elem(s.dtype, [&](auto e) {
        typedef decltype(e) E;
        k_embed<E><<<dim3(per_node * (uint32_t)s.n), dim3(kThreads), 0, c->stream>>>(tokens, c->x + table_off, c->ld, V, s.D, s.T, per_node, lanes_log2,
                                                                                    scale, static_cast<typename E::mem*>(y), s.ld);
        return hipGetLastError();
    });
}

size_t embed_grad_scratch(const RowsShape& s, int32_t V) { return GradSpace(s, V).bytes; }

hipError_t launch_embed_grad(const gpga_ctx* c, const RowsShape& s, const int32_t* tokens, int64_t table_off, int32_t V, float scale,
                             const void* dy, bool accumulate, void* scratch) {
    const GradSpace space(s, V);
    char* base = static_cast<char*>(scratch);
    auto words = [&](size_t at) { return reinterpret_cast<uint32_t*>(base + at); };
    auto ints = [&](size_t at) { return reinterpret_cast<int32_t*>(base + at); };
    if (space.tiles) {
        int bits = 0;
        while (bits < 32 && ((uint32_t)V + 1u) >> bits) ++bits;
        k_sort_tile<<<dim3(space.tiles * (uint32_t)s.n), dim3(kSortThreads), 0, c->stream>>>(tokens, s.T, V, space.tiles, bits, words(space.tile_keys),
                                                                                           ints(space.tile_pos));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const uint32_t merge_blocks = space.tiles > 1 ? blocks_for(s.T, kThreads) : 0;
    const uint32_t merge_per_node = merge_blocks + blocks_for((int64_t)V + 1, kThreads);
    k_merge<<<dim3(merge_per_node * (uint32_t)s.n), dim3(kThreads), 0, c->stream>>>(words(space.tile_keys), ints(space.tile_pos), s.T, V, space.tiles,
                                                                                   merge_blocks, merge_per_node, words(space.keys), ints(space.pos),
                                                                                   ints(space.start));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const uint32_t rows_per_block = 16, per_node = blocks_for(V, rows_per_block);
    return with_elem(s.dtype, [&](auto el) {
        typedef decltype(el) E;
        k_embed_grad<E><<<dim3(per_node * (uint32_t)s.n), dim3(kThreads), 0, c->stream>>>(words(space.keys), ints(space.pos), ints(space.start), s.T, V, s.D,
                                                                                         static_cast<const typename E::mem*>(dy), s.ld, scale, accumulate,
                                                                                         rows_per_block, per_node, c->g + table_off, c->ld);
        return hipGetLastError();
    });
}
