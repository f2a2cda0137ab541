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
// The items of a row of the table lie side by side in the sorted order, and their rows of dy are added in that order, which is
// the order of their positions.  A wavefront adds up to kRun items.  Longer rows (frequent tokens) are cut where the sorted
// order reaches a multiple of kRun: a wavefront for each such chunk leaves the sum of its part in `partial`, and
// k_embed_join adds the parts.  A chunk holds parts of at most two long rows, one that reaches its first item (slot 0) and
// one that reaches its last (slot 1, unless it is the same).
constexpr int kRun = 32;
constexpr int kTurns = 4;               // column turns kept in registers at once
constexpr int kTurnCols = kWave * 4;    // four columns a lane: an fp32 store of a wavefront is 1 KiB without gaps

struct GradArgs {
    const uint32_t* keys;   // sorted, T a node
    const int32_t* pos;
    const int32_t* start;   // V + 1 a node
    int32_t T, V, D;
    int64_t ld, ldg;
    float scale;
    int32_t accumulate;
    uint32_t chunks;            // of a node
    uint32_t chunk_blocks;      // workgroups of a node that take chunks; the others take rows
    uint32_t blocks_per_node;
    uint32_t rows_per_wave;     // 1 .. 64
    float* partial;             // n x chunks x 2 x D
    float* g;                   // the table's columns of node 0
};

// sum[k] = sum of columns (first_turn + k) * kTurnCols + 4 * lane .. + 3 over `count` <= 64 rows of dy; lane e holds the position of row e.
template <typename E>
__device__ __forceinline__ void sum_rows(const typename E::mem* __restrict__ rows, int64_t ld, int32_t D, int32_t at, int32_t count, int32_t c0,
                                         float (*sum)[4]) {
#pragma unroll
    for (int k = 0; k < kTurns; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[k][j] = 0.f;
    constexpr int kAhead = 4;  // rows whose loads are under way together
    int32_t e = 0;
    for (; e + kAhead <= count; e += kAhead) {
        float v[kAhead][kTurns][4];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const typename E::mem* row = rows + (int64_t)__builtin_amdgcn_readlane(at, e + i) * ld;
#pragma unroll
            for (int k = 0; k < kTurns; ++k)
                if (c0 + k * kTurnCols < D) row_load4<E>(row, c0 + k * kTurnCols, D, v[i][k]);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
#pragma unroll
            for (int k = 0; k < kTurns; ++k)
                if (c0 + k * kTurnCols < D)
#pragma unroll
                    for (int j = 0; j < 4; ++j) sum[k][j] += v[i][k][j];
    }
    for (; e < count; ++e) {
        const typename E::mem* row = rows + (int64_t)__builtin_amdgcn_readlane(at, e) * ld;
#pragma unroll
        for (int k = 0; k < kTurns; ++k)
            if (c0 + k * kTurnCols < D) {
                float v[4];
                row_load4<E>(row, c0 + k * kTurnCols, D, v);
#pragma unroll
                for (int j = 0; j < 4; ++j) sum[k][j] += v[j];
            }
    }
}

template <typename E>
__global__ __launch_bounds__(kThreads) void k_embed_grad(GradArgs a, const typename E::mem* __restrict__ dy) {
    const uint32_t node = blockIdx.x / a.blocks_per_node, b = blockIdx.x - node * a.blocks_per_node;
    const int lane = threadIdx.x & (kWave - 1);
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const uint32_t* keys = a.keys + (int64_t)node * a.T;
    const int32_t* pos = a.pos + (int64_t)node * a.T;
    const int32_t* start = a.start + (int64_t)node * (a.V + 1ll);
    const typename E::mem* rows = dy + (int64_t)node * a.T * a.ld;
    float sum[kTurns][4];
    if (b < a.chunk_blocks) {
        const uint32_t chunk = b * (kThreads / kWave) + wave;
        if (chunk >= a.chunks) return;
        const int32_t first = (int32_t)chunk * kRun, end = a.T - first < kRun ? a.T : first + kRun;
        const uint32_t head = keys[first], tail = keys[end - 1];
        float* part = a.partial + ((int64_t)node * a.chunks + chunk) * 2 * a.D;
        for (int slot = 0; slot < 2; ++slot) {
            const uint32_t key = slot ? tail : head;
            if (key >= (uint32_t)a.V || (slot && tail == head)) continue;
            const int32_t row_from = start[key], row_to = start[key + 1];
            if (row_to - row_from <= kRun) continue;
            const int32_t from = slot ? row_from : first, to = row_to < end ? row_to : end;
            const int32_t at = pos[from + (lane < to - from ? lane : 0)];
            for (int32_t c0 = lane * 4; c0 - lane * 4 < a.D; c0 += kTurns * kTurnCols) {
                sum_rows<E>(rows, a.ld, a.D, at, to - from, c0, sum);
#pragma unroll
                for (int k = 0; k < kTurns; ++k)
                    if (c0 + k * kTurnCols < a.D) row_store4<ElemF32>(part + (int64_t)slot * a.D, c0 + k * kTurnCols, a.D, sum[k]);
            }
        }
        return;
    }
    const bool bad = a.T > 0 && keys[a.T - 1] == (uint32_t)a.V + 1u;
    const int64_t v0 = ((int64_t)(b - a.chunk_blocks) * (kThreads / kWave) + wave) * a.rows_per_wave;
    const int32_t mine = a.V - v0 < (int64_t)a.rows_per_wave ? (int32_t)(a.V - v0) : (int32_t)a.rows_per_wave;
    if (mine <= 0) return;
    const int32_t begin = start[v0 + (lane < mine ? lane : mine)], next = start[v0 + (lane < mine ? lane + 1 : mine)];
    uint64_t todo = __ballot(lane < mine && (bad || (next - begin <= kRun && (next > begin || !a.accumulate))));
    while (todo) {
        const int r = __builtin_ctzll(todo);
        todo &= todo - 1;
        const int32_t from = __builtin_amdgcn_readlane(begin, r), count = bad ? 0 : __builtin_amdgcn_readlane(next, r) - from;
        float* out = a.g + (int64_t)node * a.ldg + (v0 + r) * a.D;
        const int32_t at = count ? pos[from + (lane < count ? lane : 0)] : 0;
        for (int32_t c0 = lane * 4; c0 - lane * 4 < a.D; c0 += kTurns * kTurnCols) {
            sum_rows<E>(rows, a.ld, a.D, at, count, c0, sum);
#pragma unroll
            for (int k = 0; k < kTurns; ++k) {
                const int32_t c = c0 + k * kTurnCols;
                if (c >= a.D) break;
                float had[4] = {0.f, 0.f, 0.f, 0.f};
                if (a.accumulate) row_load4<ElemF32>(out, c, a.D, had);
#pragma unroll
                for (int j = 0; j < 4; ++j) sum[k][j] = bad ? __builtin_nanf("") : had[j] + a.scale * sum[k][j];
                row_store4<ElemF32>(out, c, a.D, sum[k]);
            }
        }
    }
}

// Adds the parts of each long row, kTurnCols columns a workgroup: the one whose chunk holds the row's first item.  Its wavefronts
// take contiguous shares of the parts; everything in a fixed order.
__global__ __launch_bounds__(kThreads) void k_embed_join(GradArgs a, uint32_t column_blocks) {
    constexpr int kWaves = kThreads / kWave;
    __shared__ float s_part[kWaves][kTurnCols];
    const uint32_t unit = blockIdx.x / column_blocks, node = unit / a.chunks, chunk = unit - node * a.chunks;
    const uint32_t* keys = a.keys + (int64_t)node * a.T;
    const int32_t* start = a.start + (int64_t)node * (a.V + 1ll);
    const int32_t first = (int32_t)chunk * kRun, end = a.T - first < kRun ? a.T : first + kRun;
    const uint32_t key = keys[end - 1];
    if (key >= (uint32_t)a.V || keys[a.T - 1] == (uint32_t)a.V + 1u) return;
    const int32_t row_from = start[key], row_to = start[key + 1];
    if (row_from < first || row_to - row_from <= kRun) return;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int32_t c = (int32_t)(blockIdx.x - unit * column_blocks) * kTurnCols + lane * 4;
    const uint32_t parts = (uint32_t)(row_to - 1) / kRun - chunk + 1, share = (parts + kWaves - 1) / kWaves;
    const uint32_t from = wave * share, to = from + share < parts ? from + share : parts;
    const float* part = a.partial + ((int64_t)node * a.chunks + chunk) * 2 * a.D;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    if (c < a.D) {
#pragma unroll 4
        for (uint32_t p = from; p < to; ++p) {
            float v[4];
            row_load4<ElemF32>(part + ((int64_t)p * 2 + (p == 0 && row_from > first ? 1 : 0)) * a.D, c, a.D, v);
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[j] += v[j];
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) s_part[wave][j * kWave + lane] = sum[j];
    __syncthreads();
    if (wave == 0 && c < a.D) {
        float* out = a.g + (int64_t)node * a.ldg + (int64_t)key * a.D;
        float had[4] = {0.f, 0.f, 0.f, 0.f};
        if (a.accumulate) row_load4<ElemF32>(out, c, a.D, had);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            for (int w = 1; w < kWaves; ++w) sum[j] += s_part[w][j * kWave + lane];
            sum[j] = had[j] + a.scale * sum[j];
        }
        row_store4<ElemF32>(out, c, a.D, sum);
    }
}

uint32_t blocks_for(int64_t items, int64_t per_block) { return (uint32_t)((items + per_block - 1) / per_block); }

size_t padded(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

// Scratch of the gradient: sorted keys and positions (of the tiles, and merged where there are several), row starts, parts of long rows.
struct GradSpace {
    size_t items, tile_keys, tile_pos, keys, pos, start, partial, bytes;
    uint32_t tiles, chunks;
    GradSpace(const RowsShape& s, int32_t V) {
        items = (size_t)s.n * (size_t)s.T;
        tiles = s.T > 0 ? blocks_for(s.T, kTile) : 0;
        const size_t one = padded(items * 4);
        tile_keys = 0;
        tile_pos = one;
        keys = tiles > 1 ? 2 * one : tile_keys;
        pos = tiles > 1 ? 3 * one : tile_pos;
        start = (tiles > 1 ? 4 : 2) * one;
        partial = start + padded((size_t)s.n * ((size_t)V + 1) * 4);
        chunks = s.T > kRun ? blocks_for(s.T, kRun) : 0;  // no row is long otherwise
        bytes = partial + padded((size_t)s.n * chunks * 2 * (size_t)s.D * 4);
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
    GradArgs a = {};
    a.keys = words(space.keys);
    a.pos = ints(space.pos);
    a.start = ints(space.start);
    a.T = s.T;
    a.V = V;
    a.D = s.D;
    a.ld = s.ld;
    a.ldg = c->ld;
    a.scale = scale;
    a.accumulate = accumulate;
    a.chunks = space.chunks;
    a.chunk_blocks = blocks_for(a.chunks, kThreads / kWave);
    const int64_t spread = (int64_t)s.n * V / 16384;
    a.rows_per_wave = (uint32_t)(spread < 1 ? 1 : spread < 4 ? spread : 4);
    a.blocks_per_node = a.chunk_blocks + blocks_for(V, (int64_t)a.rows_per_wave * (kThreads / kWave));
    a.partial = reinterpret_cast<float*>(base + space.partial);
    a.g = c->g + table_off;
    hipError_t e2 = with_elem(s.dtype, [&](auto el) {
        typedef decltype(el) E;
        k_embed_grad<E><<<dim3(a.blocks_per_node * (uint32_t)s.n), dim3(kThreads), 0, c->stream>>>(a, static_cast<const typename E::mem*>(dy));
        return hipGetLastError();
    });
    if (e2 != hipSuccess || !a.chunks) return e2;
    const uint32_t column_blocks = blocks_for(s.D, kTurnCols);
    k_embed_join<<<dim3(a.chunks * column_blocks * (uint32_t)s.n), dim3(kThreads), 0, c->stream>>>(a, column_blocks);
    return hipGetLastError();
}
