// Embedding lookup with scaling, and its gradient by sorted tokens, for n nodes with a table each.
//
//   y[i,t,:]  = scale * E_i[tok[i,t],:]
//   dE_i[v,:] = scale * sum over t with tok[i,t] = v of dy[i,t,:]        (+ what g holds, if it is to be added to)
//
// tok < 0 is padding (a row of zeros, no gradient); a token of V or more is never an address: its row of y is NaN, and in
// the gradient the whole block of its node.
#include <utility>

#include "gpga_rows.hpp"

namespace {

constexpr int kThreads = 256;

// ---- lookup ----------------------------------------------------------------------------------------------------------
// 2^lanes_log2 lanes a row, eight columns a lane and turn, kTurns turns' loads under way together.  One workgroup for each
// kThreads >> lanes_log2 rows of a node.  Bound by the rows written: 8 x 4096 rows of 768 bf16 out of 32000 fp32 rows a node in 17.9 us
// (50 MB written, 43 MB of distinct table rows: 5.2 TB/s).  One token a node: 3 us, a chain of two loads.
constexpr int kTurns = 3;

template <typename E>
__global__ __launch_bounds__(kThreads) void k_embed(const int32_t* __restrict__ tokens, const float* __restrict__ table, int64_t ldx,
                                                    int32_t V, int32_t D, int32_t T, uint32_t blocks_per_node, int lanes_log2, float scale,
                                                    typename E::mem* __restrict__ y, int64_t ld, bool stream, uint32_t first_block) {
    typedef Elem<float, E::kNarrow> P;
    const uint32_t block = first_block + blockIdx.x, node = block / blocks_per_node;
    const int32_t t = (int32_t)((block - node * blocks_per_node) * (uint32_t)(kThreads >> lanes_log2)) + (int32_t)(threadIdx.x >> lanes_log2);
    if (t >= T) return;
    const int64_t row = (int64_t)node * T + t;
    const int32_t tok = tokens[row];
    const bool real = tok >= 0 && tok < V;
    const float other = tok < 0 ? 0.f : __builtin_nanf("");
    const float* src = table + (int64_t)node * ldx + (int64_t)(real ? tok : 0) * D;
    typename E::mem* dst = y + row * ld;
    const int32_t step = kOct << lanes_log2, mine = (int32_t)(threadIdx.x & ((1u << lanes_log2) - 1u)) * kOct;
    for (int32_t c0 = 0; c0 < D; c0 += kTurns * step) {
        Piece<P, kOct> in[kTurns];
#pragma unroll
        for (int k = 0; k < kTurns; ++k)
            if (c0 + k * step < D) in[k] = piece_load<kOct, P>(src, c0 + k * step + mine, D);
#pragma unroll
        for (int k = 0; k < kTurns; ++k) {
            const int32_t c = c0 + k * step + mine;
            if (c < D) {
                float v[kOct];
                piece_get<kOct, P>(in[k], c, D, v);
#pragma unroll
                for (int j = 0; j < kOct; ++j) v[j] = real ? v[j] * scale : other;
                piece_put<kOct, E>(dst, c, D, v, stream);
            }
        }
    }
}

// ---- sorting the tokens of a node ---------------------------------------------------------------------------------------
// A workgroup sorts a tile of (token, position) pairs in LDS, least significant digit first and stable, so equal tokens stay in
// the order of their positions; k_merge puts the tiles of a node together, in pairs, where there are several.  Keys: the token, V for
// padding, V + 1 for a token that is out of range.  Digits have up to 10 bits: counting them costs one step a bit whatever their
// width, and a pass over the tile more is what costs.  The workgroups behind those zero the table's columns of g, which takes
// longer than the sort and waits for nothing.
constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / kWave;
constexpr int kTile = 8 * kSortThreads;       // items of a tile, the last one's fewer
constexpr int kDigitBits = 10, kDigits = 1 << kDigitBits;
static_assert(kDigits == kSortThreads, "a thread a digit");

struct ZeroArgs {
    uint32_t sorting;       // workgroups; those behind them zero
    uint32_t per_node;
    int64_t count, ldg;     // floats of a node's block, distance of the blocks
    float* g;
};
// One piece of four floats a lane: 786 MB are zeroed in 125 us (110 at least) beside the sort of 4096 tokens a node, and in 118 beside
// that of 8192, whose LDS leaves a compute unit one workgroup; with four pieces a lane the whole gradient took 169 us, with one
// 160.  The pieces are those of the 128-byte lines of memory, wherever in one the block begins: with pieces counted from its
// beginning 526 MB took 102 us at 8 bytes past a boundary, so 94.
constexpr int kZeroCols = kSortThreads * 4;

__device__ __forceinline__ void zero_block(const ZeroArgs& z, uint32_t b) {
    const uint32_t node = b / z.per_node;
    float* g = z.g + (int64_t)node * z.ldg;
    const int64_t before = (int64_t)(reinterpret_cast<uintptr_t>(g) / 4 % 32);  // floats of the first line in front of the block
    const int64_t e = (int64_t)(b - node * z.per_node) * kZeroCols + threadIdx.x * 4 - before;
    const float zero[4] = {0.f, 0.f, 0.f, 0.f};
    if (e >= 0 && e + 4 <= z.count) {
        piece_put<4, ElemF32>(g + e, 0, 4, zero);
    } else {
        for (int j = 0; j < 4; ++j)
            if (e + j >= 0 && e + j < z.count) g[e + j] = 0.f;
    }
}

// kItems items a thread: 8, or fewer where no tile has more.
template <int kItems>
__global__ __launch_bounds__(kSortThreads) void k_sort_tile(const int32_t* __restrict__ tokens, int32_t T, int32_t V, uint32_t tiles, int bits,
                                                            uint32_t* __restrict__ keys, int32_t* __restrict__ pos, ZeroArgs zero, uint32_t first_block) {
    const uint32_t block = first_block + blockIdx.x;
    if (block >= zero.sorting) {
        zero_block(zero, block - zero.sorting);
        return;
    }
    __shared__ uint32_t s_key[kItems * kSortThreads];
    __shared__ uint16_t s_pos[kItems * kSortThreads];
    __shared__ uint16_t s_count[kSortWaves][kDigits];
    __shared__ uint32_t s_total[kSortWaves];
    const uint32_t node = block / tiles;
    const int32_t base = (int32_t)(block - node * tiles) * kTile;
    const int64_t from = (int64_t)node * T + base;
    const int32_t count = T - base < kTile ? T - base : kTile;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int32_t first = wave * kWave * kItems + lane;  // item j of a lane: first + j * 64

    uint32_t key[kItems];
    uint16_t at[kItems];
#pragma unroll
    for (int j = 0; j < kItems; ++j) {
        const int32_t e = first + j * kWave;
        const int32_t tok = tokens[from + (e < count ? e : 0)];
        at[j] = (uint16_t)e;
        // past the end: behind everything
        key[j] = e >= count ? 0xffffffffu : tok < 0 ? (uint32_t)V : tok >= V ? (uint32_t)V + 1u : (uint32_t)tok;
    }
    const int passes = (bits + kDigitBits - 1) / kDigitBits, width = (bits + passes - 1) / passes;
    const uint32_t mask = (1u << width) - 1u;
    for (int pass = 0; pass < passes; ++pass) {
        for (int d = threadIdx.x; d < kSortWaves * kDigits / 2; d += kSortThreads) reinterpret_cast<uint32_t*>(&s_count[0][0])[d] = 0u;
        __syncthreads();
        // lanes whose item has the same digit, one step a bit: peers &= ~(ballot ^ own bit on all places)
        uint32_t rank[kItems], low[kItems], high[kItems];
#pragma unroll
        for (int j = 0; j < kItems; ++j) low[j] = high[j] = 0xffffffffu;
        for (int b = 0; b < width; ++b) {
#pragma unroll
            for (int j = 0; j < kItems; ++j) {
                const int32_t own = (int32_t)(key[j] << (31 - pass * width - b)) >> 31;
                const uint64_t set = __ballot(own != 0);
                low[j] = __builtin_amdgcn_bitop3_b32(low[j], (uint32_t)set, (uint32_t)own, 0x90);
                high[j] = __builtin_amdgcn_bitop3_b32(high[j], (uint32_t)(set >> 32), (uint32_t)own, 0x90);
            }
        }
#pragma unroll
        for (int j = 0; j < kItems; ++j) {
            const uint64_t peers = (uint64_t)high[j] << 32 | low[j];
            const uint32_t before = __builtin_popcountll(peers & ((1ull << lane) - 1ull));
            // one lane a digit counts for all its peers; a wavefront's LDS accesses stay in order
            volatile uint16_t* counter = &s_count[wave][(key[j] >> (pass * width)) & mask];
            const uint32_t had = *counter;
            __builtin_amdgcn_wave_barrier();
            if (before == 0) *counter = (uint16_t)(had + (uint32_t)__builtin_popcountll(peers));
            __builtin_amdgcn_wave_barrier();
            rank[j] = had + before;
        }
        __syncthreads();
        // where each wavefront's items of a digit begin: digits in order, wavefronts in order within a digit
        uint32_t total = 0, ahead;
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) total += s_count[w][threadIdx.x];
        ahead = total;
#pragma unroll
        for (int off = 1; off < kWave; off <<= 1) {
            const uint32_t up = __shfl_up(ahead, off, kWave);
            if (lane >= off) ahead += up;
        }
        if (lane == kWave - 1) s_total[wave] = ahead;
        __syncthreads();
        uint32_t begin = ahead - total;
        for (int w = 0; w < wave; ++w) begin += s_total[w];
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t held = s_count[w][threadIdx.x];
            s_count[w][threadIdx.x] = (uint16_t)begin;
            begin += held;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kItems; ++j) {
            const uint32_t to = s_count[wave][(key[j] >> (pass * width)) & mask] + rank[j];
            s_key[to] = key[j];
            s_pos[to] = at[j];
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kItems; ++j) {
            key[j] = s_key[first + j * kWave];
            at[j] = s_pos[first + j * kWave];
        }
    }
#pragma unroll
    for (int j = 0; j < kItems; ++j) {
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

// Merges sorted runs of `run` items in pairs, by rank: an item's place is its place in its run plus the items of the other run that
// come before it.
__global__ __launch_bounds__(kThreads) void k_merge(const uint32_t* __restrict__ from_keys, const int32_t* __restrict__ from_pos, int32_t T, int64_t run,
                                                    uint32_t blocks_per_node, uint32_t* __restrict__ keys, int32_t* __restrict__ pos) {
    const uint32_t node = blockIdx.x / blocks_per_node;
    const int64_t e = (int64_t)(blockIdx.x - node * blocks_per_node) * kThreads + threadIdx.x;
    if (e >= T) return;
    const uint32_t* mine = from_keys + (int64_t)node * T;
    const int64_t pair = e / (2 * run) * 2 * run;
    const bool second = e >= pair + run;
    const int64_t other = second ? pair : pair + run;  // the run beside
    const int64_t count = other >= T ? 0 : T - other < run ? T - other : run;
    const uint32_t key = mine[e];
    // equal tokens of the first run come first
    const int64_t to = e - (second ? run : 0) + (count ? keys_below(mine + other, (int32_t)count, second ? key + 1u : key) : 0);
    keys[(int64_t)node * T + to] = key;
    pos[(int64_t)node * T + to] = from_pos[(int64_t)node * T + e];
}

// ---- gradient ----------------------------------------------------------------------------------------------------------
// The items of a row of the table lie side by side in the sorted order, and their rows of dy are added in that order, which is
// the order of their positions.  A wavefront takes kTurnCols columns of kRun consecutive items, whatever rows they belong to, so frequent
// tokens cost no more than others.  A row that lies within its items goes straight to g; of a row that reaches into other chunks
// it leaves a part in `partial` (slot 0: the row of its first item, slot 1: the row of its last item where that is another),
// and k_embed_join adds the parts.  Rows without items hold the zeros of the sort's launch, or what g is to be added to.
//
// 8 x 4096 tokens, 32000 x 768 fp32 rows a node, bf16: zeros 125 us (6.3 TB/s) with the sort beside them, sums 31, joins 5.6; a
// wavefront a row of the table, which the most frequent token keeps for its 250 rows of dy, took 848 in all.  The sums after so
// large a fill wait (68 MB in 31 us; longer chunks and more loads under way change nothing); leaving used rows out of the zeros, to
// zero beside the sums, mixes reads and writes and took 170 to 218 in all.
constexpr int kRun = 16;
constexpr int kAhead = 8;               // items whose rows are loaded together
constexpr int kTurnCols = kWave * 4;    // columns of a wavefront, four a lane: an fp32 store is 1 KiB without gaps
constexpr int kMostTurns = 16;          // wavefronts of a workgroup, all of one chunk: the lines that two share stay on one XCD

struct GradArgs {
    const uint32_t* keys;   // sorted, T a node
    const int32_t* pos;
    uint32_t n, first_block;
    int32_t T, V, D;
    int64_t ld, ldg;
    float scale;
    int32_t accumulate;
    uint32_t chunks;            // of a node
    uint32_t column_blocks;     // of kTurnCols
    uint32_t column_groups;     // workgroups that these make
    float* partial;             // n x chunks x 2 x D
    float* g;                   // the table's columns of node 0
};

// Four columns of a row of g from their sum and what g holds.
template <typename P>
__device__ __forceinline__ void put_sum(const GradArgs& a, float* out, int32_t c, const float* had, const float* sum) {
    float v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = had[j] + a.scale * sum[j];
    piece_put<4, P>(out, c, a.D, v);
}

template <typename E, bool kAdd>
__global__ __launch_bounds__(kMostTurns * kWave) void k_embed_grad(GradArgs a, const typename E::mem* __restrict__ dy) {
    typedef Elem<float, E::kNarrow> P;
    const int lane = threadIdx.x & (kWave - 1);
    const uint32_t block = a.first_block + blockIdx.x;
    const uint32_t unit = block / a.column_groups, group = block - unit * a.column_groups, node = unit / a.chunks, chunk = unit - node * a.chunks;
    const uint32_t* keys = a.keys + (int64_t)node * a.T;
    const int32_t first = (int32_t)chunk * kRun, count = a.T - first < kRun ? a.T - first : kRun;
    const uint32_t key = keys[first + (lane < count ? lane : count - 1)];
    const int32_t at = a.pos[(int64_t)node * a.T + first + (lane < count ? lane : count - 1)];
    const uint32_t end = keys[a.T - 1], before = chunk ? keys[first - 1] : 0xffffffffu, after = first + count < a.T ? keys[first + count] : 0xffffffffu;
    if (end == (uint32_t)a.V + 1u) {  // a token was out of range: NaN everywhere, a share of the block for each workgroup
        const int64_t all = (int64_t)a.V * a.D, shares = (int64_t)a.chunks * a.column_groups, share = (all + shares - 1) / shares;
        const int64_t from = ((int64_t)chunk * a.column_groups + group) * share, to = from + share < all ? from + share : all;
        for (int64_t e = from + threadIdx.x; e < to; e += blockDim.x) a.g[(int64_t)node * a.ldg + e] = __builtin_nanf("");
        return;
    }
    const uint32_t down = __shfl_down(key, 1, kWave);
    // items that are the last of their row here, and those of padding, which is behind all rows
    const uint64_t last = __ballot(lane < count && (lane == count - 1 || key != down)), padding = __ballot(lane < count && key >= (uint32_t)a.V);
    const int real = padding ? __builtin_ctzll(padding) : count;
    const int32_t c = (int32_t)(group * blockDim.x + threadIdx.x) * 4;
    const bool on = c < a.D;
    const typename E::mem* rows = dy + (int64_t)node * a.T * a.ld;
    float* g = a.g + (int64_t)node * a.ldg;
    float* part = a.partial + ((int64_t)node * a.chunks + chunk) * 2 * a.D;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    bool fresh = true;  // the row began within the chunk
    for (int e = 0; e < real; e += kAhead) {
        Piece<E, 4> in[kAhead];
        Piece<P, 4> held[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int item = e + i < real ? e + i : real - 1;  // loads without a branch: the last item again
            in[i] = piece_load<4, E>(rows + (int64_t)__builtin_amdgcn_readlane(at, item) * a.ld, c, a.D);
            if (kAdd && (last >> item & 1))
                held[i] = piece_load<4, P>(g + (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)key, item) * a.D, c, a.D);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (e + i < real) {
                float v[4];
                piece_get<4, E>(in[i], c, a.D, v);
                if (e + i == 0) fresh = (uint32_t)__builtin_amdgcn_readlane((int)key, 0) != before;
#pragma unroll
                for (int j = 0; j < 4; ++j) sum[j] += v[j];
                if (last >> (e + i) & 1) {
                    const uint32_t row = (uint32_t)__builtin_amdgcn_readlane((int)key, e + i);
                    const bool goes_on = e + i == count - 1 && row == after;
                    if (on) {
                        float had[4] = {0.f, 0.f, 0.f, 0.f};
                        if (kAdd) piece_get<4, P>(held[i], c, a.D, had);
                        // slot 0 if the row holds the first item too
                        if (fresh && !goes_on) put_sum<P>(a, g + (int64_t)row * a.D, c, had, sum);
                        else piece_put<4, P>(part + (row == (uint32_t)__builtin_amdgcn_readlane((int)key, 0) ? 0 : a.D), c, a.D, sum);
                    }
                    sum[0] = sum[1] = sum[2] = sum[3] = 0.f;
                    fresh = true;
                }
            }
        }
    }
}

// Adds the parts of each row that reaches into several chunks, kTurnCols columns a wavefront: the one of the chunk in which the row
// begins.  Rows of more than kLongRow parts are added by the workgroup, a contiguous share for each of its wavefronts.
// Everything in a fixed order.
constexpr int kLongRow = 8;

template <typename P>
__device__ __forceinline__ void add_parts(const GradArgs& a, const float* part, uint32_t from, uint32_t to, bool second, int32_t c, float* sum) {
#pragma unroll 8
    for (uint32_t p = from; p < to; ++p) {
        float v[4];
        piece_read<4, P>(part + ((int64_t)p * 2 + (p == 0 && second ? 1 : 0)) * a.D, c, a.D, v);
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[j] += v[j];
    }
}
template <typename P>
__device__ __forceinline__ void put_row(const GradArgs& a, uint32_t node, uint32_t key, int32_t c, const float* sum) {
    float* out = a.g + (int64_t)node * a.ldg + (int64_t)key * a.D;
    float had[4] = {0.f, 0.f, 0.f, 0.f};
    if (a.accumulate) piece_read<4, P>(out, c, a.D, had);
    put_sum<P>(a, out, c, had, sum);
}

template <typename P>
__global__ __launch_bounds__(kThreads) void k_embed_join(GradArgs a, uint32_t blocks_per_node) {
    constexpr int kWaves = kThreads / kWave;
    __shared__ float s_part[kWaves][kTurnCols];
    __shared__ uint32_t s_parts[kWaves], s_key[kWaves];
    __shared__ bool s_second[kWaves];
    const uint32_t block = a.first_block + blockIdx.x, unit = block / a.column_blocks, node = unit / blocks_per_node, chunk0 = (unit - node * blocks_per_node) * kWaves;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const uint32_t chunk = chunk0 + wave;
    const uint32_t* keys = a.keys + (int64_t)node * a.T;
    const int32_t c = (int32_t)(block - unit * a.column_blocks) * kTurnCols + lane * 4;
    const float* parts_of_node = a.partial + (int64_t)node * a.chunks * 2 * a.D;
    const int64_t first = (int64_t)chunk * kRun, next = first + kRun;
    uint32_t parts = 0, key = 0;
    bool second = false;
    if (next < a.T) {  // otherwise nothing goes on from here
        const uint32_t at_first = keys[first], on = keys[next], ahead = chunk ? keys[first - 1] : 0xffffffffu, end = keys[a.T - 1];
        key = keys[next - 1];
        second = at_first != key;
        // the row goes on, is a row, and begins here
        if (key == on && key < (uint32_t)a.V && end <= (uint32_t)a.V && (second || ahead != key)) {
            parts = 1;  // this chunk's and those of the chunks that begin with the row
            for (uint64_t same = ~0ull; same == ~0ull; parts += (uint32_t)__builtin_popcountll(same)) {
                const int64_t at = first + (int64_t)(parts + lane) * kRun;
                same = __ballot(at < a.T && keys[at < a.T ? at : 0] == key);
            }
        }
    }
    if (parts && parts <= kLongRow && c < a.D) {
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
        add_parts<P>(a, parts_of_node + (int64_t)chunk * 2 * a.D, 0, parts, second, c, sum);
        put_row<P>(a, node, key, c, sum);
    }
    if (lane == 0) {
        s_parts[wave] = parts;
        s_key[wave] = key;
        s_second[wave] = second;
    }
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) {
        parts = s_parts[w];
        if (parts <= kLongRow) continue;
        const uint32_t share = (parts + kWaves - 1) / kWaves, from = wave * share, to = from + share < parts ? from + share : parts;
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
        if (c < a.D) add_parts<P>(a, parts_of_node + (int64_t)(chunk0 + w) * 2 * a.D, from, to, s_second[w], c, sum);
#pragma unroll
        for (int j = 0; j < 4; ++j) s_part[wave][j * kWave + lane] = sum[j];
        __syncthreads();
        if (wave == 0 && c < a.D) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                for (int v = 1; v < kWaves; ++v) sum[j] += s_part[v][j * kWave + lane];
            put_row<P>(a, node, s_key[w], c, sum);
        }
        __syncthreads();
    }
}

template <int V>
struct Const {
    static constexpr int value = V;
};

uint32_t blocks_for(int64_t items, int64_t per_block) { return (uint32_t)((items + per_block - 1) / per_block); }

size_t padded(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

// Scratch of the gradient: sorted keys and positions (twice where tiles are merged), parts of rows.
struct GradSpace {
    size_t keys[2], pos[2], partial, bytes;
    uint32_t tiles, chunks;
    explicit GradSpace(const RowsShape& s) {
        tiles = s.T > 0 ? blocks_for(s.T, kTile) : 0;
        chunks = s.T > 0 ? blocks_for(s.T, kRun) : 0;
        const size_t one = padded((size_t)s.n * (size_t)s.T * 4);
        keys[0] = 0;
        pos[0] = one;
        keys[1] = tiles > 1 ? 2 * one : 0;
        pos[1] = tiles > 1 ? 3 * one : one;
        partial = (tiles > 1 ? 4 : 2) * one;
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
    auto launch = [&](auto e) {
        typedef decltype(e) E;
        return launch_blocks((uint64_t)per_node * s.n, kThreads, [&](uint32_t first, dim3 grid) {
            k_embed<E><<<grid, dim3(kThreads), 0, c->stream>>>(tokens, c->x + table_off, c->ld, V, s.D, s.T, per_node, lanes_log2, scale,
                                                               static_cast<typename E::mem*>(y), s.ld, stream_rows(s, y), first);
        });
    };
    return s.D < kOct ? with_narrow_elem(s.dtype, launch) : with_elem(s.dtype, launch);
}

size_t embed_grad_scratch(const RowsShape& s) { return GradSpace(s).bytes; }

hipError_t launch_embed_grad(const gpga_ctx* c, const RowsShape& s, const int32_t* tokens, int64_t table_off, int32_t V, float scale,
                             const void* dy, bool accumulate, void* scratch) {
    const GradSpace space(s);
    char* base = static_cast<char*>(scratch);
    auto words = [&](size_t at) { return reinterpret_cast<uint32_t*>(base + at); };
    auto ints = [&](size_t at) { return reinterpret_cast<int32_t*>(base + at); };
    int bits = 0;
    while (bits < 32 && ((uint32_t)V + 1u) >> bits) ++bits;
    ZeroArgs zero = {};
    zero.sorting = space.tiles * (uint32_t)s.n;
    zero.count = (int64_t)V * s.D;
    zero.per_node = accumulate ? 0 : blocks_for(zero.count + 31, kZeroCols);
    zero.ldg = c->ld;
    zero.g = c->g + table_off;
    const uint64_t blocks = zero.sorting + (uint64_t)zero.per_node * s.n;
    auto sort = [&](auto items) {
        return launch_blocks(blocks, kSortThreads, [&](uint32_t first, dim3 grid) {
            k_sort_tile<decltype(items)::value><<<grid, dim3(kSortThreads), 0, c->stream>>>(tokens, s.T, V, space.tiles, bits, words(space.keys[0]),
                                                                                           ints(space.pos[0]), zero, first);
        });
    };
    hipError_t e = s.T <= kSortThreads ? sort(Const<1>()) : s.T <= 4 * kSortThreads ? sort(Const<4>()) : sort(Const<8>());
    if (e != hipSuccess) return e;
    if (s.T == 0) return hipSuccess;
    uint32_t *keys = words(space.keys[0]), *other_keys = words(space.keys[1]);
    int32_t *pos = ints(space.pos[0]), *other_pos = ints(space.pos[1]);
    for (int64_t run = kTile; run < s.T; run *= 2) {
        const uint32_t per_node = blocks_for(s.T, kThreads);
        k_merge<<<dim3(per_node * (uint32_t)s.n), dim3(kThreads), 0, c->stream>>>(keys, pos, s.T, run, per_node, other_keys, other_pos);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
        std::swap(keys, other_keys);
        std::swap(pos, other_pos);
    }
    GradArgs a = {};
    a.n = (uint32_t)s.n;
    a.keys = keys;
    a.pos = pos;
    a.T = s.T;
    a.V = V;
    a.D = s.D;
    a.ld = s.ld;
    a.ldg = c->ld;
    a.scale = scale;
    a.accumulate = accumulate;
    a.chunks = space.chunks;
    a.column_blocks = blocks_for(s.D, kTurnCols);
    a.column_groups = blocks_for(a.column_blocks, kMostTurns);
    a.partial = reinterpret_cast<float*>(base + space.partial);
    a.g = c->g + table_off;
    auto launch = [&](auto el) {
        typedef decltype(el) E;
        const uint32_t threads = kWave * blocks_for(a.column_blocks, a.column_groups);
        const typename E::mem* rows = static_cast<const typename E::mem*>(dy);
        e = launch_blocks((uint64_t)a.chunks * a.column_groups * s.n, threads, [&](uint32_t first, dim3 grid) {
            a.first_block = first;
            if (accumulate) k_embed_grad<E, true><<<grid, dim3(threads), 0, c->stream>>>(a, rows);
            else k_embed_grad<E, false><<<grid, dim3(threads), 0, c->stream>>>(a, rows);
        });
        if (e != hipSuccess || a.chunks < 2) return e;
        const uint32_t per_node = blocks_for(a.chunks, kThreads / kWave);
        return launch_blocks((uint64_t)per_node * a.column_blocks * s.n, kThreads, [&](uint32_t first, dim3 grid) {
            a.first_block = first;
            k_embed_join<Elem<float, E::kNarrow>><<<grid, dim3(kThreads), 0, c->stream>>>(a, per_node);
        });
    };
    return s.D < 4 ? with_narrow_elem(s.dtype, launch) : with_elem(s.dtype, launch);
}
