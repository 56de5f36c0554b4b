// no_embed_fwd / no_embed_bwd: rows of a table by id, scaled, and the gradient of the table.
#include "rows.hpp"
#include "radix.hpp"

namespace no {

// out[i] = scale row_scale[id] table[id]: no arithmetic to speak of, bound by the rows' round trips. A group of lanes (a power of two, at most 64) copies a row in runs of
// W values, 16 bytes a lane or more on the wider side. The next row's id is requested before this row's values, so that a row costs one round trip, its scale beside it.
// 118000 rows of 256 e4m3 values with scales into bf16: 18.6 us, 4.8 TB/s of the bytes that it cannot do without (runs of 16 values: 22.3). Stores go past the caches (by them 26.9 us; read next, all in all 46.4 and 44.7). Up to 8192 blocks (2048: 30000 rows of 4096
// bf16 values 86.0 us for 84.5, 50000 x 1000 bf16 into fp32 65.5 for 59.6). Requests of several runs ahead gain nothing (four: 89.4 us for 83.5).
template <typename T, typename O, int W, bool SHORT>
__global__ void __launch_bounds__(256) embed_fwd_kernel(RowsOf table, int64_t n_rows, int32_t dim, const float* __restrict__ row_scale, const int32_t* __restrict__ ids,
                                                        const int32_t* d_n, int32_t cap, float scale, RowsOf out, int32_t g_log2) {
    const int32_t n = rows_here(d_n, cap), lane = lane_id(), g = 1 << g_log2, sub = lane >> g_log2, u0 = lane & (g - 1), rows = 64 >> g_log2;
    const int64_t wave = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 6, stride = (int64_t)gridDim.x * 4 * rows;
    int64_t r = wave * rows + sub;
    int32_t id = r < n ? ids[r] : -1;
    for (; r - sub < n; r += stride) {
        const int32_t next = r + stride < n ? ids[r + stride] : -1;
        const bool there = id >= 0 && id < n_rows;
        const float by = there ? (row_scale ? scale * row_scale[id] : scale) : 0.0f;
        const T* src = table.row<T>(there ? id : 0);
        for (int32_t c = u0 * W; c < dim && r < n; c += g * W) {
            const Place<W, SHORT> place(c, dim);
            Run<T, W> v;
            if (there) place.load(v, src);
            float f[W];
            v.get(f);
#pragma unroll
            for (int w = 0; w < W; ++w) f[w] = there ? f[w] * by : 0.0f;
            Run<O, W> o;
            o.set(f);
            if constexpr (SHORT) o.store(out.row<O>(r) + c, dim - c);
            else o.store_once(out.row<O>(r) + place.at);        // (what two lanes hold, both store)
        }
        id = next;
    }
}

template <typename T, typename O>
static void launch_embed(const RowsOf& table, int64_t n_rows, int32_t dim, const float* row_scale, const int32_t* ids, const int32_t* d_n, int32_t cap, float scale,
                         const RowsOf& out, hipStream_t st) {
    constexpr int W = sizeof(T) == 4 && sizeof(O) == 4 ? 4 : 8;
    const int32_t units = (int32_t)ceil_div(dim, W);
    int g_log2 = 0;
    while ((1 << g_log2) < units && g_log2 < 6) ++g_log2;
    int64_t blocks = ceil_div(ceil_div(cap, 64 >> g_log2), 4);
    if (blocks > 8192) blocks = 8192;
    if (dim >= W) hipLaunchKernelGGL((embed_fwd_kernel<T, O, W, false>), dim3((unsigned)blocks), dim3(256), 0, st, table, n_rows, dim, row_scale, ids, d_n, cap, scale, out, g_log2);
    else hipLaunchKernelGGL((embed_fwd_kernel<T, O, W, true>), dim3((unsigned)blocks), dim3(256), 0, st, table, n_rows, dim, row_scale, ids, d_n, cap, scale, out, g_log2);
}

// ------------------------------------------------------------------------------------------------------- gradient
//
// G[v] = scale * sum over the positions i with ids[i] == v of g[i]. The positions are ordered by id (stable, so by position within an id); then the
// ordered list is cut into chunks of 8 to 64 positions whatever the ids are, and a lane group walks a chunk with the sum of the id at hand
// in registers: an id that is named a thousand times costs what a thousand rare ones do. Sums of ids that lie inside a chunk go
// straight to the table; those that reach over a chunk's border go to the workspace and are added up, in chunk order, by a second launch. Rows that no
// id names are found by a search in the ordered ids and cleared beside the sums. No float atomics: the same ids give the same bits.
// Bound by memory: every gradient row is read once, every table row written once. 65536 rows of 2048 bf16 values, popular ids, into 131072 rows: 295 us, of which order 5.5 + 8.3 + 4.8,
// sums 265 (1.34 GB, 5.1 TB/s), borders 15.

constexpr int EMBED_TILE = 1024;                    // positions that a block orders in LDS
// Positions that need no order (embed_few_kernel), while they have few columns too. 777 positions of 100 columns: 6.3 us for 13.5, all of one id 16.3 for 14.9; 200 of 8000: 12.0 for 14.2;
// but 1000 of 8000: 37.8 for 26.2.
constexpr int32_t EMBED_FEW = 1024;
static inline bool embed_few(int32_t n, int32_t dim) { return n <= 256 || (n <= EMBED_FEW && n * ceil_div(dim, 256) <= 4096); }
// Positions whose places are counted in one launch; more are ordered by tiles and ranks (6000 of 64 columns: 22.2 us by counting, 20.7 by tiles; 8192: 23.3 and 20.8).
constexpr int32_t EMBED_RANK_MOST = 4096;
// More than these go through the radix sort (131072 of 64 columns: 66 us by tiles, 76 by radix; 200000: 129 and 95).
constexpr int32_t EMBED_MERGE_MOST = 131072;

// Chunks shorter than 64 are taken while 64 and so on down to twice their length leave fewer than 1024 wavefronts' work, n * (512 columns' worth of wavefronts) / (2 chunk) < 1025: their parts are these values at most, and a row.
constexpr int64_t EMBED_SHORT_PARTS = 2050 * 512;

struct EmbedPlan {      // the workspace, cut up
    int64_t n, tiles, chunks;
    int32_t chunk;
    bool merged, radix;
    size_t keys, pos, keys_tmp, pos_tmp, rank, sort_ws, parts, total;
    EmbedPlan(int32_t n_, int32_t dim) : n(n_), tiles(ceil_div(n_, EMBED_TILE)), chunk(64) {
        // Long chunks leave few sums to join (65536 positions of 2048 columns: all in all 296 us by chunks of 64, 323 of 16), as long as
        // there are wavefronts for the whole chip, four to a compute unit with eight rows each on their way (107952 x 65 bf16: 48.5 us, for eight to a compute unit 57.1, for two 47.7; 18834 x 176:
        // 25.0, 25.0 and 26.9).
        const int64_t units = ceil_div(dim, 8), lanes = (int64_t)1 << ilog2_ceil((uint64_t)(units < 64 ? units : 64));
        while (chunk > 8 && n * ceil_div(units, 64) * lanes / 64 / chunk < 1024) chunk >>= 1;
        chunks = ceil_div(n, chunk);
        radix = n > EMBED_MERGE_MOST;
        merged = !radix && n > EMBED_RANK_MOST;
        const size_t list = (size_t)(tiles ? tiles : 1) * EMBED_TILE * 4;
        keys = 0;
        pos = keys + list;
        keys_tmp = pos + list;
        pos_tmp = keys_tmp + (merged || radix ? list : 0);
        rank = pos_tmp + (merged || radix ? list : 0);
        sort_ws = rank + (merged ? list : 0);
        parts = sort_ws + (radix ? (size_t)ceil_div((int64_t)radix_ws_bytes(n), 16) * 16 : 0);
        total = embed_few(n_, dim) ? 16 : parts + (size_t)chunks * 2 * (size_t)dim * 4 + 16;
    }
    // Room for any plan of these sizes or smaller ones (a plan's own needs do not grow with them): a program makes one workspace for its longest list.
    size_t room(int32_t dim) const {
        if (embed_few((int32_t)n, dim)) return 16;
        const size_t list = (size_t)tiles * EMBED_TILE * 4, ranks = n <= EMBED_RANK_MOST ? 0 : n <= EMBED_MERGE_MOST ? list : (size_t)EMBED_MERGE_MOST * 4;
        const size_t sort = radix ? (size_t)ceil_div((int64_t)RadixPlan(n).room_words() * 4, 16) * 16 : 0;
        const int64_t least = ceil_div(n, 64) * dim, most = ceil_div(n, 8) * dim, brief = most < EMBED_SHORT_PARTS + dim ? most : EMBED_SHORT_PARTS + dim;
        return list * (n <= EMBED_RANK_MOST ? 2 : 4) + (ranks > sort ? ranks : sort) + (size_t)(least > brief ? least : brief) * 8 + 16;
    }
};

// The place of a position in the order by id, then by position, is the number of positions before it in that order. n^2 comparisons, but in one
// launch and from registers: a lane per position, and the sixteen wavefronts of a block take the positions it is compared with 64 at a time, which are wholly
// left of the block's own, its own, or right of them: equal ids count on the left, by lane among its own, and not on the right.
__global__ void __launch_bounds__(1024) embed_count_kernel(const int32_t* __restrict__ ids, const int32_t* d_n, int32_t cap, uint32_t* keys, uint32_t* pos) {
    __shared__ uint32_t part[16][64];
    const int32_t n = rows_here(d_n, cap), own = (int32_t)blockIdx.x;
    if (own * 64 >= n) return;
    const int32_t lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int32_t)(threadIdx.x >> 6)), i = own * 64 + lane;
    const uint32_t* key = reinterpret_cast<const uint32_t*>(ids);       // ids outside the table are larger than all inside, as unsigned
    const uint32_t mine = i < n ? key[i] : 0u;
    uint32_t before = 0;
    for (int32_t g = wave; g * 64 < n; g += 16) {
        const uint32_t* const p = key + g * 64;
        if (g != own && (g + 1) * 64 <= n) {                            // scalar loads: 64 ids in four requests
            if (g < own) {
#pragma unroll
                for (int q = 0; q < 64; ++q) before += p[q] <= mine;
            } else {
#pragma unroll
                for (int q = 0; q < 64; ++q) before += p[q] < mine;
            }
        } else {                                                        // its own, or the last ones, behind whose end nothing counts
            const int32_t here = g * 64 + lane < n ? (int32_t)p[lane] : -1;
#pragma unroll
            for (int q = 0; q < 64; ++q) {
                const uint32_t k = (uint32_t)__builtin_amdgcn_readlane(here, q);
                before += k < mine || (k == mine && g == own && q < lane);
            }
        }
    }
    part[wave][lane] = before;
    __syncthreads();
    if (wave == 0 && i < n) {
        uint32_t at = 0;
#pragma unroll
        for (int w = 0; w < 16; ++w) at += part[w][lane];
        keys[at] = mine;
        pos[at] = (uint32_t)i;
    }
}

// A tile's positions in order: a bitonic network over (id, position in the tile), an element a thread; distances under 64 stay in a wavefront, the ten steps of more go
// through LDS. K: 32 bits where the ids leave 10 of them, else 64. Ids outside the table come last, and behind them what is not there (~0).
template <typename K>
__global__ void __launch_bounds__(1024) embed_tile_kernel(const int32_t* __restrict__ ids, const int32_t* d_n, int32_t cap, uint32_t n_rows, uint32_t* keys, uint32_t* pos,
                                                          uint32_t* rank) {
    __shared__ K held[2][EMBED_TILE];
    const int32_t n = rows_here(d_n, cap), base = (int32_t)blockIdx.x * EMBED_TILE, t = threadIdx.x, here = min(EMBED_TILE, n - base);
    if (here <= 0) return;
    K x = t < here ? (K)min((uint32_t)ids[base + t], n_rows) << 10 | (K)t : ~(K)0;
    int turn = 0;
    // (written out: with the distances as constants a step is half of the instructions, which sixteen wavefronts on one compute unit pay for)
#pragma unroll
    for (int k = 2; k <= EMBED_TILE; k <<= 1)
#pragma unroll
        for (int j = k >> 1; j > 0; j >>= 1) {
            K o;
            if (j >= 64) {              // (the other half of `held` was read before the barrier of the step between)
                held[turn][t] = x;
                __syncthreads();
                o = held[turn][t ^ j];
                turn ^= 1;
            } else if constexpr (sizeof(K) == 4) o = (K)__shfl_xor((int)x, j, 64);
            else o = (K)__shfl_xor((unsigned long long)x, j, 64);
            const K small = o < x ? o : x, large = o < x ? x : o;
            x = ((t & k) == 0) == ((t & j) == 0) ? small : large;
        }
    const bool there = t < here;
    keys[base + t] = there ? (uint32_t)(x >> 10) : ~0u;
    pos[base + t] = there ? (uint32_t)(x & 1023) + (uint32_t)base : 0u;
    rank[base + t] = 0;
}

// An element's place among all tiles is the number of smaller ones in each, where equal ids count in the tiles left of its own. A block takes a tile's elements and a
// share of the tiles to search, four at a time, so that four searches go on beside each other; the shares add up in whole numbers, in any order.
__global__ void __launch_bounds__(1024) embed_rank_kernel(const uint32_t* __restrict__ keys, const int32_t* d_n, int32_t cap, int32_t shares, uint32_t* rank) {
    __shared__ __attribute__((aligned(16))) uint32_t held[4][EMBED_TILE];
    const int32_t n = rows_here(d_n, cap), own = (int32_t)blockIdx.x, t = threadIdx.x;
    if (own * EMBED_TILE >= n) return;
    const int32_t tiles = (n + EMBED_TILE - 1) / EMBED_TILE;
    const uint32_t key = keys[own * EMBED_TILE + t];
    uint32_t before = 0;
    for (int32_t o = blockIdx.y * 4; o < tiles; o += shares * 4) {
        __syncthreads();
        const int32_t part = t >> 8, quad = t & 255;
        reinterpret_cast<uint4*>(held[part])[quad] = o + part < tiles ? reinterpret_cast<const uint4*>(keys + (o + part) * EMBED_TILE)[quad] : uint4{~0u, ~0u, ~0u, ~0u};
        __syncthreads();
        // elements below key, or up to it in earlier tiles (key + 1 does not wrap: an id is at most n_rows; what is not there is not stored)
        uint32_t at[4] = {0, 0, 0, 0};
#pragma unroll
        for (int step = EMBED_TILE / 2; step > 0; step >>= 1)
#pragma unroll
            for (int q = 0; q < 4; ++q) at[q] += held[q][at[q] + step - 1] < (o + q < own ? key + 1 : key) ? step : 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (o + q >= tiles) continue;
            before += o + q == own ? (uint32_t)t : at[q] + (held[q][at[q]] < (o + q < own ? key + 1 : key));
        }
    }
    if (key != ~0u) atomicAdd(&rank[own * EMBED_TILE + t], before);
}

__global__ void __launch_bounds__(256) embed_place_kernel(const uint32_t* __restrict__ keys_in, const uint32_t* __restrict__ pos_in, const uint32_t* __restrict__ rank,
                                                          const int32_t* d_n, int32_t cap, uint32_t* keys, uint32_t* pos) {
    const int32_t n = rows_here(d_n, cap), i = (int32_t)(blockIdx.x * 256 + threadIdx.x);
    if (i / EMBED_TILE * EMBED_TILE >= n || keys_in[i] == ~0u) return;
    keys[rank[i]] = keys_in[i];
    pos[rank[i]] = pos_in[i];
}

// What the first pass of the radix sort reads: ids outside the table, and positions that are not there, come last.
struct IdSource {
    const int32_t* ids;
    const int32_t* d_n;
    int32_t cap;
    uint32_t none;
    __device__ __forceinline__ uint32_t key(int64_t i) const { return i < rows_here(d_n, cap) ? min((uint32_t)ids[i], none) : none; }
    __device__ __forceinline__ void keys_checked(int64_t i, int here, uint32_t (&k)[RS_ITEMS]) const {
#pragma unroll
        for (int it = 0; it < RS_ITEMS; ++it) k[it] = it < here ? key(i + it) : 0u;
    }
    __device__ __forceinline__ uint32_t val(int64_t i) const { return (uint32_t)i; }
};

struct EmbedSums {
    const uint32_t* keys;
    const uint32_t* pos;
    const int32_t* d_n;
    int32_t cap;
    float scale;
    bool accumulate;
    RowsOf grad, table;
    int64_t n_rows;
    int32_t dim, chunk; // positions a chunk
    float* parts;       // [chunks][2][dim]: the sum of an id that began in an earlier chunk, and of one that goes on in the next
};

// Clears those of the rows [v0, v0 + 16) whose bit is set.
__device__ __forceinline__ void clear_rows(const EmbedSums& a, int64_t v0, uint32_t empty) {
    Run<float, 4> zero;
    const float z[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    zero.set(z);
    const bool whole = a.dim >= 4;
    while (empty) {
        const int32_t at = __builtin_ctz(empty);
        empty &= empty - 1;
        float* row = a.table.row<float>(v0 + at);
        for (int32_t c = lane_id() * 4; c < a.dim; c += 256) {
            if (whole) zero.store(row + min(c, a.dim - 4));
            else zero.store(row + c, a.dim - c);
        }
    }
}

// Few positions, in one launch and without an order: a wavefront per position and 64 runs of columns looks its id up among all of them; where the position is the id's first it adds
// the rows of all of its positions, in order, and where these are many (more than four rounds of requests) the block's four wavefronts add a quarter each. Bound by the latency of its
// round trips: ids, the id's rows eight at a time, the table's.
template <typename T, int W, bool ADD, bool SHORT>
__global__ void __launch_bounds__(256) embed_few_kernel(EmbedSums a, const int32_t* __restrict__ ids, int32_t col_tiles, uint32_t sum_blocks) {
    constexpr int Q = EMBED_FEW / 64, UNR = 8;
    constexpr int32_t SHARED = 4 * UNR;
    __shared__ float part[4][W][64];
    __shared__ uint16_t list[4][EMBED_FEW];
    const int32_t n = rows_here(a.d_n, a.cap), lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int32_t)(threadIdx.x >> 6));
    int32_t id[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) id[q] = lane + q * 64 < n ? ids[lane + q * 64] : -1;
    for (int64_t v0 = ((int64_t)blockIdx.x - sum_blocks) * 64 + wave * 16; blockIdx.x >= sum_blocks; v0 += ((int64_t)gridDim.x - sum_blocks) * 64) {
        if (v0 >= a.n_rows) return;
        uint32_t named = 0;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int64_t at = id[q] - v0;
            named |= at >= 0 && at < 16 ? 1u << at : 0u;
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) named |= __shfl_xor(named, o, 64);
        const uint32_t empty = __builtin_amdgcn_readfirstlane(~named & (v0 + 16 <= a.n_rows ? 0xffffu : (1u << (a.n_rows - v0)) - 1u));
        clear_rows(a, v0, empty);
    }
    const int32_t item0 = (int32_t)blockIdx.x * 4, of = lane < 4 && (item0 + lane) / col_tiles < n ? ids[(item0 + lane) / col_tiles] : -1;
    for (int32_t it = 0; it < 4; ++it) {            // the block's four in turn, the same decisions in each wavefront
        const int32_t item = item0 + it, i = item / col_tiles, col = (item % col_tiles * 64 + lane) * W, width = a.dim - col;
        const int32_t mine = __builtin_amdgcn_readlane(of, it);
        if (mine < 0 || mine >= a.n_rows) continue;
        int32_t first = n, count = 0;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const uint64_t here = __ballot(id[q] == mine);
            if (here && count == 0) first = q * 64 + __builtin_ctzll(here);
            count += __builtin_popcountll(here);
        }
        const bool shared = count > SHARED;
        if (first != i || (!shared && wave != it)) continue;
        const Place<W, SHORT> place(width > 0 ? col : 0, a.dim);
        Run<float, W> old;
        float* const to = a.table.row<float>(mine);
        if (ADD && wave == it) place.load(old, (const float*)to);
        // of a shared id's positions those [from, from + share), by their place among them
        const int32_t share = shared ? (count + 3) / 4 : count, from = shared ? wave * share : 0;
        float acc[W];
#pragma unroll
        for (int w = 0; w < W; ++w) acc[w] = 0.0f;
        int32_t before = 0;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const uint64_t here = __ballot(id[q] == mine);
            const int32_t at = before + __builtin_popcountll(here & ((1ull << lane) - 1)) - from;
            if (id[q] == mine && at >= 0 && at < share) list[wave][at] = (uint16_t)(q * 64 + lane);
            before += __builtin_popcountll(here);
        }
        Team<64, 64>::sync();
        const int32_t len = min(share, count - from);
        for (int32_t j = 0; j < len; j += UNR) {
            Run<T, W> r[UNR];
            int32_t p[UNR];
#pragma unroll
            for (int k = 0; k < UNR; ++k) p[k] = list[wave][min(j + k, len - 1)];       // (behind the last the same row again, which does not count)
#pragma unroll
            for (int k = 0; k < UNR; ++k) place.load(r[k], (const T*)a.grad.row<T>(__builtin_amdgcn_readfirstlane(p[k])));
#pragma unroll
            for (int k = 0; k < UNR; ++k) {
                float f[W];
                r[k].get(f);
#pragma unroll
                for (int w = 0; w < W; ++w) acc[w] += j + k < len ? f[w] : 0.0f;
            }
        }
        Team<64, 64>::sync();                               // (the list is read)
        if (shared) {
            __syncthreads();                                // (the last shared id's sums are read)
#pragma unroll
            for (int w = 0; w < W; ++w) part[wave][w][lane] = acc[w];
            __syncthreads();
            if (wave != it) continue;
#pragma unroll
            for (int w = 0; w < W; ++w) acc[w] = ((part[0][w][lane] + part[1][w][lane]) + part[2][w][lane]) + part[3][w][lane];
        }
        if (width <= 0) continue;
        float f[W];
        if (ADD) old.get(f);
#pragma unroll
        for (int w = 0; w < W; ++w) f[w] = ADD ? f[w] + a.scale * acc[w] : a.scale * acc[w];
        place.store(f, to);
    }
}

template <typename T, int W, bool ADD, bool SHORT>
__global__ void __launch_bounds__(256) embed_sums_kernel(EmbedSums a, int64_t chunks, int32_t g_log2, int32_t col_tiles, uint32_t sum_blocks) {
    const int32_t n = rows_here(a.d_n, a.cap), lane = lane_id();
    for (int64_t v0 = ((int64_t)blockIdx.x - sum_blocks) * 64 + (threadIdx.x >> 6) * 16; blockIdx.x >= sum_blocks;
         v0 += ((int64_t)gridDim.x - sum_blocks) * 64) {     // rows without an id: 16 to a wavefront at a time
        if (v0 >= a.n_rows) return;
        const int64_t v = v0 + (lane & 15);
        int32_t lo = 0, hi = n;
        while (lo < hi) {
            const int32_t mid = lo + ((hi - lo) >> 1);
            if ((int64_t)a.keys[mid] < v) lo = mid + 1; else hi = mid;
        }
        const uint32_t empty = (uint32_t)__ballot(v < a.n_rows && !(lo < n && (int64_t)a.keys[lo] == v)) & 0xffffu;
        clear_rows(a, v0, empty);
    }
    const int32_t groups = 64 >> g_log2, u = lane & ((1 << g_log2) - 1);
    const int64_t item = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * groups + (lane >> g_log2);
    const int64_t chunk = item / col_tiles;
    const int32_t col = ((int32_t)(item % col_tiles) * 64 + u) * W, width = a.dim - col;
    const int64_t e0 = chunk * a.chunk;
    if (chunk >= chunks || e0 >= n || width <= 0) return;
    const int32_t len = (int32_t)min((int64_t)a.chunk, n - e0);
    const uint32_t before = chunk ? a.keys[e0 - 1] : ~0u, after = e0 + len < n ? a.keys[e0 + len] : ~0u;
    const Place<W, SHORT> place(col, a.dim);
    float* const parts = a.parts + chunk * 2 * a.dim;
    const uint32_t n_rows = (uint32_t)a.n_rows;     // (fewer than 2^31)
    float acc[W];
#pragma unroll
    for (int w = 0; w < W; ++w) acc[w] = 0.0f;
    int32_t start = 0;
    constexpr int UNR = ADD && W == 8 ? 4 : 8;      // rows requested before the first is added
    for (int32_t e = 0; e < len; e += UNR) {
        uint32_t key[UNR + 1], p[UNR];
        Run<T, W> r[UNR];
        Run<float, W> old[ADD ? UNR : 1];
#pragma unroll
        for (int k = 0; k < UNR; ++k) {
            key[k] = e + k < len ? a.keys[e0 + e + k] : ~0u;
            p[k] = e + k < len ? a.pos[e0 + e + k] : 0u;
        }
        key[UNR] = e + UNR < len ? a.keys[e0 + e + UNR] : ~0u;
#pragma unroll
        for (int k = 0; k < UNR; ++k) {
            if (key[k] >= n_rows) continue;
            place.load(r[k], (const T*)a.grad.row<T>(p[k]));
            // the row that a run's sum is added to, requested with the run's last gradient
            if (ADD && key[k + 1] != key[k]) place.load(old[ADD ? k : 0], (const float*)a.table.row<float>(key[k]));
        }
#pragma unroll
        for (int k = 0; k < UNR; ++k) {
            if (key[k] >= n_rows) continue;
            float f[W];
            r[k].get(f);
#pragma unroll
            for (int w = 0; w < W; ++w) acc[w] += f[w];
            if (key[k + 1] == key[k]) continue;     // (an id at the chunk's end goes on in the next, or does not: its sum is stored either way)
            const bool last = e + k + 1 == len;
            if (start == 0 && key[k] == before) place.store(acc, parts);
            else if (last && key[k] == after) place.store(acc, parts + a.dim);
            else {
                if constexpr (ADD) old[ADD ? k : 0].get(f);
#pragma unroll
                for (int w = 0; w < W; ++w) f[w] = ADD ? f[w] + a.scale * acc[w] : a.scale * acc[w];
                place.store(f, a.table.row<float>(key[k]));
            }
            start = e + k + 1;
#pragma unroll
            for (int w = 0; w < W; ++w) acc[w] = 0.0f;
        }
    }
}

// Adds up the sums that reach over borders: the chunk where such an id begins owns it. A wavefront looks at a chunk, counts the id's later chunks 64 at a time, and adds their
// parts by itself where they are few; the parts of an id with many are shared by the block's eight wavefronts.
template <bool SHORT>
__global__ void __launch_bounds__(512) embed_join_kernel(EmbedSums a, int64_t chunks) {
    constexpr int64_t FEW = 16;
    __shared__ float share[8][64][4];
    __shared__ int64_t many[8];             // parts of a wavefront's id, where they are many
    const int32_t n = rows_here(a.d_n, a.cap), lane = lane_id(), wave = (int32_t)(threadIdx.x >> 6), ch = a.chunk;
    const int32_t col = ((int32_t)blockIdx.y * 64 + lane) * 4, width = a.dim - col;
    const int64_t here = min(chunks, ceil_div(n, ch));
    const Place<4, SHORT> place(width > 0 ? col : 0, a.dim);
    auto add = [&](int64_t c, int64_t p0, int64_t p1, float (&acc)[4]) {
#pragma unroll 8
        for (int64_t p = p0; p < p1; ++p) {
            Run<float, 4> r;
            place.load(r, (const float*)a.parts + ((c + p) * 2 + (p == 0)) * a.dim);
            float f[4];
            r.get(f);
#pragma unroll
            for (int w = 0; w < 4; ++w) acc[w] += f[w];
        }
    };
    auto put = [&](uint32_t key, const float (&sum)[4]) {
        if (width <= 0) return;
        float* to = a.table.row<float>(key);
        float f[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (a.accumulate) {
            Run<float, 4> old;
            place.load(old, (const float*)to);
            old.get(f);
        }
#pragma unroll
        for (int w = 0; w < 4; ++w) f[w] += a.scale * sum[w];
        place.store(f, to);
    };
    for (int64_t c0 = (int64_t)blockIdx.x * 8; c0 + 1 < here; c0 += (int64_t)gridDim.x * 8) {
        const int64_t c = c0 + wave;
        int64_t parts = 0;
        uint32_t key = 0;
        float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (c + 1 < here) {
            // everything that most borders need at once, before it is known whether an id reaches over this one: the ids around it, the next chunks' first ids, the first two parts
            const uint32_t first = a.keys[c * ch], next = a.keys[(c + 1) * ch], prior = c > 0 ? a.keys[c * ch - 1] : ~0u;
            key = a.keys[(c + 1) * ch - 1];
            uint32_t ahead = a.keys[min(c + 2 + lane, here - 1) * ch];
            Run<float, 4> two[2];
            place.load(two[0], (const float*)a.parts + (c * 2 + 1) * a.dim);
            place.load(two[1], (const float*)a.parts + (c + 1) * 2 * a.dim);
            if ((int64_t)key < a.n_rows && next == key && !(first == key && prior == key)) {
                int64_t end = c + 2;            // the first chunk that does not begin with this id
                for (;;) {
                    const uint64_t same = __ballot(end + lane < here && ahead == key);
                    end += same == ~0ull ? 64 : __builtin_ctzll(~same);
                    if (same != ~0ull) break;
                    ahead = a.keys[min(end + lane, here - 1) * ch];
                }
                parts = end - c;
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    float f[4];
                    two[p].get(f);
#pragma unroll
                    for (int w = 0; w < 4; ++w) acc[w] += f[w];
                }
            }
        }
        if (parts > 0 && parts <= FEW) {
            add(c, 2, parts, acc);
            put(key, acc);
        }
        if (lane == 0) many[wave] = parts > FEW ? parts : 0;
        __syncthreads();
        for (int w = 0; w < 8; ++w) {
            const int64_t all = many[w], each = (all + 7) / 8, p0 = min(all, wave * each), p1 = min(all, p0 + each);
            if (all == 0) continue;
            float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            add(c0 + w, p0, p1, acc);
#pragma unroll
            for (int q = 0; q < 4; ++q) share[wave][lane][q] = acc[q];
            __syncthreads();
            if (wave == w) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    acc[q] = share[0][lane][q];
#pragma unroll
                    for (int o = 1; o < 8; ++o) acc[q] += share[o][lane][q];
                }
                put(key, acc);
            }
            __syncthreads();
        }
        __syncthreads();
    }
}

// Blocks that clear rows: 64 rows each, in turn where there are very many.
static int64_t clear_blocks(const EmbedSums& a) {
    const int64_t blocks = ceil_div(a.n_rows, 64);
    return a.accumulate ? 0 : blocks < (1 << 20) ? blocks : 1 << 20;
}

template <typename T>
static void launch_few(const EmbedSums& a, const int32_t* ids, hipStream_t st) {
    constexpr int W = 16 / (int)sizeof(T);
    const int32_t col_tiles = (int32_t)ceil_div(a.dim, 64 * W);
    const int64_t sum_blocks = ceil_div((int64_t)a.cap * col_tiles, 4);
    const dim3 grid((unsigned)(sum_blocks + clear_blocks(a)));
#define NO_AS(ADD, SHORT) hipLaunchKernelGGL((embed_few_kernel<T, W, ADD, SHORT>), grid, dim3(256), 0, st, a, ids, col_tiles, (uint32_t)sum_blocks)
    if (a.accumulate) { if (a.dim >= W) NO_AS(true, false); else NO_AS(true, true); }
    else { if (a.dim >= W) NO_AS(false, false); else NO_AS(false, true); }
#undef NO_AS
}

template <typename T>
static void launch_sums(const EmbedSums& a, int64_t chunks, hipStream_t st) {
    constexpr int W = 16 / (int)sizeof(T);
    const int32_t units = (int32_t)ceil_div(a.dim, W), col_tiles = (int32_t)ceil_div(units, 64);
    int g_log2 = 0;
    while ((1 << g_log2) < units && g_log2 < 6) ++g_log2;
    const int64_t sum_blocks = ceil_div(ceil_div(chunks * col_tiles, 64 >> g_log2), 4);
    const dim3 grid((unsigned)(sum_blocks + clear_blocks(a)));
#define NO_AS(ADD, SHORT) hipLaunchKernelGGL((embed_sums_kernel<T, W, ADD, SHORT>), grid, dim3(256), 0, st, a, chunks, g_log2, col_tiles, (uint32_t)sum_blocks)
    if (a.accumulate) { if (a.dim >= W) NO_AS(true, false); else NO_AS(true, true); }
    else { if (a.dim >= W) NO_AS(false, false); else NO_AS(false, true); }
#undef NO_AS
}

}  // namespace no

using namespace no;

extern "C" int32_t no_embed_fwd(const void* d_table, no_dtype dt, int64_t n_rows, int32_t dim, int64_t table_stride_bytes,
                                const float* d_row_scale, const int32_t* d_ids, const int32_t* d_n_ids, int32_t n_ids_cap, float scale,
                                void* d_out, no_dtype dt_out, int64_t out_stride_bytes, void* stream) {
    clear_error();
    NO_REQUIRE(dt == NO_F32 || dt == NO_BF16 || dt == NO_E4M3, NO_ERR_INVALID_ARG, "no_embed_fwd: unknown table type");
    NO_REQUIRE(dt_out == NO_F32 || dt_out == NO_BF16, NO_ERR_INVALID_ARG, "no_embed_fwd: outputs are NO_F32 or NO_BF16");
    NO_REQUIRE(n_rows >= 1 && dim >= 1 && n_ids_cap >= 0, NO_ERR_INVALID_ARG, "no_embed_fwd: bad sizes");
    NO_REQUIRE(dim <= NO_MAX_EMBED_DIM, NO_ERR_UNSUPPORTED, "no_embed_fwd: rows of more than %d values", NO_MAX_EMBED_DIM);
    NO_CHECK(check_rows("no_embed_fwd", "table", d_table, dt, n_rows, dim, table_stride_bytes));
    NO_CHECK(check_rows("no_embed_fwd", "out", d_out, dt_out, n_ids_cap, dim, out_stride_bytes));
    if (n_ids_cap == 0) return NO_OK;
    NO_REQUIRE(d_ids, NO_ERR_INVALID_ARG, "no_embed_fwd: ids are NULL");
    const RowsOf table = rows_of(d_table, table_stride_bytes), out = rows_of(d_out, out_stride_bytes);
#define NO_EMBED(T, O) launch_embed<T, O>(table, n_rows, dim, d_row_scale, d_ids, d_n_ids, n_ids_cap, scale, out, (hipStream_t)stream)
    if (dt_out == NO_F32) { if (dt == NO_F32) NO_EMBED(float, float); else if (dt == NO_BF16) NO_EMBED(bf16_t, float); else NO_EMBED(e4m3_t, float); }
    else { if (dt == NO_F32) NO_EMBED(float, bf16_t); else if (dt == NO_BF16) NO_EMBED(bf16_t, bf16_t); else NO_EMBED(e4m3_t, bf16_t); }
#undef NO_EMBED
    return launch_status("no_embed_fwd");
}

extern "C" size_t no_embed_ws_bytes(int32_t n_ids_cap, int32_t dim) {
    if (n_ids_cap < 0 || dim < 1 || dim > NO_MAX_EMBED_DIM) return 0;
    return EmbedPlan(n_ids_cap, dim).room(dim);
}

extern "C" int32_t no_embed_bwd(const void* d_grad_out, no_dtype dt, int64_t grad_stride_bytes, const int32_t* d_ids, const int32_t* d_n_ids,
                                int32_t n_ids_cap, float scale, int32_t accumulate, float* d_grad_table, int64_t n_rows, int32_t dim,
                                int64_t table_stride_bytes, void* d_ws, size_t ws_bytes, void* stream) {
    clear_error();
    const char* who = "no_embed_bwd";
    NO_REQUIRE(dt == NO_F32 || dt == NO_BF16, NO_ERR_INVALID_ARG, "%s: gradients are NO_F32 or NO_BF16", who);
    NO_REQUIRE(n_rows >= 1 && n_rows <= INT32_MAX && dim >= 1 && n_ids_cap >= 0, NO_ERR_INVALID_ARG, "%s: bad sizes", who);
    NO_REQUIRE(dim <= NO_MAX_EMBED_DIM, NO_ERR_UNSUPPORTED, "%s: rows of more than %d values", who, NO_MAX_EMBED_DIM);
    NO_CHECK(check_rows(who, "grad_out", d_grad_out, dt, n_ids_cap, dim, grad_stride_bytes));
    NO_CHECK(check_rows(who, "grad_table", d_grad_table, NO_F32, n_rows, dim, table_stride_bytes));
    NO_REQUIRE(d_ids || n_ids_cap == 0, NO_ERR_INVALID_ARG, "%s: ids are NULL", who);
    NO_REQUIRE(d_ws && (uintptr_t)d_ws % 16 == 0, NO_ERR_INVALID_ARG, "%s: the workspace is NULL or misaligned", who);
    const EmbedPlan plan(n_ids_cap, dim);
    NO_REQUIRE(ws_bytes >= plan.total, NO_ERR_CAPACITY, "%s: workspace too small", who);
    hipStream_t st = (hipStream_t)stream;
    char* ws = (char*)d_ws;
    uint32_t *keys = (uint32_t*)(ws + plan.keys), *pos = (uint32_t*)(ws + plan.pos);
    const EmbedSums a{keys, pos, d_n_ids, n_ids_cap, scale, accumulate != 0, rows_of(d_grad_out, grad_stride_bytes), rows_of(d_grad_table, table_stride_bytes), n_rows, dim,
                      plan.chunk, (float*)(ws + plan.parts)};
    if (embed_few(n_ids_cap, dim)) {
        if (n_ids_cap == 0 && accumulate) return NO_OK;
        if (dt == NO_F32) launch_few<float>(a, d_ids, st);
        else launch_few<bf16_t>(a, d_ids, st);
        return launch_status(who);
    }
    const unsigned tiles = (unsigned)plan.tiles;
    if (plan.merged) {
        uint32_t *k = (uint32_t*)(ws + plan.keys_tmp), *v = (uint32_t*)(ws + plan.pos_tmp), *rank = (uint32_t*)(ws + plan.rank);
        if (n_rows < (1 << 22)) hipLaunchKernelGGL(embed_tile_kernel<uint32_t>, dim3(tiles), dim3(1024), 0, st, d_ids, d_n_ids, n_ids_cap, (uint32_t)n_rows, k, v, rank);
        else hipLaunchKernelGGL(embed_tile_kernel<uint64_t>, dim3(tiles), dim3(1024), 0, st, d_ids, d_n_ids, n_ids_cap, (uint32_t)n_rows, k, v, rank);
        // about 512 blocks, two to a compute unit
        const unsigned groups = (tiles + 3) / 4, wanted = (512 + tiles - 1) / tiles, shares = wanted < groups ? wanted : groups;
        hipLaunchKernelGGL(embed_rank_kernel, dim3(tiles, shares), dim3(1024), 0, st, k, d_n_ids, n_ids_cap, (int32_t)shares, rank);
        hipLaunchKernelGGL(embed_place_kernel, dim3(tiles * (EMBED_TILE / 256)), dim3(256), 0, st, k, v, rank, d_n_ids, n_ids_cap, keys, pos);
    } else if (!plan.radix) {
        hipLaunchKernelGGL(embed_count_kernel, dim3((unsigned)ceil_div(n_ids_cap, 64)), dim3(1024), 0, st, d_ids, d_n_ids, n_ids_cap, keys, pos);
    } else {
        const int bits = ilog2_ceil((uint64_t)n_rows + 1), passes = radix_passes(bits), digit = radix_digit_bits(bits);
        const RadixPlan radix(n_ids_cap);
        uint32_t *k[2] = {keys, (uint32_t*)(ws + plan.keys_tmp)}, *v[2] = {pos, (uint32_t*)(ws + plan.pos_tmp)};
        int to = (passes & 1) ? 0 : 1;          // the last pass ends in the first pair of arrays
        for (int p = 0; p < passes; ++p, to ^= 1) {
            const int shift = p * digit, width = bits - shift < digit ? bits - shift : digit;
            if (p == 0) NO_CHECK(radix_pass(IdSource{d_ids, d_n_ids, n_ids_cap, (uint32_t)n_rows}, radix, shift, width, k[to], v[to], ws + plan.sort_ws, st));
            else NO_CHECK(radix_pass(PairArrays{k[to ^ 1], v[to ^ 1]}, radix, shift, width, k[to], v[to], ws + plan.sort_ws, st));
        }
    }
    if (dt == NO_F32) launch_sums<float>(a, plan.chunks, st);
    else launch_sums<bf16_t>(a, plan.chunks, st);
    const int64_t eights = ceil_div(plan.chunks - 1, 8);
    const dim3 grid((unsigned)(eights < 4096 ? eights : 4096), (unsigned)ceil_div(dim, 256));
    if (dim >= 4) hipLaunchKernelGGL(embed_join_kernel<false>, grid, dim3(512), 0, st, a, plan.chunks);
    else hipLaunchKernelGGL(embed_join_kernel<true>, grid, dim3(512), 0, st, a, plan.chunks);
    return launch_status(who);
}
