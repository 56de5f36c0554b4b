// no_embed_fwd / no_embed_bwd: rows of a table by id, scaled, and the gradient of the table.
#include "rows.hpp"
#include "radix.hpp"

namespace no {

// A group of lanes (a power of two, at most 64) copies a row in runs of W values, W such that the wider side moves 16 or 32 bytes a lane. The next
// row's id is requested before this row's values, so that a row costs one round trip, its scale beside it.
template <typename T, typename O, int W, int UNR>
__global__ void __launch_bounds__(256) embed_fwd_kernel(RowsOf table, int64_t n_rows, int32_t dim, const float* __restrict__ row_scale, const int32_t* __restrict__ ids,
                                                        const int32_t* d_n, int32_t cap, float scale, RowsOf out, int32_t units, int32_t g_log2) {
    const int32_t n = rows_here(d_n, cap), lane = lane_id(), g = 1 << g_log2, sub = lane >> g_log2, u0 = lane & (g - 1), rows = 64 >> g_log2;
    const int64_t wave = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 6, stride = (int64_t)gridDim.x * 4 * rows;
    int64_t r = wave * rows + sub;
    int32_t id = r < n ? ids[r] : -1;
    for (; r - sub < n; r += stride) {
        const int32_t next = r + stride < n ? ids[r + stride] : -1;
        const bool there = id >= 0 && id < n_rows;
        const float by = there ? (row_scale ? scale * row_scale[id] : scale) : 0.0f;
        const T* src = table.row<T>(there ? id : 0);
        for (int32_t ub = u0; ub < units && r < n; ub += g * UNR) {
            Run<T, W> v[UNR];
#pragma unroll
            for (int j = 0; j < UNR; ++j) {
                const int32_t c = (ub + j * g) * W;
                if (there && c < dim) v[j].load(src + c, dim - c, from_f32<T>(0.0f));
            }
#pragma unroll
            for (int j = 0; j < UNR; ++j) {
                const int32_t c = (ub + j * g) * W;
                if (c >= dim) break;
                float f[W];
                v[j].get(f);
#pragma unroll
                for (int w = 0; w < W; ++w) f[w] = there ? f[w] * by : 0.0f;
                Run<O, W> o;
                o.set(f);
                o.store(out.row<O>(r) + c, dim - c);
            }
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
    if (blocks > 2048) blocks = 2048;
    if (units > 64) hipLaunchKernelGGL((embed_fwd_kernel<T, O, W, 4>), dim3((unsigned)blocks), dim3(256), 0, st, table, n_rows, dim, row_scale, ids, d_n, cap, scale, out, units, g_log2);
    else hipLaunchKernelGGL((embed_fwd_kernel<T, O, W, 1>), dim3((unsigned)blocks), dim3(256), 0, st, table, n_rows, dim, row_scale, ids, d_n, cap, scale, out, units, g_log2);
}

// ------------------------------------------------------------------------------------------------------- gradient
//
// G[v] = scale * sum over the positions i with ids[i] == v of g[i]. The positions are ordered by id (stable, so by position within an id); then the
// ordered list is cut into chunks of 8 or 32 positions whatever the ids are, and a lane group walks a chunk with the sum of the id at hand
// in registers: an id that is named a thousand times costs what a thousand rare ones do. Sums of ids that lie inside a chunk go
// straight to the table; those that reach over a chunk's border go to the workspace and are added up, in chunk order, by a second launch. Rows that no
// id names are found by a search in the ordered ids and cleared beside the sums. No atomics: the same ids give the same bits.

constexpr int EMBED_TILE = 4096;                    // positions that a block orders in LDS
constexpr int32_t EMBED_MERGE_MOST = 131072;        // positions that are ordered by tiles and ranks; more go through the radix sort

struct EmbedPlan {      // the workspace, cut up
    int64_t n, tiles, chunks;
    int32_t chunk;
    bool merged, radix;
    size_t keys, pos, keys_tmp, pos_tmp, rank, sort_ws, parts, total;
    EmbedPlan(int32_t n_, int32_t dim) : n(n_), tiles(ceil_div(n_, EMBED_TILE)), chunk(n_ <= 16384 ? 8 : 32) {
        chunks = ceil_div(n, chunk);
        radix = n > EMBED_MERGE_MOST;
        merged = !radix && tiles > 1;
        const size_t list = (size_t)(tiles ? tiles : 1) * EMBED_TILE * 4;
        keys = 0;
        pos = keys + list;
        keys_tmp = pos + list;
        pos_tmp = keys_tmp + (merged || radix ? list : 0);
        rank = pos_tmp + (merged || radix ? list : 0);
        sort_ws = rank + (merged ? list : 0);
        parts = sort_ws + (radix ? (size_t)ceil_div((int64_t)radix_ws_bytes(n), 16) * 16 : 0);
        total = parts + (size_t)chunks * 2 * (size_t)dim * 4 + 16;
    }
};

// A tile's positions in order, in LDS: a bitonic network over (id, position in the tile), four elements a thread, so that distances of 1 and 2 stay in a
// thread, 4 to 128 in a wavefront, and only the ten steps of 256 and more go through LDS. K: 32 bits where the ids leave 12 of them, else 64. Ids
// outside the table, and positions that are not there, come last.
template <typename K>
__global__ void __launch_bounds__(1024) embed_tile_kernel(const int32_t* __restrict__ ids, const int32_t* d_n, int32_t cap, uint32_t n_rows, uint32_t* keys, uint32_t* pos,
                                                          uint32_t* rank) {
    __shared__ K held[EMBED_TILE];
    const int32_t n = rows_here(d_n, cap), base = (int32_t)blockIdx.x * EMBED_TILE, t = threadIdx.x, here = min(EMBED_TILE, n - base);
    if (here <= 0) return;
    K x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int32_t i = 4 * t + e;
        const uint32_t key = i < here ? min((uint32_t)ids[base + i], n_rows) : 0u;
        x[e] = i < here ? ((K)key << 12 | (K)i) : ~(K)0;
    }
    const int32_t m = here <= 4 ? 4 : 1 << (32 - __builtin_clz((uint32_t)here - 1));       // elements behind it are all padding
    auto order = [](K& lo, K& hi, bool up) {
        const K a = lo < hi ? lo : hi, b = lo < hi ? hi : lo;
        lo = up ? a : b;
        hi = up ? b : a;
    };
    for (int k = 2; k <= m; k <<= 1) {
        for (int j = k >> 1; j >= 256; j >>= 1) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 4; ++e) held[4 * t + e] = x[e];
            __syncthreads();
            const bool keep_small = ((4 * t & k) == 0) == ((4 * t & j) == 0);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const K o = held[(4 * t ^ j) + e];
                x[e] = (o < x[e]) == keep_small ? o : x[e];
            }
        }
        for (int j = min(k >> 1, 128); j >= 4; j >>= 1) {
            const bool keep_small = ((4 * t & k) == 0) == ((4 * t & j) == 0);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                K o;
                if constexpr (sizeof(K) == 4) o = (K)__shfl_xor((int)x[e], j >> 2, 64);
                else o = (K)__shfl_xor((unsigned long long)x[e], j >> 2, 64);
                x[e] = (o < x[e]) == keep_small ? o : x[e];
            }
        }
        const bool up = (4 * t & k) == 0;
        if (k >= 4) {
            order(x[0], x[2], up);
            order(x[1], x[3], up);
            order(x[0], x[1], up);
            order(x[2], x[3], up);
        } else {                                    // pairs, in turn up and down
            order(x[0], x[1], true);
            order(x[2], x[3], false);
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int32_t i = 4 * t + e;
        const bool there = i < here;
        keys[base + i] = there ? (uint32_t)(x[e] >> 12) : ~0u;
        pos[base + i] = there ? (uint32_t)(x[e] & 4095) + (uint32_t)base : 0u;
        if (rank) rank[base + i] = 0;
    }
}

// An element's place among all tiles is the number of smaller ones in each, where equal ids count in the tiles left of its own. A block takes 1024 elements of a
// tile and a share of the tiles to search; the shares add up in whole numbers, in any order.
__global__ void __launch_bounds__(1024) embed_rank_kernel(const uint32_t* __restrict__ keys, const int32_t* d_n, int32_t cap, int32_t shares, uint32_t* rank) {
    __shared__ __attribute__((aligned(16))) uint32_t held[EMBED_TILE];
    const int32_t n = rows_here(d_n, cap), i = (int32_t)blockIdx.x * 1024 + (int32_t)threadIdx.x, own = (int32_t)blockIdx.x / (EMBED_TILE / 1024);
    if (own * EMBED_TILE >= n) return;
    const int32_t tiles = (n + EMBED_TILE - 1) / EMBED_TILE;
    const uint32_t key = keys[i];
    uint32_t before = 0;
    for (int32_t o = blockIdx.y; o < tiles; o += shares) {
        if (o == own) {
            before += (uint32_t)(i - own * EMBED_TILE);
            continue;
        }
        __syncthreads();
        reinterpret_cast<uint4*>(held)[threadIdx.x] = reinterpret_cast<const uint4*>(keys + o * EMBED_TILE)[threadIdx.x];
        __syncthreads();
        // elements below `to`, or up to it in earlier tiles (key + 1 does not wrap: an id is at most n_rows; what is not there is not stored)
        const uint32_t to = o < own ? key + 1 : key;
        uint32_t at = 0;
#pragma unroll
        for (int step = EMBED_TILE / 2; step > 0; step >>= 1) at += held[at + step - 1] < to ? step : 0;
        before += at + (held[at] < to);
    }
    if (key != ~0u) atomicAdd(&rank[i], before);
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

template <typename T, int W, bool ADD>
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
        uint32_t empty = (uint32_t)__ballot(v < a.n_rows && !(lo < n && (int64_t)a.keys[lo] == v)) & 0xffffu;
        Run<float, 4> zero;
        const float z[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        zero.set(z);
        while (empty) {
            const int32_t at = __builtin_ctz(empty);
            empty &= empty - 1;
            float* row = a.table.row<float>(v0 + at);
            for (int32_t c = lane * 4; c < a.dim; c += 256) zero.store(row + c, a.dim - c);
        }
    }
    const int32_t groups = 64 >> g_log2, u = lane & ((1 << g_log2) - 1);
    const int64_t item = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * groups + (lane >> g_log2);
    const int64_t chunk = item / col_tiles;
    const int32_t col = ((int32_t)(item % col_tiles) * 64 + u) * W, width = a.dim - col;
    const int64_t e0 = chunk * a.chunk;
    if (chunk >= chunks || e0 >= n || width <= 0) return;
    const int32_t len = (int32_t)min((int64_t)a.chunk, n - e0);
    const uint32_t before = chunk ? a.keys[e0 - 1] : ~0u, after = e0 + len < n ? a.keys[e0 + len] : ~0u;
    float* const parts = a.parts + chunk * 2 * a.dim + col;
    const uint32_t n_rows = (uint32_t)a.n_rows;     // (fewer than 2^31)
    float acc[W];
#pragma unroll
    for (int w = 0; w < W; ++w) acc[w] = 0.0f;
    int32_t start = 0;
    constexpr int UNR = ADD ? 4 : 8;                // rows requested before the first is added
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
            r[k].load(a.grad.row<T>(p[k]) + col, width, from_f32<T>(0.0f));
            // the row that a run's sum is added to, requested with the run's last gradient
            if (ADD && key[k + 1] != key[k]) old[ADD ? k : 0].load(a.table.row<float>(key[k]) + col, width, 0.0f);
        }
#pragma unroll
        for (int k = 0; k < UNR; ++k) {
            if (key[k] >= n_rows) continue;
            float f[W];
            r[k].get(f);
#pragma unroll
            for (int w = 0; w < W; ++w) acc[w] += f[w];
            if (key[k + 1] == key[k]) continue;     // (an id at the chunk's end goes on in the next, or does not: its sum is stored either way)
            Run<float, W> out;
            const bool last = e + k + 1 == len;
            if (start == 0 && key[k] == before) { out.set(acc); out.store(parts, width); }
            else if (last && key[k] == after) { out.set(acc); out.store(parts + a.dim, width); }
            else {
                if constexpr (ADD) old[ADD ? k : 0].get(f);
#pragma unroll
                for (int w = 0; w < W; ++w) f[w] = ADD ? f[w] + a.scale * acc[w] : a.scale * acc[w];
                out.set(f);
                out.store(a.table.row<float>(key[k]) + col, width);
            }
            start = e + k + 1;
#pragma unroll
            for (int w = 0; w < W; ++w) acc[w] = 0.0f;
        }
    }
}

// Adds up the sums that reach over borders: the chunk where such an id begins owns it. A block's eight wavefronts share the later chunks' parts, and look for their
// number 64 chunks at a time.
__global__ void __launch_bounds__(512) embed_join_kernel(EmbedSums a, int64_t chunks) {
    __shared__ float share[8][64][4];
    const int32_t n = rows_here(a.d_n, a.cap), lane = lane_id(), wave = (int32_t)(threadIdx.x >> 6), ch = a.chunk;
    const int32_t col = ((int32_t)blockIdx.y * 64 + lane) * 4, width = a.dim - col;
    const int64_t here = min(chunks, ceil_div(n, ch));
    for (int64_t c = blockIdx.x; c + 1 < here; c += gridDim.x) {
        const uint32_t first = a.keys[c * ch], key = a.keys[(c + 1) * ch - 1], next = a.keys[(c + 1) * ch], prior = c > 0 ? a.keys[c * ch - 1] : ~0u;
        if ((int64_t)key >= a.n_rows || next != key || (first == key && prior == key)) continue;
        int64_t end = c + 2;                    // the first chunk that does not begin with this id
        for (;;) {
            const uint64_t same = __ballot(end + lane < here && a.keys[min(end + lane, here - 1) * ch] == key);
            end += same == ~0ull ? 64 : __builtin_ctzll(~same);
            if (same != ~0ull) break;
        }
        const int64_t parts = end - c, each = ceil_div(parts, 8), p0 = min(parts, wave * each), p1 = min(parts, p0 + each);
        float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (width > 0) {
#pragma unroll 8
            for (int64_t p = p0; p < p1; ++p) {
                Run<float, 4> r;
                r.load(a.parts + ((c + p) * 2 + (p == 0)) * a.dim + col, width, 0.0f);
                float f[4];
                r.get(f);
#pragma unroll
                for (int w = 0; w < 4; ++w) acc[w] += f[w];
            }
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 4; ++w) share[wave][lane][w] = acc[w];
        __syncthreads();
        if (wave == 0 && width > 0) {
            float* to = a.table.row<float>(key) + col;
            Run<float, 4> out;
            float f[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            if (a.accumulate) { out.load(to, width, 0.0f); out.get(f); }
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                float sum = share[0][lane][w];
#pragma unroll
                for (int o = 1; o < 8; ++o) sum += share[o][lane][w];
                f[w] += a.scale * sum;
            }
            out.set(f);
            out.store(to, width);
        }
    }
}

template <typename T>
static void launch_sums(const EmbedSums& a, int64_t chunks, hipStream_t st) {
    constexpr int W = 16 / (int)sizeof(T);
    const int32_t units = (int32_t)ceil_div(a.dim, W), col_tiles = (int32_t)ceil_div(units, 64);
    int g_log2 = 0;
    while ((1 << g_log2) < units && g_log2 < 6) ++g_log2;
    const int64_t sum_blocks = ceil_div(ceil_div(chunks * col_tiles, 64 >> g_log2), 4), zero_rows = ceil_div(a.n_rows, 64),
                  zero_blocks = a.accumulate ? 0 : zero_rows < (1 << 20) ? zero_rows : 1 << 20;
    const dim3 grid((unsigned)(sum_blocks + zero_blocks));
    if (a.accumulate) { if (sum_blocks) hipLaunchKernelGGL((embed_sums_kernel<T, W, true>), grid, dim3(256), 0, st, a, chunks, g_log2, col_tiles, (uint32_t)sum_blocks); }
    else hipLaunchKernelGGL((embed_sums_kernel<T, W, false>), grid, dim3(256), 0, st, a, chunks, g_log2, col_tiles, (uint32_t)sum_blocks);
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
    return EmbedPlan(n_ids_cap, dim).total;
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
    if (n_ids_cap > 0) {
        if (!plan.radix) {
            uint32_t *k = plan.merged ? (uint32_t*)(ws + plan.keys_tmp) : keys, *v = plan.merged ? (uint32_t*)(ws + plan.pos_tmp) : pos,
                     *rank = plan.merged ? (uint32_t*)(ws + plan.rank) : nullptr;
            const unsigned tiles = (unsigned)plan.tiles;
            if (n_rows < (1 << 20)) hipLaunchKernelGGL(embed_tile_kernel<uint32_t>, dim3(tiles), dim3(1024), 0, st, d_ids, d_n_ids, n_ids_cap, (uint32_t)n_rows, k, v, rank);
            else hipLaunchKernelGGL(embed_tile_kernel<uint64_t>, dim3(tiles), dim3(1024), 0, st, d_ids, d_n_ids, n_ids_cap, (uint32_t)n_rows, k, v, rank);
            if (plan.merged) {
                const unsigned shares = tiles >= 64 ? 2 : tiles >= 32 ? 4 : tiles < 8 ? tiles : 8;
                hipLaunchKernelGGL(embed_rank_kernel, dim3(tiles * (EMBED_TILE / 1024), shares), dim3(1024), 0, st, k, d_n_ids, n_ids_cap, (int32_t)shares, rank);
                hipLaunchKernelGGL(embed_place_kernel, dim3(tiles * (EMBED_TILE / 256)), dim3(256), 0, st, k, v, rank, d_n_ids, n_ids_cap, keys, pos);
            }
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
    }
    const EmbedSums a{keys, pos, d_n_ids, n_ids_cap, scale, accumulate != 0, rows_of(d_grad_out, grad_stride_bytes), rows_of(d_grad_table, table_stride_bytes), n_rows, dim,
                      plan.chunk, (float*)(ws + plan.parts)};
    if (dt == NO_F32) launch_sums<float>(a, plan.chunks, st);
    else launch_sums<bf16_t>(a, plan.chunks, st);
    if (plan.chunks > 1)
        hipLaunchKernelGGL(embed_join_kernel, dim3((unsigned)(plan.chunks - 1 < 1024 ? plan.chunks - 1 : 1024), (unsigned)ceil_div(dim, 256)), dim3(512), 0, st, a, plan.chunks);
    return launch_status(who);
}
