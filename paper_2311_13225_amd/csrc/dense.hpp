// Matrix products of 16-bit operands (bf16, or fp16 pieces of fp32 values) on the matrix cores, with fp32 sums: the dense layer (linear.hip) and the orthogonalised
// update (orthogonalise.hip). C[m, n] = sum over the pairs (p, q) of planes of sum over k of A_p(m, k) B_q(k, n); an operand of one plane is the matrix itself, one of several holds
// the pieces of wider values. An operand lies ALONG the reduction (k contiguous in memory) or across it.
#pragma once
#include "rows.hpp"

namespace no {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

// Addresses and pitches of whole 16 bytes. ALONG: `extent` rows of k values, zeros from K up to the next multiple of 8; across: rows k of `extent` values, a multiple of 8.
struct DenseOperand {
    const char* p;
    int64_t pitch, plane, matrix;       // bytes from row to row, plane to plane, matrix to matrix
    int32_t extent;
};

struct DenseArgs {
    DenseOperand a, b;
    int32_t M, N, K;
    const int32_t *d_M, *d_K;           // device scalars that limit M or K (NULL: none)
    uint32_t pairs_a, pairs_b;          // planes of the pairs, four bits each, in order
    int32_t n_pairs, splits, tiles_m, tiles_n;
};

static inline size_t round_256(size_t b) { return (b + 255) / 256 * 256; }
static inline int64_t wide_of(int64_t dim) { return (dim + 7) / 8 * 8; }       // values of a row of whole 16 bytes

constexpr int DENSE_BK = 64;            // reduction indices a step
constexpr uint32_t DENSE_NOWHERE = 0x80000000u;      // past every buffer's range: reads as 0

// One operand's tile of R rows (or columns) and 64 reduction indices in LDS, loaded by T threads in requests of 16 bytes that go straight to LDS. A request's 64 lanes fill 1 KB in lane
// order, so the order of the units in LDS is made by which unit a lane asks for: ALONG, unit u of row r stands at place u ^ (r & 7) of its 128 bytes; across, the 32
// bytes of 16 columns of row k stand at place c ^ f(k), f(k) = (k & 3) | (k >> 3 & 1) << 2. Then the 64 lanes of a fragment's read meet every bank equally often.
template <bool ALONG, int R, int T>
struct DenseTile {
    static constexpr int BYTES = R * DENSE_BK * 2, REQ = BYTES / (16 * T), PER_ROW = ALONG ? 8 : R / 8;
    static_assert(BYTES % (16 * T) == 0 && T % PER_ROW == 0 && (ALONG || R >= 64), "whole requests");
    uint32_t off[REQ];
    int32_t k_first;                    // the reduction index that this thread's first request begins with
    const char* base;                   // the tile's origin in the matrix
    int64_t step;                       // bytes from one step to the next
    __device__ __forceinline__ static int mix(int k) { return ((k & 3) | (k >> 3 & 1) << 2) & (R / 16 - 1); }
    __device__ __forceinline__ void open(const DenseOperand& o, int64_t matrix, int32_t first) {
        const int tid = (int)threadIdx.x;
#pragma unroll
        for (int i = 0; i < REQ; ++i) {
            const int c = i * T + tid, line = c / PER_ROW, place = c % PER_ROW;
            if (ALONG) {
                const int unit = place ^ (line & 7);
                off[i] = first + line < o.extent ? (uint32_t)line * (uint32_t)o.pitch + (uint32_t)unit * 16u : DENSE_NOWHERE;
                if (i == 0) k_first = unit * 8;
            } else {
                const int unit = ((place >> 1) ^ mix(line)) << 1 | (place & 1);
                off[i] = first + unit * 8 < o.extent ? (uint32_t)line * (uint32_t)o.pitch + (uint32_t)unit * 16u : DENSE_NOWHERE;
                if (i == 0) k_first = line;
            }
        }
        base = o.p + matrix * o.matrix + (ALONG ? (int64_t)first * o.pitch : (int64_t)first * 2);
        step = ALONG ? DENSE_BK * 2 : DENSE_BK * o.pitch;
    }
    // what is there from reduction index k0 on of a plane of `K` of them, into `to`
    __device__ __forceinline__ void request(const DenseOperand& o, int plane, int32_t k0, int32_t K, char* to) const {
        const char* from = base + plane * o.plane + (int64_t)(k0 / DENSE_BK) * step;
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)from, 0, 0x7fffffff, 0x00020000);
        const int wave = (int)threadIdx.x >> 6;
        const bool whole = k0 + DENSE_BK <= K;
#pragma unroll
        for (int i = 0; i < REQ; ++i) {
            const int k = k0 + k_first + (ALONG ? 0 : i * (T / PER_ROW));
            const uint32_t at = whole || k < K ? off[i] : DENSE_NOWHERE;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)(to + (i * T + wave * 64) * 16), 16, at, 0, 0, 0);
        }
    }
    // The fragment of 16 rows (columns) from 16 q on, reduction indices [32 h, 32 h + 32): lane l has row l % 16 and indices 8 (l / 16) + [0, 8).
    __device__ __forceinline__ static s16x8 fragment(const char* from, int q, int h) {
        const int l = (int)threadIdx.x & 63, g = l >> 4, j = l & 15;
        if constexpr (ALONG) return *reinterpret_cast<const s16x8*>(from + q * 2048 + j * 128 + (((h * 4 + g) ^ (j & 7)) << 4));
        else {
            // four rows of 16 columns at a time, turned on the way: lane j of 16 asks for 4 values of row j / 4 and gets column j of the four rows
            typedef __attribute__((address_space(3))) s16x4* lds;
            const char* p = from + (h * 32 + g * 8 + (j >> 2)) * (R * 2) + ((q ^ mix(g * 8 + (j >> 2))) << 5) + (j & 3) * 8;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)p), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(p + 4 * R * 2));
            return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
};

template <typename H> __device__ __forceinline__ f32x4 dense_mfma(s16x8 a, s16x8 b, f32x4 c);
template <> __device__ __forceinline__ f32x4 dense_mfma<__bf16>(s16x8 a, s16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ f32x4 dense_mfma<_Float16>(s16x8 a, s16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// A block's place: tiles are dealt to the dies in runs, and walked in bands of `band` tile rows, so that a die's blocks share rows and columns in its L2.
// HALF: the tiles on and above the diagonal of a square alone.
static inline unsigned dense_grid(int64_t tiles_m, int64_t tiles_n, bool half) { return (unsigned)(ceil_div(half ? tiles_m * (tiles_m + 1) / 2 : tiles_m * tiles_n, 8) * 8); }
template <bool HALF>
__device__ __forceinline__ bool dense_place(const DenseArgs& g, int band, int& tm, int& tn) {
    const int total = HALF ? g.tiles_m * (g.tiles_m + 1) / 2 : g.tiles_m * g.tiles_n, padded = (int)gridDim.x;
    const int id = ((int)blockIdx.x % 8) * (padded / 8) + (int)blockIdx.x / 8;
    if (id >= total) return false;
    if (HALF) {         // column tn begins behind tn (tn + 1) / 2 tiles (fewer than 2^24 of them, so the root is off by one at most)
        tn = (int)((sqrtf(8.0f * (float)id + 1.0f) - 1.0f) * 0.5f);
        tn += (tn + 1) * (tn + 2) / 2 <= id ? 1 : 0;
        tn -= tn * (tn + 1) / 2 > id ? 1 : 0;
        tm = id - tn * (tn + 1) / 2;
        return true;
    }
    const int per = band * g.tiles_n, b = id / per, rest = id - b * per, rows = min(band, g.tiles_m - b * band);
    tm = b * band + rest % rows;
    tn = rest / rows;
    return true;
}

// C's tile of BM x BN by WM x WN wavefronts, each BM/WM x BN/WN of it in fragments of 16 x 16; two LDS copies, the next step's on its way while this one's is multiplied. The epilogue
// gets eight consecutive columns of a row: E::put(epilogue's arguments, product's, m, n, columns there, sums).
template <typename H, bool AL, bool BL, int BM, int BN, int WM, int WN, typename E>
__global__ void __launch_bounds__(64 * WM * WN) dense_kernel(const DenseArgs g, const typename E::Args e) {
    constexpr int T = 64 * WM * WN, I = BM / WM / 16, J = BN / WN / 16;
    typedef DenseTile<AL, BM, T> TA;
    typedef DenseTile<BL, BN, T> TB;
    __shared__ __attribute__((aligned(1024))) char lds[2 * (TA::BYTES + TB::BYTES)];
    int tm, tn;
    if (!dense_place<E::MIRROR>(g, 8, tm, tn)) return;
    const int32_t M = rows_here(g.d_M, g.M), K = rows_here(g.d_K, g.K), m0 = tm * BM, n0 = tn * BN;
    if (m0 >= M) return;
    const int wave = (int)threadIdx.x >> 6, wm = wave / WN, wn = wave % WN, l = (int)threadIdx.x & 63;
    TA ta;
    TB tb;
    DenseOperand oa = g.a, ob = g.b;
    if (AL) oa.extent = min(oa.extent, M);
    ta.open(oa, blockIdx.z, m0);
    tb.open(ob, blockIdx.z, n0);
    const int32_t per_pair = (K + DENSE_BK - 1) / DENSE_BK, steps = per_pair * g.n_pairs;
    const int32_t first = (int32_t)((int64_t)steps * blockIdx.y / g.splits), last = (int32_t)((int64_t)steps * (blockIdx.y + 1) / g.splits);
    const int32_t KA = AL ? (K + 7) & ~7 : K, KB = BL ? (K + 7) & ~7 : K;
    int pair = per_pair ? first / per_pair : 0, in_pair = first - pair * per_pair;
    auto request = [&](char* to) {
        ta.request(oa, g.pairs_a >> (4 * pair) & 15, in_pair * DENSE_BK, KA, to);
        tb.request(ob, g.pairs_b >> (4 * pair) & 15, in_pair * DENSE_BK, KB, to + TA::BYTES);
        if (++in_pair == per_pair) { in_pair = 0; ++pair; }
    };
    f32x4 acc[I][J];
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    char* now = lds;
    char* then = lds + TA::BYTES + TB::BYTES;
    if (first < last) request(now);
    for (int32_t s = first; s < last; ++s) {
        __builtin_amdgcn_s_waitcnt(0x0f70);        // vmcnt(0): this step's operands have arrived
        __syncthreads();
        if (s + 1 < last) request(then);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            s16x8 a[I], b[J];
#pragma unroll
            for (int j = 0; j < J; ++j) b[j] = TB::fragment(now + TA::BYTES, wn * J + j, h);
#pragma unroll
            for (int i = 0; i < I; ++i) a[i] = TA::fragment(now, wm * I + i, h);
#pragma unroll
            for (int i = 0; i < I; ++i)
#pragma unroll
                for (int j = 0; j < J; ++j) acc[i][j] = dense_mfma<H>(b[j], a[i], acc[i][j]);
        }
        char* t = now; now = then; then = t;
    }
    // The sums go through LDS, 32 rows of a wavefront at a time, so that eight consecutive columns of a row meet in a lane and the lanes beside it go on along the row.
    constexpr int COLS = BN / WN, PITCH = COLS + 4, LANES = COLS / 8, RI = I < 2 ? I : 2, ROWS = RI * 16, PASS = 64 / LANES;
    static_assert(WM * WN * ROWS * PITCH * 4 <= (int)sizeof(lds) && I % RI == 0 && ROWS % PASS == 0, "room for a wavefront's rows");
    __syncthreads();
    float* mine = reinterpret_cast<float*>(lds) + wave * ROWS * PITCH;
#pragma unroll
    for (int i0 = 0; i0 < I; i0 += RI) {
        Team<64, T>::sync();
#pragma unroll
        for (int i = 0; i < RI; ++i)
#pragma unroll
            for (int j = 0; j < J; ++j) *reinterpret_cast<f32x4*>(mine + (i * 16 + (l & 15)) * PITCH + j * 16 + (l >> 4) * 4) = acc[i0 + i][j];
        Team<64, T>::sync();
        const int32_t mw = m0 + (wm * I + i0) * 16, nw = n0 + wn * COLS;
#pragma unroll 1
        for (int r = l / LANES; r < ROWS; r += PASS) {
            const int32_t m = mw + r, n = nw + l % LANES * 8;
            if (m >= M || n >= g.N) continue;
            float v[8];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const f32x4 x = *reinterpret_cast<const f32x4*>(mine + r * PITCH + l % LANES * 8 + q * 4);
#pragma unroll
                for (int w = 0; w < 4; ++w) v[4 * q + w] = x[w];
            }
            E::put(e, g, m, n, min(8, g.N - n), v);
        }
        if constexpr (E::MIRROR) {          // the same values as C[n, m], eight consecutive m a lane
            if (tm == tn) continue;
#pragma unroll 1
            for (int c = l / (ROWS / 8); c < COLS; c += 64 / (ROWS / 8)) {
                const int32_t n = nw + c, m = mw + l % (ROWS / 8) * 8;
                if (m >= M || n >= g.N) continue;
                float v[8];
#pragma unroll
                for (int w = 0; w < 8; ++w) v[w] = mine[(l % (ROWS / 8) * 8 + w) * PITCH + c];
                E::mirror(e, g, n, m, min(8, M - m), v);
            }
        }
    }
}

}  // namespace no
