// Matrix products of 16-bit operands (bf16, or fp16 pieces of fp32 values) on the matrix cores, with fp32 sums: the dense layer (linear.hip) and the orthogonalised
// update (orthogonalise.hip). C[m, n] = sum over k of A(m, k) B(k, n), where a value is one 16-bit piece, or the sum of P of them, P = 2 or 3, whose products are taken but for the smallest. An operand lies ALONG the reduction (k contiguous in memory) or across it.
#pragma once
#include "rows.hpp"

namespace no {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

// Addresses and pitches of whole 16 bytes. ALONG: `extent` rows of k values, zeros from K up to the next multiple of 8; across: rows k of `extent` values, a multiple of 8.
// The pieces of a row lie behind each other, `plane` bytes apart.
struct DenseOperand {
    const char* p;
    int64_t pitch, matrix;              // bytes from row to row, matrix to matrix
    int32_t plane, extent;
};

struct DenseArgs {
    DenseOperand a, b;
    int32_t M, N, K;
    const int32_t *d_M, *d_K;           // device scalars that limit M or K (NULL: none)
    int32_t splits, tiles_m, tiles_n;
};

static inline size_t round_256(size_t b) { return (b + 255) / 256 * 256; }
static inline int64_t wide_of(int64_t dim) { return (dim + 7) / 8 * 8; }       // values of a row of whole 16 bytes

// A step takes slabs of 32 reduction indices: two of a matrix of one piece, else one of each piece.
constexpr int dense_slabs(int P) { return P == 1 ? 2 : P; }
constexpr int dense_bk(int P) { return P == 1 ? 64 : 32; }
constexpr uint32_t DENSE_NOWHERE = 0x80000000u;      // past every buffer's range: reads as 0

// One operand's tile of R rows (or columns) and a step's slabs in LDS, loaded by T threads in requests of 16 bytes that go straight to LDS. A request's 64 lanes fill 1 KB in lane
// order, so the order of the units in LDS is made by which unit a lane asks for: ALONG, unit u of row r stands at place u ^ (r & 7) of its 128 bytes (three pieces: at
// u ^ (r >> 2 & 3) of its 192); across, the 32 bytes of 16 columns of line k stand at place c ^ f(k), f(k) = (k & 3) | (k >> 3 & 1) << 2. Then the 64 lanes of a fragment's read meet every
// bank equally often.
template <int P, bool ALONG, int R, int T>
struct DenseTile {
    static constexpr int SLABS = dense_slabs(P), BK = dense_bk(P), PER_ROW = ALONG ? SLABS * 4 : R / 8, BYTES = R * SLABS * 64, REQ = BYTES / (16 * T);
    static_assert(BYTES % (16 * T) == 0 && (ALONG || (R >= 64 && T % PER_ROW == 0)), "whole requests");
    uint32_t off[REQ];
    const char* base;                   // the tile's origin in the matrix
    int64_t step;                       // bytes from one step to the next
    __device__ __forceinline__ static int mix(int k) { return ((k & 3) | (k >> 3 & 1) << 2) & (R / 16 - 1); }
    // what request i of this thread asks for: line of the tile, unit of the line
    __device__ __forceinline__ static void which(int i, int& line, int& unit) {
        const int c = i * T + (int)threadIdx.x, place = c % PER_ROW;
        line = c / PER_ROW;
        unit = !ALONG ? ((place >> 1) ^ mix(line)) << 1 | (place & 1) : P == 3 ? place ^ (line >> 2 & 3) : place ^ (line & 7);
    }
    __device__ __forceinline__ void open(const DenseOperand& o, int64_t matrix, int32_t first) {
#pragma unroll
        for (int i = 0; i < REQ; ++i) {
            int line, unit;
            which(i, line, unit);
            if (ALONG) off[i] = first + line < o.extent ? (uint32_t)line * (uint32_t)o.pitch + (uint32_t)(P == 1 ? unit * 16 : (unit >> 2) * o.plane + (unit & 3) * 16) : DENSE_NOWHERE;
            else off[i] = first + unit * 8 < o.extent ? (uint32_t)(P == 1 ? line : line & 31) * (uint32_t)o.pitch + (uint32_t)((P == 1 ? 0 : (line >> 5) * o.plane) + unit * 16) : DENSE_NOWHERE;
        }
        base = o.p + matrix * o.matrix + (ALONG ? (int64_t)first * o.pitch : (int64_t)first * 2);
        step = ALONG ? BK * 2 : BK * o.pitch;
    }
    // Request i alone, by hand: the compiler takes a request for a write of LDS that every later read of LDS has to wait for, and cannot know that the two go to different copies. What it
    // fills is waited for in dense_meet(). Nothing is masked here: cut() comes before the first step that is not whole.
    __device__ __forceinline__ i32x4 source(int32_t s) const {
        const uint64_t at = (uint64_t)(base + (int64_t)s * step);
        return i32x4{(int)(uint32_t)at, (int)(uint32_t)(at >> 32), 0x7fffffff, 0x00020000};
    }
    __device__ __forceinline__ void request_one(int i, i32x4 rsrc, uint32_t to) const {
        asm volatile("s_add_u32 m0, %2, %3\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" : : "v"(off[i]), "s"(rsrc), "s"(to), "i"(i * T * 16) : "memory", "scc");
    }
    // From here on only the first `left` reduction indices of a step are asked for.
    __device__ __forceinline__ void cut(int32_t left) {
#pragma unroll
        for (int i = 0; i < REQ; ++i) {
            int line, unit;
            which(i, line, unit);
            const int k = ALONG ? (P == 1 ? unit : unit & 3) * 8 : P == 1 ? line : line & 31;
            if (k >= left) off[i] = DENSE_NOWHERE;
        }
    }
    // The fragment of 16 rows (columns) from 16 q on, slab h: lane l has row l % 16 and indices 8 (l / 16) + [0, 8).
    __device__ __forceinline__ static s16x8 fragment(const char* from, int q, int h) {
        const int l = (int)threadIdx.x & 63, g = l >> 4, j = l & 15;
        if constexpr (ALONG) return *reinterpret_cast<const s16x8*>(from + q * 16 * (SLABS * 64) + j * (SLABS * 64) + (P == 3 ? (h * 4 + (g ^ (j >> 2))) << 4 : ((h * 4 + g) ^ (j & 7)) << 4));
        else {
            // four lines of 16 columns at a time, turned on the way: lane j of 16 asks for 4 values of line j / 4 and gets column j of the four lines
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
template <typename H, int I, int J>
__device__ __forceinline__ void dense_multiply(f32x4 (&acc)[I][J], const s16x8 (&a)[I], const s16x8 (&b)[J]) {
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j) acc[i][j] = dense_mfma<H>(b[j], a[i], acc[i][j]);
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
        tn = __builtin_amdgcn_readfirstlane(tn);
        tm = id - tn * (tn + 1) / 2;
        return true;
    }
    const int per = band * g.tiles_n, b = id / per, rest = id - b * per, rows = min(band, g.tiles_m - b * band);
    tm = b * band + rest % rows;
    tn = rest / rows;
    return true;
}

// The sums of a block's tile to the epilogue: through LDS, 32 rows of a wavefront at a time, so that eight consecutive columns of a row meet in a lane and the lanes beside it go on along
// the row: E::put(epilogue's arguments, product's, m, n, columns there, sums).
template <int BM, int BN, int WM, int WN, typename E, int I, int J>
__device__ __forceinline__ void dense_finish(const DenseArgs& g, const typename E::Args& e, int tm, int tn, int32_t M, f32x4 (&acc)[I][J], char* lds) {
    constexpr int T = 64 * WM * WN, COLS = BN / WN, PITCH = COLS + 4, LANES = COLS / 8, RI = I < 2 ? I : 2, ROWS = RI * 16, PASS = 64 / LANES;
    static_assert(I % RI == 0 && ROWS % PASS == 0, "whole passes");
    const int wave = (int)threadIdx.x >> 6, wm = wave / WN, wn = wave % WN, l = (int)threadIdx.x & 63;
    const int32_t m0 = tm * BM, n0 = tn * BN;
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

constexpr int dense_shared(int P, int BM, int BN, int WM, int WN, int STAGES) {
    const int tiles = STAGES * (BM + BN) * dense_slabs(P) * 64, rows = WM * WN * (BM / WM < 32 ? BM / WM : 32) * (BN / WN + 4) * 4;
    return tiles > rows ? tiles : rows;
}

// Waits for this wavefront's requests but the youngest YOUNG and for its LDS reads, then for the block: what those requests filled stands in LDS for all, and what was read before may be
// overwritten.
template <int YOUNG>
__device__ __forceinline__ void dense_meet() {
    static_assert(YOUNG < 64, "the counter's range");
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(YOUNG) : "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// C's tile of BM x BN by WM x WN wavefronts, each BM/WM x BN/WN of it in fragments of 16 x 16, and STAGES copies in LDS: while a step is multiplied, the next STAGES - 1 are on their way.
// For tiles of which a compute unit holds several blocks (two copies), for grids that leave it but one (four: the memory's latency is then what a step costs), and for values in three pieces.
template <typename H, int P, bool AL, bool BL, int BM, int BN, int WM, int WN, int STAGES, typename E>
__global__ void __launch_bounds__(64 * WM * WN) dense_kernel(const DenseArgs g, const typename E::Args e) {
    constexpr int T = 64 * WM * WN, I = BM / WM / 16, J = BN / WN / 16;
    typedef DenseTile<P, AL, BM, T> TA;
    typedef DenseTile<P, BL, BN, T> TB;
    constexpr int COPY = TA::BYTES + TB::BYTES, REQ = TA::REQ + TB::REQ;
    __shared__ __attribute__((aligned(1024))) char lds[dense_shared(P, BM, BN, WM, WN, STAGES)];
    int tm, tn;
    if (!dense_place<E::MIRROR>(g, 8, tm, tn)) return;
    const int32_t M = rows_here(g.d_M, g.M), K = rows_here(g.d_K, g.K), m0 = tm * BM, n0 = tn * BN;
    if (m0 >= M) return;
    const int wave = (int)threadIdx.x >> 6, wm = wave / WN, wn = wave % WN;
    TA ta;
    TB tb;
    DenseOperand oa = g.a;
    if (AL) oa.extent = min(oa.extent, M);
    ta.open(oa, blockIdx.z, m0);
    tb.open(g.b, blockIdx.z, n0);
    const int32_t steps = (K + TA::BK - 1) / TA::BK, first = (int32_t)((int64_t)steps * blockIdx.y / g.splits), last = (int32_t)((int64_t)steps * (blockIdx.y + 1) / g.splits);
    const int32_t whole = K / TA::BK;
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds + (uint32_t)wave * 1024u);
    f32x4 acc[I][J];
    f32x4 big[P == 3 ? I : 1][P == 3 ? J : 1];       // of three pieces: the largest product's sums apart from the other five's
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j) {
            acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            if constexpr (P == 3) big[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
    // (steps past K are zeros, those past `last` are loaded and not used)
    auto request = [&](int32_t s, uint32_t copy) {
        if (s >= whole) {
            const int32_t left = K - s * TA::BK;
            ta.cut(AL ? (left + 7) & ~7 : left);
            tb.cut(BL ? (left + 7) & ~7 : left);
        }
        const i32x4 ra = ta.source(s), rb = tb.source(s);
#pragma unroll
        for (int i = 0; i < TA::REQ; ++i) ta.request_one(i, ra, lds0 + copy);
#pragma unroll
        for (int i = 0; i < TB::REQ; ++i) tb.request_one(i, rb, lds0 + copy + TA::BYTES);
    };
#pragma unroll
    for (int c = 0; c < STAGES - 1; ++c) request(first + c, c * COPY);
    uint32_t at = 0;
    for (int32_t s = first; s < last; ++s) {
        dense_meet<REQ * (STAGES - 2)>();
        request(s + STAGES - 1, at == 0 ? (STAGES - 1) * COPY : at - COPY);        // into the copy of the step before
        const char* now = lds + at;
        auto take_a = [&](s16x8 (&a)[I], int h) {
#pragma unroll
            for (int i = 0; i < I; ++i) a[i] = TA::fragment(now, wm * I + i, h);
        };
        auto take_b = [&](s16x8 (&b)[J], int h) {
#pragma unroll
            for (int j = 0; j < J; ++j) b[j] = TB::fragment(now + TA::BYTES, wn * J + j, h);
        };
        if constexpr (P == 1) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                s16x8 a[I], b[J];
                take_b(b, h);
                take_a(a, h);
                dense_multiply<H>(acc, a, b);
            }
        } else if constexpr (P == 2) {
            s16x8 a0[I], a1[I], b0[J], b1[J];
            take_b(b0, 0);
            take_a(a1, 1);
            dense_multiply<H>(acc, a1, b0);
            take_b(b1, 1);
            take_a(a0, 0);
            dense_multiply<H>(acc, a0, b1);
            dense_multiply<H>(acc, a0, b0);
        } else {
            // (a2 b0) (a0 b2) (a1 b1) (a1 b0) (a0 b1), and (a0 b0) apart
            s16x8 a[3][I], b[3][J];
            take_b(b[0], 0);
            take_a(a[2], 2);
            dense_multiply<H>(acc, a[2], b[0]);
            take_a(a[0], 0);
            dense_multiply<H>(big, a[0], b[0]);
            take_b(b[2], 2);
            dense_multiply<H>(acc, a[0], b[2]);
            take_b(b[1], 1);
            take_a(a[1], 1);
            dense_multiply<H>(acc, a[1], b[1]);
            dense_multiply<H>(acc, a[1], b[0]);
            dense_multiply<H>(acc, a[0], b[1]);
        }
        at = at == (STAGES - 1) * COPY ? 0 : at + COPY;
    }
    if constexpr (P == 3)
#pragma unroll
        for (int i = 0; i < I; ++i)
#pragma unroll
            for (int j = 0; j < J; ++j) acc[i][j] += big[i][j];
    dense_meet<0>();
    dense_finish<BM, BN, WM, WN, E>(g, e, tm, tn, M, acc, lds);
}

// One product into accumulation registers. (Left to the compiler, sums that fill half of a wavefront's registers are moved to and fro between the two kinds in every step.) Operands come from
// LDS reads, which the compiler waits for; after the last one dense_settle() has to stand before the sums are read.
template <typename H> __device__ __forceinline__ void dense_mfma_in_place(f32x4& c, s16x8 b, s16x8 a);
template <> __device__ __forceinline__ void dense_mfma_in_place<__bf16>(f32x4& c, s16x8 b, s16x8 a) {
    asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(b), "v"(a));
}
template <> __device__ __forceinline__ void dense_mfma_in_place<_Float16>(f32x4& c, s16x8 b, s16x8 a) {
    asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(c) : "v"(b), "v"(a));
}
__device__ __forceinline__ void dense_settle() { asm volatile("s_nop 15\n\ts_nop 15" ::: "memory"); }

// The same for large products: a tile of 256 x 256 by four wavefronts of 128 x 128, one a SIMD, whose registers hold the next fragments beside the ones that are multiplied, so that reads of LDS,
// requests and products go on together, and the block meets once a step. A copy of LDS is free when its last fragments are in registers: the step after next is requested right then, and has a
// whole step's time to arrive. LDS is read 16 bytes for 8192 multiplications (by eight wavefronts of 128 x 64: 24 bytes, which takes LDS as long as the products).
template <typename H, int P, bool AL, bool BL, typename E>
__global__ void __launch_bounds__(256, 1) dense_large_kernel(const DenseArgs g, const typename E::Args e) {
    static_assert(P <= 2, "three pieces do not fit the registers");
    constexpr int B = 256, T = 256, I = 8, J = 8;
    typedef DenseTile<P, AL, B, T> TA;
    typedef DenseTile<P, BL, B, T> TB;
    __shared__ __attribute__((aligned(1024))) char lds[dense_shared(P, B, B, 2, 2, 2)];
    int tm, tn;
    if (!dense_place<E::MIRROR>(g, 8, tm, tn)) return;
    const int32_t M = rows_here(g.d_M, g.M), K = rows_here(g.d_K, g.K), m0 = tm * B, n0 = tn * B;
    if (m0 >= M) return;
    const int wave = (int)threadIdx.x >> 6, wm = wave >> 1, wn = wave & 1;
    TA ta;
    TB tb;
    DenseOperand oa = g.a;
    if (AL) oa.extent = min(oa.extent, M);
    ta.open(oa, blockIdx.z, m0);
    tb.open(g.b, blockIdx.z, n0);
    const int32_t steps = (K + TA::BK - 1) / TA::BK, first = (int32_t)((int64_t)steps * blockIdx.y / g.splits), last = (int32_t)((int64_t)steps * (blockIdx.y + 1) / g.splits);
    f32x4 acc[I][J];
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j) {
            acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            asm volatile("" : "+a"(acc[i][j]));
        }
    constexpr int COPY = TA::BYTES + TB::BYTES, REQ = TA::REQ + TB::REQ;
    static_assert(REQ == 16, "one request for four products");
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds + (uint32_t)wave * 1024u);
    const int32_t whole = K / TA::BK;
    i32x4 ra, rb;
    // what comes before the requests of step s (those past K are zeros, those past `last` are loaded and not used)
    auto aim = [&](int32_t s) {
        if (s >= whole) {
            const int32_t left = K - s * TA::BK;
            ta.cut(AL ? (left + 7) & ~7 : left);
            tb.cut(BL ? (left + 7) & ~7 : left);
        }
        ra = ta.source(s);
        rb = tb.source(s);
    };
    auto request = [&](int n, int copy) {
        if (n < TA::REQ) ta.request_one(n, ra, lds0 + copy * COPY);
        else tb.request_one(n - TA::REQ, rb, lds0 + copy * COPY + TA::BYTES);
    };
    auto take = [&](int n, s16x8 (&a)[I], int ha, s16x8 (&b)[J], int hb, int copy) {       // fragment n of the sixteen: in the order in which the products want them
        if (n < 4) b[n] = TB::fragment(lds + copy * COPY + TA::BYTES, wn * J + n, hb);
        else if (n == 4) a[0] = TA::fragment(lds + copy * COPY, wm * I, ha);
        else if (n < 9) b[n - 1] = TB::fragment(lds + copy * COPY + TA::BYTES, wn * J + n - 1, hb);
        else a[n - 8] = TA::fragment(lds + copy * COPY, wm * I + n - 8, ha);
    };
    // Product n of 64, and the end of what may stand beside it: a wavefront issues in order, and while a product is at work the next one waits, so that other instructions are free only
    // one or two at a time, between products (four products and then what four of them need: 503 us for what takes 400 so).
    auto one = [&](int n, s16x8 (&a)[I], s16x8 (&b)[J]) {
        dense_mfma_in_place<H>(acc[n >> 3][n & 7], b[n & 7], a[n >> 3]);
        __builtin_amdgcn_sched_barrier(0);
    };
    aim(first);
#pragma unroll
    for (int n = 0; n < REQ; ++n) request(n, 0);
    aim(first + 1);
#pragma unroll
    for (int n = 0; n < REQ; ++n) request(n, 1);
    dense_meet<0>();
    s16x8 a0[I], a1[I], b0[J], b1[J];
    auto step = [&](auto copy_of, int32_t s) {
        constexpr int now = decltype(copy_of)::value;
        if constexpr (P == 1) {
#pragma unroll
            for (int n = 0; n < 64; ++n) {
                if (n % 2 == 0 && n < 32) take(n / 2, a1, 1, b1, 1, now);
                one(n, a0, b0);
            }
            aim(s + 2);
            dense_meet<0>();
#pragma unroll
            for (int n = 0; n < 64; ++n) {
                if (n % 4 == 0) take(n / 4, a0, 0, b0, 0, now ^ 1);
                if (n % 4 == 2) request(n / 4, now);
                one(n, a1, b1);
            }
        } else {
#pragma unroll
            for (int n = 0; n < 64; ++n) {
                if (n % 4 == 0) take(n / 4, a0, 0, b1, 1, now);
                one(n, a1, b0);
            }
#pragma unroll
            for (int n = 0; n < 64; ++n) one(n, a0, b0);
            aim(s + 2);
            dense_meet<0>();
#pragma unroll
            for (int n = 0; n < 64; ++n) {
                if (n % 4 == 0) take(n / 4, a1, 1, b0, 0, now ^ 1);
                if (n % 4 == 2) request(n / 4, now);
                one(n, a0, b1);
            }
        }
    };
#pragma unroll
    for (int n = 0; n < 16; ++n) take(n, P == 1 ? a0 : a1, P == 1 ? 0 : 1, b0, 0, 0);
    int32_t s = first;
    for (; s + 1 < last; s += 2) {
        step(std::integral_constant<int, 0>{}, s);
        step(std::integral_constant<int, 1>{}, s + 1);
    }
    if (s < last) step(std::integral_constant<int, 0>{}, s);
    dense_settle();
    dense_meet<0>();
    dense_finish<B, B, 2, 2, E>(g, e, tm, tn, M, acc, lds);
}

}  // namespace no
