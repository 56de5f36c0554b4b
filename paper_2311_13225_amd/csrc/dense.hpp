// Matrix products of 16-bit operands (bf16, or fp16 pieces of fp32 values) on the matrix cores, with fp32 sums: the dense layer (linear.hip) and the orthogonalised
// update (orthogonalise.hip). C[m, n] = sum over k of A(m, k) B(k, n), where a value is one 16-bit piece, or the sum of P of them, P = 2 or 3, whose products are taken but for the smallest. An operand lies ALONG the reduction (k contiguous in memory) or across it.
#pragma once
#include "rows.hpp"

namespace no {

typedef float f32x4 __attribute__((ext_vector_type(4)));
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
    int32_t splits, tiles_m, tiles_n, matrices;
};

static inline size_t round_256(size_t b) { return (b + 255) / 256 * 256; }
static inline int64_t wide_of(int64_t dim) { return (dim + 7) / 8 * 8; }       // values of a row of whole 16 bytes

// A step takes slabs of 32 reduction indices: two of a matrix of one piece, else one of each piece.
constexpr int dense_slabs(int P) { return P == 1 ? 2 : P; }
constexpr int dense_bk(int P) { return P == 1 ? 64 : 32; }
constexpr uint32_t DENSE_NOWHERE = 0x80000000u;      // past every buffer's range: reads as 0

// One operand's tile of R rows (or columns) and a step's slabs in LDS, loaded by T threads in requests of 16 bytes that go straight to LDS. A request's 64 lanes fill 1 KB in lane
// order, so the order of the units in LDS is made by which unit a lane asks for: ALONG, unit u of row r stands at place u ^ (r & 7) of its 128 bytes (three pieces: at
// u ^ (r >> 2 & 3) of its 192); across, the 32 bytes of 16 columns of line k stand at place c ^ f(k), f(k) = (k & 3) | (k >> 3 & 1) << 2 (192 columns, whose lines begin half of the banks apart: (k >> 1 & 1) |
// (k >> 3 & 1) << 1). Then the 64 lanes of a fragment's read meet every bank equally often
// (SQ_LDS_BANK_CONFLICT 0 with one piece; with more, where requests and reads meet, up to 6 % of the cycles in the large tiles, 17 % in two pieces of 128 x 128).
template <int P, bool ALONG, int R, int T>
struct DenseTile {
    static constexpr int SLABS = dense_slabs(P), BK = dense_bk(P), PER_ROW = ALONG ? SLABS * 4 : R / 8, BYTES = R * SLABS * 64, REQ = BYTES / (16 * T);
    static_assert(BYTES % (16 * T) == 0 && R >= 32, "whole requests");
    uint32_t off[REQ];
    const char* base;                   // the tile's origin in the matrix
    int64_t step;                       // bytes from one step to the next
    __device__ __forceinline__ static int mix(int k) { return R == 192 ? (k >> 1 & 1) | (k >> 3 & 1) << 1 : ((k & 3) | (k >> 3 & 1) << 2) & (R / 16 - 1); }
    // what request i of this thread asks for: line of the tile, unit of the line
    __device__ __forceinline__ static void which(int i, int& line, int& unit) {
        const int c = i * T + ((int)threadIdx.x & (T - 1)), place = c % PER_ROW;
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
    // fills is waited for in dense_meet(). Nothing is masked here: cut() comes before the first step that is not whole. A load into LDS takes its place from m0, one wait state after a scalar instruction wrote that.
    __device__ __forceinline__ i32x4 source(int32_t s) const {
        const uint64_t at = (uint64_t)(base + (int64_t)s * step);
        return i32x4{(int)(uint32_t)at, (int)(uint32_t)(at >> 32), 0x7fffffff, 0x00020000};
    }
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"      /* (it warns of m0, which the compiler keeps no value in) */
    __device__ __forceinline__ void request_one(int i, i32x4 rsrc, uint32_t to) const {
        asm volatile("s_add_u32 m0, %2, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" : : "v"(off[i]), "s"(rsrc), "s"(to), "i"(i * T * 16) : "memory", "scc", "m0");
    }
#pragma clang diagnostic pop
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

// A block's place: the tiles of all matrices are dealt to the dies in runs, and walked in bands of eight tile rows, so that a die's blocks share rows and columns in its L2 (four Gram matrices of 512 x 2048, each
// matrix dealt to all dies: 22.2 us, to two of them 20.5).
// HALF: the tiles on and above the diagonal of a square alone.
constexpr int DENSE_BAND = 8;
static inline int64_t dense_tiles(int64_t tiles_m, int64_t tiles_n, bool half) { return half ? tiles_m * (tiles_m + 1) / 2 : tiles_m * tiles_n; }
template <bool HALF>
__device__ __forceinline__ bool dense_place(const DenseArgs& g, int& matrix, int& tm, int& tn) {
    const int padded = (int)gridDim.x, tiles = HALF ? g.tiles_m * (g.tiles_m + 1) / 2 : g.tiles_m * g.tiles_n;
    int id = ((int)blockIdx.x % 8) * (padded / 8) + (int)blockIdx.x / 8;
    if (id >= tiles * g.matrices) return false;
    matrix = id / tiles;
    id -= matrix * tiles;
    if (HALF) {         // a band's corner on the diagonal, then its whole columns
        int row = 0, rows, corner;
        for (;; row += DENSE_BAND) {
            rows = min(DENSE_BAND, g.tiles_m - row);
            corner = rows * (rows + 1) / 2;
            const int all = corner + (g.tiles_m - row - rows) * rows;
            if (id < all) break;
            id -= all;
        }
        if (id < corner) {
            int j = 0;
            while ((j + 1) * (j + 2) / 2 <= id) ++j;
            tn = row + j;
            tm = row + id - j * (j + 1) / 2;
        } else {
            id -= corner;
            tn = row + rows + id / rows;
            tm = row + id % rows;
        }
        return true;
    }
    const int per = DENSE_BAND * g.tiles_n, b = id / per, rest = id - b * per, rows = min(DENSE_BAND, g.tiles_m - b * DENSE_BAND);
    tm = b * DENSE_BAND + rest % rows;
    tn = rest / rows;
    return true;
}

// Sums of products of three pieces that are not finite, once more in fp32, one product after the other, from the values that the pieces add up to (RAW: from fp32 rows as they lie): an infinity meets the other operand's
// pieces, zeros and opposite signs among them, and a piece that is rounded up may leave fp32 where its value does not. The reduction's part is [k0, k1).
template <bool AL, bool BL, bool RAW>
struct DenseAgain {
    static constexpr bool THERE = true;
    const DenseArgs& g;
    int32_t k0, k1;
    template <bool ALONG>
    __device__ __forceinline__ static float value(const DenseOperand& o, int32_t row, int32_t k) {
        const char* p = o.p + (ALONG ? row * o.pitch + (int64_t)k * 2 : k * o.pitch + (int64_t)row * 2);
        float f = 0.0f;
#pragma unroll
        for (int q = 0; q < 3; ++q) f += to_f32(*reinterpret_cast<const bf16_t*>(p + (int64_t)q * o.plane));      // (exact, largest first)
        return f;
    }
    // The factor of row m at index k of the reduction.
    __device__ __forceinline__ float left(int32_t m, int32_t k) const {
        if constexpr (RAW) return *reinterpret_cast<const float*>(g.a.p + m * g.a.pitch + (int64_t)k * 4);
        else return value<AL>(g.a, m, k);
    }
    // Eight columns of row m from n on, `here` of them there: the sums at `at` that are not finite. A NaN stays one: then the rest of the reduction is left out. Columns that lie beside one another in memory are taken at once
    // (8192 x 2048 x 8192 with NaN in the middle row of W, every sum anew: 47 ms, one by one 100), rows one by one, for their addresses would take the registers that let three blocks share a compute unit.
    __device__ __forceinline__ void operator()(int32_t m, int32_t n, int32_t here, float* at) const {
        if constexpr (BL) {
#pragma unroll 1
            for (int w = 0; w < here; ++w) {
                if (fabsf(at[w]) < INFINITY) continue;
                constexpr int U = 8;        // products whose factors are asked for at once
                float sum = 0.0f;
#pragma unroll 1
                for (int32_t k = k0; k < k1 && sum == sum; k += U) {
                    float a[U], b[U];
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        a[u] = left(m, min(k + u, k1 - 1));
                        b[u] = value<true>(g.b, n + w, min(k + u, k1 - 1));
                    }
#pragma unroll
                    for (int u = 0; u < U; ++u) if (k + u < k1) sum = fmaf(a[u], b[u], sum);
                }
                at[w] = sum;
            }
        } else {
            bool odd = false;
#pragma unroll
            for (int w = 0; w < 8; ++w) odd |= w < here && !(fabsf(at[w]) < INFINITY);
            float sum[8] = {};
#pragma unroll 1
            for (int32_t k = k0; k < k1 && odd; ++k) {
                const float a = left(m, k);
                float b[8], f[8];
                odd = false;
#pragma unroll
                for (int q = 0; q < 3; ++q) {
                    Run<bf16_t, 8> r;       // (rows of whole eights)
                    r.load(reinterpret_cast<const bf16_t*>(g.b.p + k * g.b.pitch + (int64_t)q * g.b.plane) + n);
                    r.get(f);
#pragma unroll
                    for (int w = 0; w < 8; ++w) b[w] = q ? b[w] + f[w] : f[w];
                }
#pragma unroll
                for (int w = 0; w < 8; ++w) {
                    sum[w] = fmaf(a, b[w], sum[w]);
                    odd |= sum[w] == sum[w];
                }
            }
#pragma unroll
            for (int w = 0; w < 8; ++w) if (!(fabsf(at[w]) < INFINITY)) at[w] = sum[w];
        }
    }
};
struct DenseOnce { static constexpr bool THERE = false; };      // sums of one piece, or of two

// The sums of a block's tile to the epilogue: through LDS, 32 rows of a wavefront at a time, so that eight consecutive columns of a row meet in a lane and the lanes beside it go on along
// the row. What the epilogue reads of those rows is asked for at once, before the first of them, and waits in LDS for its row (asked for row by row, 16384 x 8192 x 2048 bf16 with a residual lost 35 us of 250 a
// tile): E::ahead(epilogue's arguments, matrix, m, n, columns there), then E::put(arguments, matrix, m, n, columns there, sums, what was read, M), which leaves in the sums what it stored; E::MIRROR: that
// is stored as C[n, m], too.
template <int BM, int BN, int WM, int WN>
struct DenseFinish {
    static constexpr int T = 64 * WM * WN, COLS = BN / WN, PITCH = COLS + 4, LANES = COLS == 96 ? 16 : COLS / 8, ROWS = BM / WM % 32 == 0 ? 32 : 16, PASS = 64 / LANES, TURNS = ROWS / PASS, AHEAD = 32;
    static constexpr int SUMS = WM * WN * ROWS * PITCH * 4, BYTES = SUMS + (TURNS > 2 ? T * TURNS * AHEAD : 0);
    static_assert(ROWS % PASS == 0, "whole passes");
};
template <int BM, int BN, int WM, int WN, typename E, int I, int J, typename Again>
__device__ __forceinline__ void dense_finish(const DenseArgs& g, const typename E::Args& e, int matrix, int tm, int tn, int32_t M, f32x4 (&acc)[I][J], char* lds, const Again& again) {
    typedef DenseFinish<BM, BN, WM, WN> F;
    constexpr int COLS = F::COLS, PITCH = F::PITCH, LANES = F::LANES, ROWS = F::ROWS, RI = ROWS / 16, PASS = F::PASS, TURNS = F::TURNS;
    constexpr bool HELD = TURNS > 2;
    typedef typename E::Ahead Ahead;
    static_assert(I % RI == 0 && sizeof(Ahead) <= F::AHEAD, "whole rounds");
    const int wave = ((int)threadIdx.x & (F::T - 1)) >> 6, wm = wave / WN, wn = wave % WN, l = (int)threadIdx.x & 63;
    const int32_t nw = tn * BN + wn * COLS, n = nw + l % LANES * 8, here = l % LANES * 8 < COLS ? min(8, g.N - n) : 0;      // (of 16 lanes to 96 columns four have none)
    float* mine = reinterpret_cast<float*>(lds) + wave * ROWS * PITCH;
    Ahead* held = reinterpret_cast<Ahead*>(lds + F::SUMS) + (wave * 64 + l);
    f32x4 odd = {0.0f, 0.0f, 0.0f, 0.0f};       // NaN from the first sum on that is not finite
    if constexpr (Again::THERE)
#pragma unroll
        for (int i = 0; i < I; ++i)
#pragma unroll
            for (int j = 0; j < J; ++j)
#pragma unroll
                for (int w = 0; w < 4; ++w) odd[w] = fmaf(acc[i][j][w], 0.0f, odd[w]);
    const bool any_odd = Again::THERE && __any((odd[0] + odd[1]) + (odd[2] + odd[3]) != 0.0f);
#pragma unroll
    for (int i0 = 0; i0 < I; i0 += RI) {
        const int32_t mw = tm * BM + (wm * I + i0) * 16, mine0 = mw + l / LANES;
        Ahead ahead[TURNS];
#pragma unroll
        for (int t = 0; t < TURNS; ++t)
            if (mine0 + t * PASS < M && here > 0) ahead[t] = E::ahead(e, matrix, mine0 + t * PASS, n, here);
        Team<64, F::T>::sync();
#pragma unroll
        for (int i = 0; i < RI; ++i)
#pragma unroll
            for (int j = 0; j < J; ++j) *reinterpret_cast<f32x4*>(mine + (i * 16 + (l & 15)) * PITCH + j * 16 + (l >> 4) * 4) = acc[i0 + i][j];
        if constexpr (HELD)
#pragma unroll
            for (int t = 0; t < TURNS; ++t) held[t * F::T] = ahead[t];
        Team<64, F::T>::sync();
        if constexpr (Again::THERE) {
            if (__builtin_expect(any_odd, 0))      // (its code out of the way: in line, 24922 x 256 x 256 takes 37.4 us for 35.1, by the fetch of what stands behind it)
#pragma unroll 1
                for (int t = 0; t < TURNS; ++t)
                    if (mine0 + t * PASS < M && here > 0) again(mine0 + t * PASS, n, here, mine + (l / LANES + t * PASS) * PITCH + l % LANES * 8);
        }
        auto turn = [&](int t, const Ahead& a) {
            const int32_t m = mine0 + t * PASS;
            if (m >= M || here <= 0) return;
            float v[8];
            f32x4* at = reinterpret_cast<f32x4*>(mine + (l / LANES + t * PASS) * PITCH + l % LANES * 8);
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const f32x4 x = at[q];
#pragma unroll
                for (int w = 0; w < 4; ++w) v[4 * q + w] = x[w];
            }
            E::put(e, matrix, m, n, here, v, a, g.M);
            if constexpr (E::MIRROR)
#pragma unroll
                for (int q = 0; q < 2; ++q) at[q] = f32x4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
        };
        if constexpr (HELD) {
#pragma unroll 1
            for (int t = 0; t < TURNS; ++t) turn(t, held[t * F::T]);
        } else {
#pragma unroll
            for (int t = 0; t < TURNS; ++t) turn(t, ahead[t]);
        }
        if constexpr (E::MIRROR) {          // eight consecutive m a lane
            if (tm == tn) continue;
            Team<64, F::T>::sync();
#pragma unroll 1
            for (int c = l / (ROWS / 8); c < COLS; c += 64 / (ROWS / 8)) {
                const int32_t n2 = nw + c, m = mw + l % (ROWS / 8) * 8;
                if (m >= M || n2 >= g.N) continue;
                float v[8];
#pragma unroll
                for (int w = 0; w < 8; ++w) v[w] = m + w < M ? mine[(l % (ROWS / 8) * 8 + w) * PITCH + c] : 0.0f;
                E::mirror(e, matrix, n2, m, v, g.M);
            }
        }
    }
}

constexpr int dense_shared(int P, int BM, int BN, int STAGES, int GROUPS, int finish) {
    const int tiles = GROUPS * STAGES * (BM + BN) * dense_slabs(P) * 64;
    return tiles > finish ? tiles : finish;
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

// One product into accumulation registers. (Left to the compiler, sums that fill half of a wavefront's registers are moved to and fro between the two kinds in every step.) Operands come from
// LDS reads, which the compiler waits for; after the last one dense_settle() has to stand before the sums are read.
template <typename H> __device__ __forceinline__ void dense_mfma_in_place(f32x4& c, s16x8 b, s16x8 a);
template <> __device__ __forceinline__ void dense_mfma_in_place<__bf16>(f32x4& c, s16x8 b, s16x8 a) {
    asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(b), "v"(a));
}
template <> __device__ __forceinline__ void dense_mfma_in_place<_Float16>(f32x4& c, s16x8 b, s16x8 a) {
    asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(c) : "v"(b), "v"(a));
}
template <int I, int J>
__device__ __forceinline__ void dense_settle(f32x4 (&acc)[I][J]) {
    asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j) asm volatile("" : "+a"(acc[i][j]));      // (nothing reads them from before)
}

// C's tile of BM x BN by WM x WN wavefronts, each BM/WM x BN/WN of it in fragments of 16 x 16, and STAGES copies in LDS. While a step is multiplied, the fragments of the next are read into the
// other half of a wavefront's registers, and the step STAGES further on is requested into the copy whose fragments are being multiplied. The block meets once a step.
// GROUPS of so many wavefronts take the steps in turn, each with copies of its own, and the first adds up the others' sums in order: for products so small that the steps' number is what they last.
template <typename H, int P, bool AL, bool BL, int BM, int BN, int WM, int WN, int STAGES, int GROUPS, typename E>
__global__ void __launch_bounds__(64 * WM * WN * GROUPS) dense_kernel(const DenseArgs g, const typename E::Args e) {
    constexpr int T = 64 * WM * WN, I = BM / WM / 16, J = BN / WN / 16, S = dense_slabs(P), PAIRS = P == 1 ? 2 : P == 2 ? 3 : 6;
    typedef DenseTile<P, AL, BM, T> TA;
    typedef DenseTile<P, BL, BN, T> TB;
    constexpr int COPY = TA::BYTES + TB::BYTES, REQ = TA::REQ + TB::REQ;
    __shared__ __attribute__((aligned(1024))) char lds[dense_shared(P, BM, BN, STAGES, GROUPS, DenseFinish<BM, BN, WM, WN>::BYTES)];
    int matrix, tm, tn;
    if (!dense_place<E::MIRROR>(g, matrix, tm, tn)) return;
    const int32_t M = rows_here(g.d_M, g.M), K = rows_here(g.d_K, g.K), m0 = tm * BM, n0 = tn * BN;
    if (m0 >= M) return;
    const int group = __builtin_amdgcn_readfirstlane((int)threadIdx.x / T), wave = ((int)threadIdx.x & (T - 1)) >> 6, wm = wave / WN, wn = wave % WN;
    char* const mine = lds + group * STAGES * COPY;
    TA ta;
    TB tb;
    DenseOperand oa = g.a;
    if (AL) oa.extent = min(oa.extent, M);
    ta.open(oa, matrix, m0);
    tb.open(g.b, matrix, n0);
    const int32_t steps = (K + TA::BK - 1) / TA::BK, first = (int32_t)((int64_t)steps * blockIdx.y / g.splits), last = (int32_t)((int64_t)steps * (blockIdx.y + 1) / g.splits);
    const int32_t end = min(K, last * TA::BK), whole = end / TA::BK;
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)mine + (uint32_t)wave * 1024u);
    f32x4 acc[I][J];
    f32x4 big[P == 3 ? I : 1][P == 3 ? J : 1];       // of three pieces: the largest product's sums apart from the other five's
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j) {
            acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            asm volatile("" : "+a"(acc[i][j]));
            if constexpr (P == 3) {
                big[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                asm volatile("" : "+a"(big[i][j]));
            }
        }
    i32x4 ra, rb;
    // what comes before the requests of step s (those past `last` are zeros)
    auto aim = [&](int32_t s) {
        if (s >= whole) {
            const int32_t left = end - s * TA::BK;
            ta.cut(AL ? (left + 7) & ~7 : left);
            tb.cut(BL ? (left + 7) & ~7 : left);
        }
        ra = ta.source(s);
        rb = tb.source(s);
    };
    auto request = [&](int n, uint32_t copy) {
        if (n < TA::REQ) ta.request_one(n, ra, lds0 + copy);
        else tb.request_one(n - TA::REQ, rb, lds0 + copy + TA::BYTES);
    };
    s16x8 fa[2][S][I], fb[2][S][J];
    // the pairs of slabs that are multiplied, in order; of pieces the smallest products first
    constexpr int PA[3][6] = {{0, 1}, {1, 0, 0}, {2, 0, 1, 1, 0, 0}}, PB[3][6] = {{0, 1}, {0, 1, 0}, {0, 2, 1, 0, 1, 0}};
    // fragment n of a step's, in the order in which the pairs want them: b before a, slab by slab
    auto take = [&](int n, s16x8 (&a)[S][I], s16x8 (&b)[S][J], const char* from) {
        constexpr int OA[3][3] = {{0, 1}, {1, 0}, {2, 0, 1}}, OB[3][3] = {{0, 1}, {0, 1}, {0, 2, 1}};
        const int h = n / (I + J), k = n % (I + J);
        if (k < J) b[OB[P - 1][h]][k] = TB::fragment(from + TA::BYTES, wn * J + k, OB[P - 1][h]);
        else a[OA[P - 1][h]][k - J] = TA::fragment(from, wm * I + k - J, OA[P - 1][h]);
    };
    constexpr int PRODUCTS = PAIRS * I * J, READS = S * (I + J), ITEMS = READS + REQ;
    uint32_t at = 0;        // the copy of the step that is multiplied
    auto step = [&](auto half_of, int32_t s) {
        constexpr int half = decltype(half_of)::value;
        dense_meet<REQ * (STAGES - 2)>();
        const uint32_t next = at == (STAGES - 1) * COPY ? 0 : at + COPY;
        aim(s + STAGES * GROUPS);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < PRODUCTS; ++n) {
#pragma unroll
            for (int k = n * ITEMS / PRODUCTS; k < (n + 1) * ITEMS / PRODUCTS; ++k) {
                if (k < READS) take(k, fa[half ^ 1], fb[half ^ 1], mine + next);
                else request(k - READS, at);
            }
            const int pair = n / (I * J), i = n / J % I, j = n % J;
            if (P == 3 && pair == 5) dense_mfma_in_place<H>(big[P == 3 ? i : 0][P == 3 ? j : 0], fb[half][PB[P - 1][pair]][j], fa[half][PA[P - 1][pair]][i]);
            else dense_mfma_in_place<H>(acc[i][j], fb[half][PB[P - 1][pair]][j], fa[half][PA[P - 1][pair]][i]);
            __builtin_amdgcn_sched_barrier(0);
        }
        at = next;
    };
#pragma unroll
    for (int c = 0; c < STAGES; ++c) {
        aim(first + group + c * GROUPS);
#pragma unroll
        for (int n = 0; n < REQ; ++n) request(n, c * COPY);
    }
    dense_meet<REQ * (STAGES - 1)>();
#pragma unroll
    for (int n = 0; n < READS; ++n) take(n, fa[0], fb[0], mine);
    const int32_t turns = (last - first + GROUPS - 1) / GROUPS;      // (as many for every group: steps past `last` are zeros)
    int32_t turn = 0;
    for (; turn + 1 < turns; turn += 2) {
        step(std::integral_constant<int, 0>{}, first + group + turn * GROUPS);
        step(std::integral_constant<int, 1>{}, first + group + (turn + 1) * GROUPS);
    }
    if (turn < turns) step(std::integral_constant<int, 0>{}, first + group + turn * GROUPS);
    dense_settle(acc);
    if constexpr (P == 3) dense_settle(big);
    if constexpr (P == 3)
#pragma unroll
        for (int i = 0; i < I; ++i)
#pragma unroll
            for (int j = 0; j < J; ++j) acc[i][j] += big[i][j];
    dense_meet<0>();
    if constexpr (GROUPS > 1) {
        static_assert((GROUPS - 1) * I * J * T * 16 <= (int)sizeof(lds), "room for the other groups' sums");
        f32x4* sums = reinterpret_cast<f32x4*>(lds) + ((int)threadIdx.x & (T - 1));
        if (group > 0)
#pragma unroll
            for (int i = 0; i < I; ++i)
#pragma unroll
                for (int j = 0; j < J; ++j) sums[((group - 1) * I * J + i * J + j) * T] = acc[i][j];
        __syncthreads();
        if (group == 0)
#pragma unroll
            for (int k = 1; k < GROUPS; ++k)
#pragma unroll
                for (int i = 0; i < I; ++i)
#pragma unroll
                    for (int j = 0; j < J; ++j) acc[i][j] += sums[((k - 1) * I * J + i * J + j) * T];
        __syncthreads();
        if (group > 0) return;
    }
    if constexpr (P == 3) dense_finish<BM, BN, WM, WN, E>(g, e, matrix, tm, tn, M, acc, lds, DenseAgain<AL, BL, false>{g, first * TA::BK, end});
    else dense_finish<BM, BN, WM, WN, E>(g, e, matrix, tm, tn, M, acc, lds, DenseOnce{});
}

// The same for large products: a tile of 256 x 256 (192 x 192 where that fills the chip better; three pieces: 256 x 128) by four wavefronts of a quarter each, one a SIMD, whose sums fill the accumulation registers; the others hold one set of
// fragments a slab, and a set is read again when the products that want it are done. A copy of LDS is free when its last fragments are in registers: the step after next is requested right then, and
// has a whole step's time to arrive. LDS is read 16 bytes for 8192 multiplications (by eight wavefronts of 128 x 64: 24 bytes, which takes LDS as long as the products).
// Bound by the matrix pipes, at work in 56 to 75 % of the cycles, at the 1.9 to 2.15 GHz that the power limit leaves them (kernels below it run at 2.35): bf16 16384 x 8192 x 2048 439 us (1.25 PFLOP/s), both products of 8192 x 2048 x 8192's gradients 195 to 200 (1.4 when the card is cold);
// two pieces, 4096^3 300 (1.37 PFLOP/s of pieces), its symmetric half 190 by 192 x 192.
template <typename H, int P, bool AL, bool BL, int BM, int BN, typename E>
__global__ void __launch_bounds__(256, 1) dense_large_kernel(const DenseArgs g, const typename E::Args e) {
    constexpr int T = 256, I = BM / 32, J = BN / 32, S = dense_slabs(P), N = I * J, EACH = N / (I + J);      // (a read for EACH products)
    typedef DenseTile<P, AL, BM, T> TA;
    typedef DenseTile<P, BL, BN, T> TB;
    constexpr int COPY = TA::BYTES + TB::BYTES, REQ = TA::REQ + TB::REQ;
    __shared__ __attribute__((aligned(1024))) char lds[dense_shared(P, BM, BN, 2, 1, DenseFinish<BM, BN, 2, 2>::BYTES)];
    int matrix, tm, tn;
    if (!dense_place<E::MIRROR>(g, matrix, tm, tn)) return;
    const int32_t M = rows_here(g.d_M, g.M), K = rows_here(g.d_K, g.K), m0 = tm * BM, n0 = tn * BN;
    if (m0 >= M) return;
    const int wave = (int)threadIdx.x >> 6, wm = wave >> 1, wn = wave & 1;
    TA ta;
    TB tb;
    DenseOperand oa = g.a;
    if (AL) oa.extent = min(oa.extent, M);
    ta.open(oa, matrix, m0);
    tb.open(g.b, matrix, n0);
    const int32_t steps = (K + TA::BK - 1) / TA::BK, first = (int32_t)((int64_t)steps * blockIdx.y / g.splits), last = (int32_t)((int64_t)steps * (blockIdx.y + 1) / g.splits);
    f32x4 acc[I][J];
    f32x4 big[P == 3 ? I : 1][P == 3 ? J : 1];
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j) {
            acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            asm volatile("" : "+a"(acc[i][j]));
            if constexpr (P == 3) {
                big[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                asm volatile("" : "+a"(big[i][j]));
            }
        }
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds + (uint32_t)wave * 1024u);
    const int32_t end = min(K, last * TA::BK), whole = end / TA::BK;
    i32x4 ra, rb;
    // what comes before the requests of step s (those past `last` are zeros)
    auto aim = [&](int32_t s) {
        if (s >= whole) {
            const int32_t left = end - s * TA::BK;
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
    s16x8 fa[S][I], fb[S][J];
    auto take_a = [&](int h, int i, int copy) { fa[h][i] = TA::fragment(lds + copy * COPY, wm * I + i, h); };
    auto take_b = [&](int h, int j, int copy) { fb[h][j] = TB::fragment(lds + copy * COPY + TA::BYTES, wn * J + j, h); };
    // Product n of the N of two slabs, and the end of what may stand beside it: a wavefront issues in order, and while a product is at work the next one waits, so that other instructions are
    // free only one or two at a time, between products (four products and then what four of them need: 503 us for what takes 465 so).
    auto one = [&](int n, int ha, int hb, f32x4 (&c)[I][J]) {
        dense_mfma_in_place<H>(c[n / J][n % J], fb[hb][n % J], fa[ha][n / J]);
        __builtin_amdgcn_sched_barrier(0);
    };
    // `items` things spread over the N products, from `begin` on, the last of them no later than `until` of N
    auto here = [](int n, int items, int until) { return n < until ? (n + 1) * items / until : items; };
    auto begun = [](int n, int items, int until) { return n < until ? n * items / until : items; };
    aim(first);
#pragma unroll
    for (int n = 0; n < REQ; ++n) request(n, 0);
    aim(first + 1);
#pragma unroll
    for (int n = 0; n < REQ; ++n) request(n, 1);
    dense_meet<REQ>();
    auto step = [&](auto copy_of, int32_t s) {
        constexpr int now = decltype(copy_of)::value;
        if constexpr (P == 1) {
#pragma unroll
            for (int n = 0; n < N; ++n) {       // the second slab, b and a in turn
#pragma unroll
                for (int k = begun(n, I + J, N / 2); k < here(n, I + J, N / 2); ++k)
                    if (k % 2) take_a(1, k / 2, now);
                    else take_b(1, k / 2, now);
                one(n, 0, 0, acc);
            }
            aim(s + 2);
            dense_meet<0>();
#pragma unroll
            for (int n = 0; n < N; ++n) {
                if (n % EACH == 0) { if (n / EACH < J) take_b(0, n / EACH, now ^ 1); else take_a(0, n / EACH - J, now ^ 1); }
                if (n % EACH == EACH / 2) request(n / EACH, now);
                one(n, 1, 1, acc);
            }
        } else if constexpr (P == 2) {
#pragma unroll
            for (int n = 0; n < N; ++n) {
                if (n % EACH == 0) { if (n / EACH < I) take_a(0, n / EACH, now); else take_b(1, n / EACH - I, now); }
                one(n, 1, 0, acc);
            }
#pragma unroll
            for (int n = 0; n < N; ++n) one(n, 0, 0, acc);
            aim(s + 2);
            dense_meet<0>();
#pragma unroll
            for (int n = 0; n < N; ++n) {
                if (n % EACH == 0) { if (n / EACH < J) take_b(0, n / EACH, now ^ 1); else take_a(1, n / EACH - J, now ^ 1); }
                if (n % EACH == EACH / 2) request(n / EACH, now);
                one(n, 0, 1, acc);
            }
        } else {
#pragma unroll
            for (int n = 0; n < N; ++n) {
                if (n % 3 == 0 && n / 3 < I) take_a(0, n / 3, now);
                one(n, 2, 0, acc);
            }
#pragma unroll
            for (int n = 0; n < N; ++n) {
                if (n % 4 == 0 && n / 4 < J) take_b(2, n / 4, now);
                one(n, 0, 0, big);
            }
#pragma unroll
            for (int n = 0; n < N; ++n) {
                if (n % 3 == 0 && n / 3 < I) take_a(1, n / 3, now);
                one(n, 0, 2, acc);
            }
#pragma unroll
            for (int n = 0; n < N; ++n) {
                if (n % 4 == 0 && n / 4 < J) take_b(1, n / 4, now);
                one(n, 1, 0, acc);
            }
            aim(s + 2);
            dense_meet<0>();
#pragma unroll
            for (int n = 0; n < N; ++n) {
                if (n % 3 == 0 && n / 3 < I) take_a(2, n / 3, now ^ 1);
                if (n % 3 == 1 && n / 3 < REQ / 2) request(n / 3, now);
                one(n, 1, 1, acc);
            }
#pragma unroll
            for (int n = 0; n < N; ++n) {
                if (n % 4 == 0 && n / 4 < J) take_b(0, n / 4, now ^ 1);
                if (n % 3 == 1 && REQ / 2 + n / 3 < REQ) request(REQ / 2 + n / 3, now);
                one(n, 0, 1, acc);
            }
        }
    };
    static_assert(P == 3 ? REQ / 2 <= N / 3 && REQ - REQ / 2 <= N / 3 : REQ == I + J && N % (I + J) == 0, "a place for every request");
#pragma unroll
    for (int j = 0; j < J; ++j) take_b(0, j, 0);
#pragma unroll
    for (int i = 0; i < I; ++i) take_a(P - 1, i, 0);
    int32_t s = first;
    for (; s + 1 < last; s += 2) {
        step(std::integral_constant<int, 0>{}, s);
        step(std::integral_constant<int, 1>{}, s + 1);
    }
    if (s < last) step(std::integral_constant<int, 0>{}, s);
    dense_settle(acc);
    if constexpr (P == 3) {
        dense_settle(big);
#pragma unroll
        for (int i = 0; i < I; ++i)
#pragma unroll
            for (int j = 0; j < J; ++j) acc[i][j] += big[i][j];
    }
    dense_meet<0>();
    if constexpr (P == 3) dense_finish<BM, BN, 2, 2, E>(g, e, matrix, tm, tn, M, acc, lds, DenseAgain<AL, BL, false>{g, first * TA::BK, end});
    else dense_finish<BM, BN, 2, 2, E>(g, e, matrix, tm, tn, M, acc, lds, DenseOnce{});
}

// Values of fp32 rows cut on their way from LDS: A is the matrix itself, ALONG, at any alignment of a value, and only its last K % 32 columns are a copy (`tail`: 32 columns, zeros at the end), so that
// nothing is read past a row; B is in three pieces, across. A tile of 256 (or 224) x 128 by four wavefronts as above, but walked by fragments of 16 rows: a fragment's 24 products go on while the next
// one is cut, one or two instructions beside each product, and the one after that is read. 24922 x 602 x 256: 58 us and 5 before it; behind a copy of A in pieces, which takes 25, 62. Bound by a
// wavefront's instructions: 585 a step, of which 168 products keep the matrix pipes busy for 43 % of the time; a third copy in LDS changes nothing, a cut's differences by two-term products, seven instructions
// for eleven, take longer (66).
struct DenseRawArgs {
    DenseArgs g;            // g.a: the rows (pitch of 4-byte multiples); g.a.plane is not used
    DenseOperand tail;
};
template <int BM, typename E>
__global__ void __launch_bounds__(256, 1) dense_raw_kernel(const DenseRawArgs ga, const typename E::Args e) {
    constexpr int BN = 128, T = 256, I = BM / 32, J = 4, PRODUCTS = 6 * J;
    typedef DenseTile<1, true, BM, T> TA;       // (32 values of 4 bytes take the place of 64 of 2)
    typedef DenseTile<3, false, BN, T> TB;
    constexpr int BK = 32, COPY = TA::BYTES + TB::BYTES, REQ = TA::REQ + TB::REQ;
    static_assert(TB::BK == BK && REQ <= 2 * PRODUCTS, "steps of both operands, and a place for every request");
    __shared__ __attribute__((aligned(1024))) char lds[dense_shared(3, BM, BN, 2, 1, DenseFinish<BM, BN, 2, 2>::BYTES)];
    const DenseArgs& g = ga.g;
    int matrix, tm, tn;
    if (!dense_place<false>(g, matrix, tm, tn)) return;
    const int32_t M = rows_here(g.d_M, g.M), K = g.K, m0 = tm * BM, n0 = tn * BN;
    if (m0 >= M) return;
    const int wave = (int)threadIdx.x >> 6, wm = wave >> 1, wn = wave & 1, l = (int)threadIdx.x & 63, gr = l >> 4, j16 = l & 15;
    TA ta;
    TB tb;
    DenseOperand oa = g.a, ot = ga.tail;
    oa.extent = ot.extent = min(oa.extent, M);
    ta.open(oa, 0, m0);
    tb.open(g.b, 0, n0);
    const int32_t steps = (K + BK - 1) / BK, first = (int32_t)((int64_t)steps * blockIdx.y / g.splits), last = (int32_t)((int64_t)steps * (blockIdx.y + 1) / g.splits);
    f32x4 acc[I][J], big[I][J];       // the largest product's sums apart from the other five's
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j) {
            acc[i][j] = big[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            asm volatile("" : "+a"(acc[i][j]));
            asm volatile("" : "+a"(big[i][j]));
        }
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds + (uint32_t)wave * 1024u);
    const int32_t whole = K / BK;
    i32x4 ra, rb;
    // what comes before the requests of step s (those past K are zeros, those past `last` are loaded and not used)
    auto aim = [&](int32_t s) {
        if (s >= whole) {
            if (s == whole && K % BK != 0) {        // the copied columns, whose rows are whole
                ta.open(ot, 0, m0);
                ta.base -= (int64_t)whole * TA::BK * 2;
            } else ta.cut(0);
            tb.cut(K - s * BK);
        }
        ra = ta.source(s);
        rb = tb.source(s);
    };
    auto request = [&](int n, int copy) {
        if (n < TA::REQ) ta.request_one(n, ra, lds0 + copy * COPY);
        else tb.request_one(n - TA::REQ, rb, lds0 + copy * COPY + TA::BYTES);
    };
    s16x8 fb[2][3][J];
    i32x4 raw[2][2];                // two fragments' values on their way: eight a lane
    i32x4 piece[2][3];              // this fragment's pieces and the next one's, pairs of values
    uint32_t r0, r1;                // what is left of the pair that is cut
    auto take_b = [&](int n, int half, int copy) { fb[half][n / J][n % J] = TB::fragment(lds + copy * COPY + TA::BYTES, wn * J + n % J, n / J); };
    // (fragments alternate from step to step, too: `turn` is a fragment's number in two steps)
    auto take_raw = [&](int turn, int i, int copy) {
        const char* row = lds + copy * COPY + ((wm * I + i) * 16 + j16) * 128;
        raw[turn & 1][0] = *reinterpret_cast<const i32x4*>(row + ((2 * gr) ^ (j16 & 7)) * 16);
        raw[turn & 1][1] = *reinterpret_cast<const i32x4*>(row + ((2 * gr + 1) ^ (j16 & 7)) * 16);
    };
    // part n of 24 of cutting a fragment's values, x = h + m + l: six a pair
    auto cut = [&](int n, int turn) {
        const int pair = n / 6, at = turn & 1;
        i32x4(&p)[3] = piece[at];
        auto round = [&](int which) {
            typedef float f2 __attribute__((ext_vector_type(2)));
            typedef __bf16 b2 __attribute__((ext_vector_type(2)));
            p[which][pair] = __builtin_bit_cast(int32_t, __builtin_convertvector((f2{__uint_as_float(r0), __uint_as_float(r1)}), b2));
        };
        auto left = [](uint32_t& r, uint32_t high) { r = __float_as_uint(__uint_as_float(r) - __uint_as_float(high)); };
        if (n % 6 == 0) {
            r0 = (uint32_t)raw[at][pair / 2][pair % 2 * 2];
            r1 = (uint32_t)raw[at][pair / 2][pair % 2 * 2 + 1];
            round(0);
        }
        if (n % 6 == 1) left(r0, (uint32_t)p[0][pair] << 16);
        if (n % 6 == 2) { left(r1, (uint32_t)p[0][pair] & 0xffff0000u); round(1); }
        if (n % 6 == 3) left(r0, (uint32_t)p[1][pair] << 16);
        if (n % 6 == 4) left(r1, (uint32_t)p[1][pair] & 0xffff0000u);
        if (n % 6 == 5) round(2);
    };
    // (what was cut last is wanted last: a piece is written five products or more before the first that reads it, which a product needs to be two instructions)
    constexpr int PA[6] = {0, 0, 0, 1, 1, 2}, PB[6] = {2, 0, 1, 1, 0, 0};
    auto one = [&](int n, int turn, int i, int half) {
        const int pair = n / J, j = n % J;
        const s16x8 a = __builtin_bit_cast(s16x8, piece[turn & 1][PA[pair]]);
        if (pair == 1) dense_mfma_in_place<__bf16>(big[i][j], fb[half][PB[pair]][j], a);
        else dense_mfma_in_place<__bf16>(acc[i][j], fb[half][PB[pair]][j], a);
        __builtin_amdgcn_sched_barrier(0);
    };
    aim(first);
#pragma unroll
    for (int n = 0; n < REQ; ++n) request(n, 0);
    aim(first + 1);
#pragma unroll
    for (int n = 0; n < REQ; ++n) request(n, 1);
    dense_meet<REQ>();
#pragma unroll
    for (int n = 0; n < 3 * J; ++n) take_b(n, 0, 0);
    take_raw(0, 0, 0);
    take_raw(1, 1, 0);
#pragma unroll
    for (int n = 0; n < 24; ++n) cut(n, 0);
    auto step = [&](auto copy_of, int32_t s) {
        constexpr int now = decltype(copy_of)::value;
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int turn = now * I + i;
            if (i == I - 2) {           // the last fragment of this copy is in registers
                aim(s + 2);
                dense_meet<0>();
            }
#pragma unroll
            for (int n = 0; n < PRODUCTS; ++n) {
                if (n == 0) {               // the fragment after the next one, into the place of the one that has been cut
                    if (i < I - 2) take_raw(turn + 2, i + 2, now);
                    else take_raw(turn + 2, i + 2 - I, now ^ 1);
                }
                cut(n, turn + 1);
                if (i >= I - 2) {
                    const int k = (i - (I - 2)) * PRODUCTS + n;
                    if (k % 4 == 0 && k / 4 < 3 * J) take_b(k / 4, now ^ 1, now ^ 1);
                    if (k % 3 == 1 && k / 3 < REQ) request(k / 3, now);
                }
                one(n, turn, i, now);
            }
        }
    };
    int32_t s = first;
    for (; s + 1 < last; s += 2) {
        step(std::integral_constant<int, 0>{}, s);
        step(std::integral_constant<int, 1>{}, s + 1);
    }
    if (s < last) step(std::integral_constant<int, 0>{}, s);
    dense_settle(acc);
    dense_settle(big);
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j) acc[i][j] += big[i][j];
    dense_meet<0>();
    dense_finish<BM, BN, 2, 2, E>(g, e, 0, tm, tn, M, acc, lds, DenseAgain<true, false, true>{g, first * BK, min(K, last * BK)});
}

// ------------------------------------------------------------------------------------------------------- plans

// Kinds of tiles: sides, blocks of which a compute unit holds at most `per_unit` (by their LDS), and an estimate of their time in microseconds: `start` for each round of blocks, and for each step `one`
// where a compute unit has one block, `more` for each block beside it. Measured with all kinds in turn at sides from 64 to 4096, sums of 256 to 4096, one to eight products; the estimates are
// within 20 % of those times, mostly. bf16, us, large / 128 / 128 deep / 64 / 64 deep / 64 in groups / 32: 4096^3 103 / 128 / 152 / 178 / 198 / 248 / 629; 2048 x 4096 x 2048
// 51 / 36 / 46 / 52 / 58 / 75 / 211; 1024 x 1024 x 4096 78 / 54 / 33 / 37 / 18 / 19 / 41; 256 x 256 x 4096 77 / 38 / 32 / 24 / 17 / 15 / 10.
struct DenseKind { int bm, bn, per_unit; double one, more, start; };
struct DensePlan { int kind, splits; };
enum { DENSE_LARGE, DENSE_192, DENSE_128, DENSE_128_DEEP, DENSE_64, DENSE_64_DEEP, DENSE_64_GROUPS, DENSE_32, DENSE_KINDS };

static const DenseKind DENSE_KIND[3][DENSE_KINDS] = {      // of one, two and three pieces
    {{256, 256, 1, 1.35, 0, 8}, {192, 192, 1, 0.85, 0, 7}, {128, 128, 2, 0.6, 0.35, 5}, {128, 128, 1, 0.5, 0, 5.5}, {64, 64, 5, 0.3, 0.12, 4}, {64, 64, 2, 0.21, 0.13, 3.7}, {64, 64, 1, 0.17, 0, 4.8}, {32, 32, 1, 0.08, 0, 4.8}},
    {{256, 256, 1, 2.1, 0, 8}, {192, 192, 1, 1.3, 0, 7}, {128, 128, 2, 0.95, 0.7, 5}, {128, 128, 1, 0.75, 0, 5}, {64, 64, 5, 0.42, 0.24, 4.5}, {64, 64, 2, 0.27, 0.17, 4}, {64, 64, 1, 0.24, 0, 5}, {32, 32, 1, 0.09, 0, 5.2}},
    {{256, 128, 1, 1.9, 0, 8}, {192, 192, 0, 0, 0, 0}, {128, 128, 1, 1.3, 0, 5}, {128, 128, 0, 0, 0, 0}, {64, 64, 3, 0.75, 0.25, 3}, {64, 64, 1, 0.42, 0, 3}, {64, 64, 0, 0, 0, 0}, {32, 32, 1, 0.25, 0, 3}}};

constexpr int64_t DENSE_TILES_MOST = (1 << 23) - 8;      // a launch's threads, 512 a tile at most, stay below 2^32; the large kind's stay so whatever memory holds

// Numbers of parts of a reduction: 1, 2, 3, 4, 8, ... 64, four steps or more in each.
constexpr int DENSE_PARTS = 64;
static inline int dense_more_parts(int splits) { return splits < 4 ? splits + 1 : splits * 2; }
static inline int64_t dense_steps(int64_t K, int P) { return ceil_div(K < 1 ? 1 : K, dense_bk(P)); }
static inline bool dense_parts_fit(int64_t steps, int splits) { return splits == 1 || steps >= splits * 4; }
static inline size_t dense_parts_bytes(int64_t splits, int64_t M, int64_t N, int64_t matrices) { return splits > 1 ? (size_t)splits * M * wide_of(N) * matrices * 4 : 0; }

// Room for the parts of any plan for a product of these or of smaller sizes. (A plan's own parts do not grow with the sizes: 2276 rows of 2048 x 8192 bf16 are split in three, 2504 are not. A program makes one
// workspace for its largest batch.)
static size_t dense_parts_room(int64_t M, int64_t N, int64_t K, int P, int64_t matrices, size_t parts_most) {
    const int64_t steps = dense_steps(K, P);
    int most = 1;
    while (most < DENSE_PARTS && dense_parts_fit(steps, dense_more_parts(most))) most = dense_more_parts(most);
    const size_t all = dense_parts_bytes(most, M, N, matrices);
    return all < parts_most ? all : parts_most;
}

// The kind of tile and the number of parts of the reduction that promise the shortest time; the parts' sums take at most `parts_most` bytes and a launch that joins them; kinds other than the
// large one need `elsewhere` us before them.
static DensePlan dense_plan(int64_t M, int64_t N, int64_t K, int P, int64_t matrices, bool half, size_t parts_most, double elsewhere = 0) {
    const int64_t steps = dense_steps(K, P);
    DensePlan best{DENSE_64, 1};
    double least = 1e300;
    for (int kind = 0; kind < DENSE_KINDS; ++kind) {
        const DenseKind& k = DENSE_KIND[P - 1][kind];
        if (k.per_unit == 0) continue;
        const int64_t a = ceil_div(M < 1 ? 1 : M, k.bm), b = ceil_div(N, k.bn), tiles = (half ? a * (a + 1) / 2 : a * b) * matrices;
        if (kind != DENSE_LARGE && tiles > DENSE_TILES_MOST) continue;
        for (int splits = 1; splits <= DENSE_PARTS; splits = dense_more_parts(splits)) {
            if (!dense_parts_fit(steps, splits) || dense_parts_bytes(splits, M, N, matrices) > parts_most) break;
            const int64_t units = ceil_div(tiles * splits, 256), rounds = ceil_div(units, k.per_unit);
            double t = (double)rounds * ((double)ceil_div(steps, splits) * (k.one + k.more * (double)((rounds > 1 ? k.per_unit : units) - 1)) + k.start);
            if (splits > 1) t += 5.0 + (double)splits * M * N * matrices * 8 / 3.5e6;
            if (kind != DENSE_LARGE) t += elsewhere;
            if (t < least) { least = t; best = DensePlan{kind, splits}; }
        }
    }
    return best;
}

// Tiles of 224 rows where they need fewer rows' time in all (24922 x 602 x 256: 224 blocks for 256 units instead of 196, 58 us for 64).
template <typename E>
static void dense_raw_launch(DenseRawArgs a, const typename E::Args& e, int splits, hipStream_t st) {
    a.g.splits = splits;
    a.g.matrices = 1;
    a.g.tiles_n = (int32_t)ceil_div(a.g.N, 128);
    auto rounds = [&](int64_t rows) { return ceil_div(ceil_div(a.g.M, rows) * a.g.tiles_n * splits, 256); };
    const bool low = rounds(224) * 224 < rounds(256) * 256;
    a.g.tiles_m = (int32_t)ceil_div(a.g.M, low ? 224 : 256);
    const dim3 grid((unsigned)(ceil_div(dense_tiles(a.g.tiles_m, a.g.tiles_n, false), 8) * 8), (unsigned)splits);
    if (low) hipLaunchKernelGGL((dense_raw_kernel<224, E>), grid, dim3(256), 0, st, a, e);
    else hipLaunchKernelGGL((dense_raw_kernel<256, E>), grid, dim3(256), 0, st, a, e);
}

template <typename H, int P, bool AL, bool BL, typename E>
static void dense_launch(DenseArgs g, const typename E::Args& e, const DensePlan& p, int64_t matrices, hipStream_t st) {
    const DenseKind& k = DENSE_KIND[P - 1][p.kind];
    g.splits = p.splits;
    g.tiles_m = (int32_t)ceil_div(g.M, k.bm);
    g.tiles_n = (int32_t)ceil_div(g.N, k.bn);
    g.matrices = (int32_t)matrices;
    const dim3 grid((unsigned)(ceil_div(dense_tiles(g.tiles_m, g.tiles_n, E::MIRROR) * matrices, 8) * 8), (unsigned)p.splits);
#define NO_DENSE(BM, BN, WM, WN, STAGES, GROUPS) hipLaunchKernelGGL((dense_kernel<H, P, AL, BL, BM, BN, WM, WN, STAGES, GROUPS, E>), grid, dim3(64 * WM * WN * GROUPS), 0, st, g, e)
    switch (p.kind) {
        case DENSE_LARGE:
            hipLaunchKernelGGL((dense_large_kernel<H, P, AL, BL, 256, (P < 3 ? 256 : 128), E>), grid, dim3(256), 0, st, g, e);
            break;
        case DENSE_192:
            if constexpr (P < 3) hipLaunchKernelGGL((dense_large_kernel<H, P, AL, BL, 192, 192, E>), grid, dim3(256), 0, st, g, e);
            break;
        case DENSE_128: NO_DENSE(128, 128, 2, 2, P < 3 ? 2 : 3, 1); break;
        case DENSE_128_DEEP:
            if constexpr (P < 3) NO_DENSE(128, 128, 2, 2, 4, 1);
            break;
        case DENSE_64: NO_DENSE(64, 64, 2, 2, 2, 1); break;
        case DENSE_64_DEEP: NO_DENSE(64, 64, 2, 2, 4, 1); break;
        case DENSE_64_GROUPS:
            if constexpr (P < 3) NO_DENSE(64, 64, 2, 2, 4, 2);
            break;
        default: NO_DENSE(32, 32, 1, 1, P < 3 ? 4 : 3, 4); break;
    }
#undef NO_DENSE
}

}  // namespace no
