// no_linear_fwd / no_linear_bwd: rows times a matrix, with bias, activation and residual, and the gradients.
#include "dense.hpp"

namespace no {

// The share of the standard normal distribution below z, and e = exp(-z^2 / 2): with x = |z| / sqrt(2), erfc(x) = e t Q(t), t = 1 / (1 + 0.44 x), Q a polynomial of degree 7 fitted to exp(x^2) erfc(x)
// (1 + 0.44 x) over [0, 10] with least relative error (1.8e-7; with the roundings of its evaluation 7e-7 up to |z| = 3, then by the exponent's, 1.4e-6 at 5, 2.2e-6 at 6, 8e-6 at 13, of a share that 1 + erf has lost by then).
// 17 instructions for share and slope together, where erff and expf are 60: the GELU gradient of 8192 x 8192
// bf16 was bound by them.
__device__ __forceinline__ float normal_share(float z, float& e) {
    const float t = __builtin_amdgcn_rcpf(1.0f + 0.44f * 0.70710678f * fabsf(z));
    e = __builtin_amdgcn_exp2f(-0.72134752f * z * z);
    float q = 0.0712223426f;
    q = q * t - 0.277943522f;
    q = q * t + 0.296680063f;
    q = q * t - 0.0201741587f;
    q = q * t + 0.215808973f;
    q = q * t + 0.217314482f;
    q = q * t + 0.248871043f;
    q = q * t + 0.248220965f;
    const float half = 0.5f * t * q * e;
    return z > 0.0f ? 1.0f - half : half;
}
__device__ __forceinline__ float logistic(float z) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504f * z)); }

template <int ACT> __device__ __forceinline__ float act_of(float z) {
    if (ACT == NO_ACT_RELU) return z > 0.0f ? z : z != z ? z : 0.0f;
    if (ACT == NO_ACT_GELU) {
        float e;
        return z * normal_share(z, e);
    }
    if (ACT == NO_ACT_SILU) return z * logistic(z);
    return z;
}
// derivative of the activation
template <int ACT> __device__ __forceinline__ float slope_of(float z) {
    if (ACT == NO_ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
    if (ACT == NO_ACT_GELU) {
        float e;
        const float share = normal_share(z, e);
        return share + z * e * 0.39894228f;
    }
    if (ACT == NO_ACT_SILU) {
        const float p = logistic(z);
        return p * (1.0f + z * (1.0f - p));
    }
    return 1.0f;
}

// What follows the sums of the forward pass: z = sum + bias, y = act(z) + residual.
struct LinearEnd {
    const float* bias;
    RowsOf residual, z, y;
    int32_t act;
};

template <typename T, int W>
__device__ __forceinline__ Run<T, W> linear_ahead(const LinearEnd& e, int64_t m, int32_t n, int32_t here) {
    Run<T, W> r;
    if (e.residual.p) r.load(e.residual.row<T>(m) + n, here, from_f32<T>(0.0f));
    return r;
}
template <int ACT, int W>
__device__ __forceinline__ void activate(float (&v)[W]) {
#pragma unroll
    for (int w = 0; w < W; ++w) v[w] = act_of<ACT>(v[w]);
}
template <typename T, int W>
__device__ __forceinline__ void linear_end(const LinearEnd& e, int64_t m, int32_t n, int32_t here, float (&v)[W], const Run<T, W>& residual) {
    if (e.bias) {
        Run<float, W> b;
        float f[W];
        b.load(e.bias + n, here, 0.0f);
        b.get(f);
#pragma unroll
        for (int w = 0; w < W; ++w) v[w] += f[w];
    }
    Run<T, W> o;
    if (e.z.p) {
        o.set(v);
        o.store(e.z.row<T>(m) + n, here);
    }
    if (e.act == NO_ACT_RELU) activate<NO_ACT_RELU>(v);
    else if (e.act == NO_ACT_GELU) activate<NO_ACT_GELU>(v);
    else if (e.act == NO_ACT_SILU) activate<NO_ACT_SILU>(v);
    if (e.residual.p) {
        float f[W];
        residual.get(f);
#pragma unroll
        for (int w = 0; w < W; ++w) v[w] += f[w];
    }
    o.set(v);
    o.store(e.y.row<T>(m) + n, here);
}

template <typename T>
struct LinearOut {
    struct Args { LinearEnd end; float* parts; int32_t pitch; };      // parts: sums of a split reduction instead, [split][M][pitch], pitch a multiple of 8: every run is whole
    static constexpr bool MIRROR = false;
    typedef Run<T, 8> Ahead;
    __device__ static __forceinline__ Ahead ahead(const Args& e, int32_t, int32_t m, int32_t n, int32_t here) { return linear_ahead<T, 8>(e.end, m, n, here); }
    __device__ static __forceinline__ void put(const Args& e, int32_t, int32_t m, int32_t n, int32_t here, float (&v)[8], const Ahead& residual, int32_t M) {
        if (e.parts) {
            Run<float, 8> o;
            o.set(v);
            o.store(e.parts + ((int64_t)blockIdx.y * M + m) * e.pitch + n);
        } else linear_end<T, 8>(e.end, m, n, here, v, residual);
    }
};

// Column sums of gz from their parts: sixteen columns a block, sixteen threads to a column.
struct BiasJob {
    const float* parts;
    int32_t n_parts, dim;
    float* grad_bias;
};
__device__ __forceinline__ void bias_block(const BiasJob& j, int32_t block) {
    __shared__ float share[16][17];
    const int32_t col = (int32_t)threadIdx.x & 15, row = (int32_t)threadIdx.x >> 4, c = block * 16 + col;
    float sum = 0.0f;
    if (c < j.dim)
#pragma unroll 4
        for (int32_t p = row; p < j.n_parts; p += 16) sum += j.parts[(int64_t)p * j.dim + c];
    share[row][col] = sum;
    __syncthreads();
    if (row > 0 || c >= j.dim) return;
    sum = 0.0f;
#pragma unroll
    for (int k = 0; k < 16; ++k) sum += share[k][col];
    j.grad_bias[c] = sum;
}
__global__ void __launch_bounds__(256) linear_bias_kernel(BiasJob j) { bias_block(j, (int32_t)blockIdx.x); }

// The parts of a split reduction added up (the launch's other blocks: column sums), four columns a thread; LANES > 1: that many threads to a place, each with every LANES-th part, whose sums are added in order.
template <typename T, int LANES>
__global__ void __launch_bounds__(256) linear_join_kernel(const float* __restrict__ parts, int32_t splits, int32_t M, const int32_t* d_M, int32_t N, LinearEnd e, int32_t blocks, BiasJob bias) {
    constexpr int PLACES = 256 / LANES;
    if ((int32_t)blockIdx.x >= blocks) return bias_block(bias, (int32_t)blockIdx.x - blocks);
    __shared__ float share[LANES][PLACES][4];
    const int place = (int)threadIdx.x % PLACES, lane = (int)threadIdx.x / PLACES;
    const int64_t per_row = ceil_div(N, 4), i = (int64_t)blockIdx.x * PLACES + place, m = i / per_row;
    const bool there = m < rows_here(d_M, M);
    const int32_t n = (int32_t)(i - m * per_row) * 4, here = min(4, N - n);
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (there) {
        const int32_t pitch = (N + 7) / 8 * 8;
        const float* from = parts + m * pitch + n;
        const int64_t stride = (int64_t)M * pitch;
#pragma unroll 4
        for (int32_t s = lane; s < splits; s += LANES) {
            Run<float, 4> r;
            float f[4];
            r.load(from + s * stride);
            r.get(f);
#pragma unroll
            for (int w = 0; w < 4; ++w) v[w] += f[w];
        }
    }
    if constexpr (LANES > 1) {
#pragma unroll
        for (int w = 0; w < 4; ++w) share[lane][place][w] = v[w];
        __syncthreads();
        if (lane > 0) return;
#pragma unroll
        for (int k = 1; k < LANES; ++k)
#pragma unroll
            for (int w = 0; w < 4; ++w) v[w] += share[k][place][w];
    }
    if (there) linear_end<T, 4>(e, m, n, here, v, linear_ahead<T, 4>(e, m, n, here));
}
template <typename T>
static void linear_join(const float* parts, int32_t splits, int32_t M, const int32_t* d_M, int32_t N, const LinearEnd& end, const BiasJob& bias, hipStream_t st) {
    const int64_t places = (int64_t)M * ceil_div(N, 4), more = bias.grad_bias ? ceil_div(bias.dim, 16) : 0;
    const bool few = splits >= 8 && places <= 65536;
    const int64_t blocks = ceil_div(places, few ? 16 : 256);
    if (few) hipLaunchKernelGGL((linear_join_kernel<T, 16>), dim3((unsigned)(blocks + more)), dim3(256), 0, st, parts, splits, M, d_M, N, end, (int32_t)blocks, bias);
    else hipLaunchKernelGGL((linear_join_kernel<T, 1>), dim3((unsigned)(blocks + more)), dim3(256), 0, st, parts, splits, M, d_M, N, end, (int32_t)blocks, bias);
}

// ------------------------------------------------------------------------------------------------------- operands
//
// A product takes rows of whole 16 bytes. bf16 rows that are none are copied into rows of a multiple of 8 values, zeros at the end; fp32 rows are cut into three bf16 planes whose sum is
// the value, x = h + m + l, rounded each time to the nearest (8 bits each, so nothing of the 24 is left over while the pieces are in range; the first one is held to the largest bf16).
__device__ __forceinline__ void dense_cut(float x, float& h, float& m, float& l) {
    constexpr float TOP = 0x1.fep127f;
    const bool fine = fabsf(x) < INFINITY;      // (an infinity or NaN is all in the first piece)
    h = to_f32(from_f32<bf16_t>(fine ? __builtin_amdgcn_fmed3f(x, -TOP, TOP) : x));
    m = fine ? to_f32(from_f32<bf16_t>(x - h)) : 0.0f;
    l = fine ? x - h - m : 0.0f;
}

template <typename T>
__device__ __forceinline__ void dense_put(const float (&f)[8], char* to, int32_t plane) {
    Run<bf16_t, 8> o;
    if constexpr (sizeof(T) == 2) {
        o.set(f);
        o.store(reinterpret_cast<bf16_t*>(to));
    } else {
        float p[3][8];
#pragma unroll
        for (int w = 0; w < 8; ++w) dense_cut(f[w], p[0][w], p[1][w], p[2][w]);
#pragma unroll
        for (int q = 0; q < 3; ++q) {
            o.set(p[q]);
            o.store(reinterpret_cast<bf16_t*>(to + q * plane));
        }
    }
}

struct PackJob {
    RowsOf x;
    const int32_t* d_n;
    int32_t cap, dim;
    char* out;              // NULL: nothing to do
    int64_t pitch;
    int32_t plane, blocks;      // plane 0: up to 32 fp32 columns as they are, zeros behind them
};
template <typename T>
__device__ __forceinline__ void pack_block(const PackJob& j, int32_t block) {
    if (sizeof(T) == 4 && j.plane == 0) {
        const int32_t n = rows_here(j.d_n, j.cap);
        for (int64_t i = (int64_t)block * 256 + threadIdx.x; i < (int64_t)n * 8; i += (int64_t)j.blocks * 256) {
            const int32_t c = (int32_t)(i & 7) * 4;
            const float* from = j.x.row<float>(i >> 3);
            f32x4 v;
#pragma unroll
            for (int w = 0; w < 4; ++w) v[w] = c + w < j.dim ? from[c + w] : 0.0f;
            *reinterpret_cast<f32x4*>(j.out + (i >> 3) * 128 + c * 4) = v;
        }
        return;
    }
    const int32_t units = (j.dim + 7) / 8, n = rows_here(j.d_n, j.cap);
    for (int64_t i = (int64_t)block * 256 + threadIdx.x; i < (int64_t)n * units; i += (int64_t)j.blocks * 256) {
        const int64_t r = i / units;
        const int32_t c = (int32_t)(i - r * units) * 8;
        Run<T, 8> v;
        float f[8];
        v.load_at(j.x.row<T>(r), c, j.dim, from_f32<T>(0.0f));
        v.get(f);
        dense_put<T>(f, j.out + r * j.pitch + c * 2, j.plane);
    }
}
template <typename T>
__global__ void __launch_bounds__(256) linear_pack_kernel(PackJob a, PackJob b) {
    if ((int32_t)blockIdx.x < a.blocks) pack_block<T>(a, (int32_t)blockIdx.x);
    else pack_block<T>(b, (int32_t)blockIdx.x - a.blocks);
}

// The gradient of the pre-activation, gz = grad_y act'(z), laid out as an operand (gz NULL: grad_y is one as it stands), and its column sums over `per` rows a block: LANES threads along a
// row, each with eight columns, and 256 / LANES rows at a time, whose sums are added in order; four of a thread's rows are requested at once.
// The launch's other blocks lay out the rows of x and the matrix for the products behind it.
// Of bf16 values gz is rounded to bf16 (a smooth slope's product by 2^-8 of it at most, relu's and none's not at all): the products then take 16-bit operands, at six times the rate of pieces, and the gradients' error over all
// is 0.0023 where their own rounding leaves 0.0017 (two pieces of gz would take both products, 400 us of 8192 x 2048 x 8192's 460, twice). The column sums take it unrounded. Bound by memory: 8192 x 8192 bf16 gelu 75 us (403 MB, 5.4 TB/s).
template <typename T, int ACT, int LANES>
__global__ void __launch_bounds__(256) linear_gz_kernel(RowsOf grad_y, RowsOf z, const int32_t* d_n, int32_t cap, int32_t dim, int32_t per, int32_t wide, int32_t blocks, char* gz,
                                                        int64_t pitch, int32_t plane, float* parts, PackJob a, PackJob b) {
    constexpr int LINES = 256 / LANES, AHEAD = 4;
    __shared__ float share[LINES][LANES * 8 + 4];
    if ((int32_t)blockIdx.x >= blocks) {
        const int32_t k = (int32_t)blockIdx.x - blocks;
        if (k < a.blocks) pack_block<T>(a, k);
        else pack_block<T>(b, k - a.blocks);
        return;
    }
    const int32_t bx = (int32_t)blockIdx.x % wide, by = (int32_t)blockIdx.x / wide;
    const int32_t n = rows_here(d_n, cap), lane = (int32_t)threadIdx.x % LANES, line = (int32_t)threadIdx.x / LANES, c = (bx * LANES + lane) * 8;
    const int64_t first = (int64_t)by * per, last = first + per < n ? first + per : n;
    float sum[8] = {};
    if (c < dim) {
        for (int64_t r0 = first + line; r0 < last; r0 += AHEAD * LINES) {
            Run<T, 8> v[AHEAD], u[AHEAD];
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) {
                const int64_t r = r0 + a * LINES < last ? r0 + a * LINES : r0;
                v[a].load_at(grad_y.row<T>(r), c, dim, from_f32<T>(0.0f));
                if (ACT != NO_ACT_NONE) u[a].load_at(z.row<T>(r), c, dim, from_f32<T>(0.0f));
            }
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) {
                const int64_t r = r0 + a * LINES;
                if (r >= last) break;
                float f[8], s[8];
                v[a].get(f);
                if (ACT != NO_ACT_NONE) {
                    u[a].get(s);
#pragma unroll
                    for (int w = 0; w < 8; ++w) f[w] *= slope_of<ACT>(s[w]);
                }
                if (gz) dense_put<T>(f, gz + r * pitch + c * 2, plane);
#pragma unroll
                for (int w = 0; w < 8; ++w) sum[w] += f[w];
            }
        }
    }
    if (!parts) return;
#pragma unroll
    for (int w = 0; w < 8; ++w) share[line][lane * 8 + w] = sum[w];
    __syncthreads();
    const int32_t at = bx * LANES * 8 + (int32_t)threadIdx.x;
    if ((int32_t)threadIdx.x >= LANES * 8 || at >= dim) return;
    float total = 0.0f;
#pragma unroll
    for (int k = 0; k < LINES; ++k) total += share[k][threadIdx.x];
    parts[(int64_t)by * dim + at] = total;
}

// ------------------------------------------------------------------------------------------------------- few rows
//
// Up to LINEAR_FEW rows of fp32, or with a bf16 matrix that a product cannot take as it is: the matrix would be copied for a single use, so it is read once, in its own order, and multiplied in
// fp32. A thread has 16 bytes of columns and every 64th row of the block's share of the reduction, for all of the rows at once; rows of x stand in LDS as fp32. (One row by a matrix of 2048 x 8192 bf16 that
// begins 2 bytes off 16: 22.9 us, by tiles of 32 x 32 where it does not 10.1, eight rows 31.6 and 10.2; fp32, one row 15.3, eight of 2048 x 2048 17.6, of 8192 x 2048 24.2, where copy and tiles of nine rows take 50.5.)
constexpr int LINEAR_FEW = 8, LINEAR_FEW_K = 1024;      // rows; reduction indices in LDS at a time

template <typename T, int MR, bool SHORT>
__global__ void __launch_bounds__(512) linear_few_kernel(RowsOf x, RowsOf w, const int32_t* d_n, int32_t cap, int32_t K, int32_t N, int32_t splits, LinearEnd e, float* parts) {
    constexpr int W = 16 / (int)sizeof(T), LANES = 8, LINES = 512 / LANES, AHEAD = MR <= 2 ? 16 : 8;      // rows of the matrix requested at once
    __shared__ __attribute__((aligned(16))) float xs[LINEAR_FEW_K * MR];
    __shared__ float share[8][MR][LANES * W];
    const int32_t n = rows_here(d_n, cap);
    const int lane = (int)threadIdx.x & (LANES - 1), line = (int)threadIdx.x / LANES;
    const int32_t c0 = (int32_t)blockIdx.x * LANES * W, c = c0 + lane * W;
    // (a run that would leave the row begins W before its end: requests are whole and nothing branches around them)
    const Place<W, SHORT> place(c < N ? c : 0, N);
    const int32_t k0 = (int32_t)((int64_t)K * blockIdx.y / splits), k1 = (int32_t)((int64_t)K * (blockIdx.y + 1) / splits);
    float acc[MR][W] = {};
    for (int32_t kb = k0; kb < k1; kb += LINEAR_FEW_K) {
        const int32_t here = min(LINEAR_FEW_K, k1 - kb);
        __syncthreads();
        for (int32_t i = (int32_t)threadIdx.x; i < here * MR; i += 512) {
            const int32_t r = i / here, k = i - r * here;
            xs[k * MR + r] = r < n ? to_f32(x.row<T>(r)[kb + k]) : 0.0f;
        }
        __syncthreads();
        for (int32_t k = line; k < here; k += AHEAD * LINES) {
            Run<T, W> v[AHEAD];
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) place.load(v[a], w.row<T>(kb + min(k + a * LINES, here - 1)));
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) {
                float f[W];
                v[a].get(f);
                const int32_t at = k + a * LINES;
                if (at < here) {
#pragma unroll
                    for (int r = 0; r < MR; ++r)
#pragma unroll
                        for (int j = 0; j < W; ++j) acc[r][j] += xs[at * MR + r] * f[j];
                }
            }
        }
    }
    // eight lines of a wavefront, then its eight wavefronts
#pragma unroll
    for (int r = 0; r < MR; ++r)
#pragma unroll
        for (int j = 0; j < W; ++j) {
            float s = acc[r][j];
#pragma unroll
            for (int o = LANES; o < 64; o <<= 1) s += __shfl_xor(s, o, 64);
            const int32_t col = place.at + j - c0;
            if (lane_id() < LANES && c < N && col >= 0) share[threadIdx.x >> 6][r][col] = s;      // (two lanes at a row's end may hold a column, with the same sum)
        }
    __syncthreads();
    constexpr int UNITS = LANES * W / 4;
    const int r = (int)threadIdx.x / UNITS, u = (int)threadIdx.x % UNITS;
    const int32_t col = c0 + u * 4;
    if (r >= MR || r >= n || col >= N) return;
    float v[4] = {};
#pragma unroll
    for (int s = 0; s < 8; ++s)
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] += share[s][r][u * 4 + j];
    const int32_t here = min(4, N - col);
    if (parts) {
        Run<float, 4> o;
        o.set(v);
        o.store(parts + ((int64_t)blockIdx.y * cap + r) * ((N + 7) / 8 * 8) + col);
    } else linear_end<T, 4>(e, r, col, here, v, linear_ahead<T, 4>(e, r, col, here));
}

// ------------------------------------------------------------------------------------------------------- plans

constexpr size_t LINEAR_PARTS_MOST = (size_t)128 << 20;      // bytes of parts, at most

static DensePlan linear_plan(int64_t M, int64_t N, int64_t K, int P, double elsewhere = 0) { return dense_plan(M, N, K, P, 1, false, LINEAR_PARTS_MOST, elsewhere); }
// Parts of the reduction: blocks with 128 KB of the matrix each, but where two parts would do so for few rows, whose join costs what it saves. us by 1 / 2 / 4 / 8 / 16 parts, of matrices that begin on 16 bytes: one bf16 row, 8192
// columns, K = 2048 11.2 / 11.9 / 11.6 / 13.9; 2048 columns, K = 8192 31.6 / 20.7 / 13.6 / 11.7 / 11.5; 4096 x 4096 16.8 / 13.9 / 11.9 / 11.5 / 13.8; eight rows, 8192 columns, K = 2048 29.6 / 24.3 / 31.7;
// 2048 columns, K = 8192 88 / 54 / 33 / 24 / 32. Half of the columns a block (64 bytes of a row, not 128): 15.1 for 11.2, 33 for 30.
static int linear_few_splits(int64_t K, int64_t N, int64_t rows, int es) {
    const int64_t most = K / 128 < 1 ? 1 : K / 128, bytes = K * (N < 128 / es ? N : 128 / es) * es;
    int splits = 1;
    while (splits < 32 && splits * 2 <= most && bytes > splits * (128 << 10)) splits *= 2;
    return splits == 2 && rows < 4 ? 1 : splits;
}
// The forward product: fp32 rows of 32 values or more, whose tile's offsets stay in 31 bits, are cut inside the large kind's product, those of other kinds by a pass before it that reads 4 and writes
// 6 bytes a value, 8 TB/s between the caches and 5 us less than it says, which short sums do not get back (us with the pass and another kind / cut inside: 2000 x 4100 x 300 72 / 56;
// 40001 x 64 x 250 34 / 38, 70000 x 127 x 130 54 / 70; with the pass and the same kind / cut inside: 24922 x 602 x 256 87 / 63).
constexpr int32_t LINEAR_RAW_LEAST = 32;
constexpr int64_t LINEAR_RAW_STRIDE = (int64_t)1 << 22;
static DensePlan linear_plan_fwd(int64_t M, int64_t N, int64_t K, int P) {
    const double pass = P == 3 && K >= LINEAR_RAW_LEAST ? (double)M * K * 10 / 8e6 - 5.0 : 0.0;
    return linear_plan(M, N, K, P, pass > 0 ? pass : 0.0);
}
static size_t linear_parts_room(int64_t M, int64_t N, int64_t K, int P) { return dense_parts_room(M, N, K, P, 1, LINEAR_PARTS_MOST); }

static inline int planes_of_type(no_dtype dt) { return dt == NO_F32 ? 3 : 1; }
static inline size_t operand_bytes(no_dtype dt, int64_t rows, int64_t dim) { return round_256((size_t)rows * wide_of(dim) * 2 * planes_of_type(dt)); }

constexpr int32_t LINEAR_GZ_ROWS = 64;      // rows a block of linear_gz_kernel, at least
static inline int64_t gz_blocks(int64_t n) {
    const int64_t b = ceil_div(n, LINEAR_GZ_ROWS);
    return b < 1 ? 1 : b < 512 ? b : 512;
}

struct LinearRoom { char* p; char* take(size_t b) { char* r = p; p += round_256(b); return r; } };

// bf16 rows of whole, aligned 16 bytes (and not so far apart that a tile's offsets leave 31 bits).
template <typename T>
static bool taken_as_it_is(const RowsOf& x, int32_t dim) {
    return sizeof(T) == 2 && (uintptr_t)x.p % 16 == 0 && x.stride % 16 == 0 && dim % 8 == 0 && x.stride <= (int64_t)1 << 22;
}

// The operand that holds `rows` rows of `dim` values: the matrix itself where a product can take it, else a copy (fp32: pieces) that `job` makes.
template <typename T>
static DenseOperand linear_operand(RowsOf x, const int32_t* d_n, int64_t rows, int32_t dim, LinearRoom& room, PackJob& job) {
    job = PackJob{x, d_n, (int32_t)rows, dim, nullptr, 0, 0, 0};
    if (taken_as_it_is<T>(x, dim)) return DenseOperand{x.p, x.stride, 0, 0, 0};
    job.plane = (int32_t)wide_of(dim) * 2;
    job.pitch = (int64_t)job.plane * planes_of_type(TypeOf<T>::code);
    job.out = room.take(operand_bytes(TypeOf<T>::code, rows, dim));
    const int64_t blocks = ceil_div(rows * ((dim + 7) / 8), 256);
    job.blocks = (int32_t)(blocks < 8192 ? blocks : 8192);
    return DenseOperand{job.out, job.pitch, 0, job.plane, 0};
}
template <typename T>
static void linear_pack(const PackJob& a, const PackJob& b, hipStream_t st) {
    if (a.blocks + b.blocks > 0) hipLaunchKernelGGL(linear_pack_kernel<T>, dim3((unsigned)(a.blocks + b.blocks)), dim3(256), 0, st, a, b);
}

template <typename T, bool AL, bool BL>
static bool linear_product(DenseArgs g, const DensePlan& p, const LinearEnd& end, float* parts, const BiasJob& bias, hipStream_t st) {
    constexpr int P = sizeof(T) == 4 ? 3 : 1;
    const typename LinearOut<T>::Args e{p.splits > 1 ? LinearEnd{} : end, p.splits > 1 ? parts : nullptr, (int32_t)wide_of(g.N)};
    dense_launch<__bf16, P, AL, BL, LinearOut<T>>(g, e, p, 1, st);
    if (p.splits > 1) linear_join<T>(parts, p.splits, g.M, g.d_M, g.N, end, bias, st);
    return p.splits > 1;        // (the column sums went along)
}

template <typename T>
static void linear_fwd(RowsOf x, RowsOf w, const int32_t* d_n, int32_t cap, int32_t d_in, int32_t d_out, const LinearEnd& end, char* ws, hipStream_t st) {
    LinearRoom room{ws};
    if (cap <= LINEAR_FEW && !taken_as_it_is<T>(w, d_out)) {
        const int splits = linear_few_splits(d_in, d_out, cap, sizeof(T));
        float* parts = splits > 1 ? (float*)ws : nullptr;
        const dim3 grid((unsigned)ceil_div(d_out, 128 / (int)sizeof(T)), (unsigned)splits);
#define NO_FEW_AS(MR, SHORT) hipLaunchKernelGGL((linear_few_kernel<T, MR, SHORT>), grid, dim3(512), 0, st, x, w, d_n, cap, d_in, d_out, splits, end, parts)
#define NO_FEW(MR) do { if (d_out < 16 / (int)sizeof(T)) NO_FEW_AS(MR, true); else NO_FEW_AS(MR, false); } while (0)
        if (cap <= 1) NO_FEW(1);
        else if (cap <= 2) NO_FEW(2);
        else if (cap <= 4) NO_FEW(4);
        else NO_FEW(8);
#undef NO_FEW
#undef NO_FEW_AS
        if (splits > 1) linear_join<T>(parts, splits, cap, d_n, d_out, end, BiasJob{}, st);
        return;
    }
    DenseArgs g{};
    PackJob jx, jw;
    g.M = cap; g.N = d_out; g.K = d_in;
    g.d_M = d_n;
    const DensePlan plan = linear_plan_fwd(cap, d_out, d_in, planes_of_type(TypeOf<T>::code));
    if constexpr (sizeof(T) == 4) {
        if (plan.kind == DENSE_LARGE && d_in >= LINEAR_RAW_LEAST && x.stride <= LINEAR_RAW_STRIDE) {        // rows are read where they are, but for the columns that fill no step
            const int32_t rest = d_in % 32;
            const int64_t blocks = rest ? ceil_div((int64_t)cap * 8, 256) : 0;
            char* tail = room.take((size_t)cap * 128);
            jx = PackJob{RowsOf{x.p + (int64_t)(d_in - rest) * 4, x.stride}, d_n, cap, rest, tail, 128, 0, (int32_t)(blocks < 2048 ? blocks : 2048)};
            g.a = DenseOperand{x.p, x.stride, 0, 0, cap};
            g.b = linear_operand<T>(w, nullptr, d_in, d_out, room, jw);
            g.b.extent = (int32_t)wide_of(d_out);
            linear_pack<T>(jx, jw, st);
            float* parts = plan.splits > 1 ? (float*)room.p : nullptr;
            dense_raw_launch<LinearOut<T>>(DenseRawArgs{g, DenseOperand{tail, 128, 0, 0, cap}}, typename LinearOut<T>::Args{parts ? LinearEnd{} : end, parts, (int32_t)wide_of(d_out)}, plan.splits, st);
            if (parts) linear_join<T>(parts, plan.splits, cap, d_n, d_out, end, BiasJob{}, st);
            return;
        }
    }
    g.a = linear_operand<T>(x, d_n, cap, d_in, room, jx);
    g.b = linear_operand<T>(w, nullptr, d_in, d_out, room, jw);
    linear_pack<T>(jx, jw, st);
    g.a.extent = cap;
    g.b.extent = (int32_t)wide_of(d_out);
    linear_product<T, true, false>(g, plan, end, (float*)room.p, BiasJob{}, st);
}

template <typename T>
static void linear_bwd(RowsOf x, RowsOf w, int32_t act, RowsOf z, RowsOf grad_y, const int32_t* d_n, int32_t cap, int32_t d_in, int32_t d_out, RowsOf grad_x, RowsOf grad_w,
                       float* grad_bias, char* ws, hipStream_t st) {
    LinearRoom room{ws};
    const bool products = grad_x.p || grad_w.p;
    const bool as_is = act == NO_ACT_NONE && taken_as_it_is<T>(grad_y, d_out);
    DenseOperand gz{grad_y.p, grad_y.stride, 0, 0, 0};
    char* to = nullptr;
    if (products && !as_is) {
        to = room.take(operand_bytes(TypeOf<T>::code, cap, d_out));
        gz = DenseOperand{to, wide_of(d_out) * 2 * planes_of_type(TypeOf<T>::code), 0, (int32_t)wide_of(d_out) * 2, 0};
    }
    const int64_t blocks = gz_blocks(cap), lanes = d_out <= 64 ? 8 : 32, wide = ceil_div(d_out, lanes * 8);
    float* sums = (float*)room.take(blocks * d_out * 4);
    PackJob jw{}, jx{};
    DenseOperand ow{}, ox{};
    if (grad_x.p && cap > 0) ow = linear_operand<T>(w, nullptr, d_in, d_out, room, jw);
    if (grad_w.p) ox = linear_operand<T>(x, d_n, cap, d_in, room, jx);
    BiasJob bias{sums, (int32_t)blocks, d_out, blocks > 1 ? grad_bias : nullptr};
    if (to || grad_bias) {
        const int32_t per = (int32_t)ceil_div(cap, blocks);
        float* parts = grad_bias ? (blocks == 1 ? grad_bias : sums) : nullptr;
#define NO_GZ_AS(ACT, LANES)                                                                                                                                                           \
    hipLaunchKernelGGL((linear_gz_kernel<T, ACT, LANES>), dim3((unsigned)(wide * blocks + jw.blocks + jx.blocks)), dim3(256), 0, st, grad_y, z, d_n, cap, d_out, per, (int32_t)wide,   \
                       (int32_t)(wide * blocks), to, gz.pitch, gz.plane, parts, jw, jx)
#define NO_GZ(ACT) do { if (lanes == 8) NO_GZ_AS(ACT, 8); else NO_GZ_AS(ACT, 32); } while (0)
        if (act == NO_ACT_RELU) NO_GZ(NO_ACT_RELU);
        else if (act == NO_ACT_GELU) NO_GZ(NO_ACT_GELU);
        else if (act == NO_ACT_SILU) NO_GZ(NO_ACT_SILU);
        else NO_GZ(NO_ACT_NONE);
#undef NO_GZ
#undef NO_GZ_AS
    } else linear_pack<T>(jw, jx, st);
    auto joined = [&](bool went) { if (went) bias.grad_bias = nullptr; };
    if (grad_x.p && cap > 0) {
        DenseArgs g{};
        g.a = gz; g.b = ow;
        g.a.extent = cap;
        g.b.extent = d_in;
        g.M = cap; g.N = d_in; g.K = d_out;
        g.d_M = d_n;
        joined(linear_product<T, true, true>(g, linear_plan(g.M, g.N, g.K, planes_of_type(TypeOf<T>::code)), LinearEnd{nullptr, {nullptr, 0}, {nullptr, 0}, grad_x, NO_ACT_NONE}, (float*)room.p, bias, st));
    }
    if (grad_w.p) {
        DenseArgs g{};
        g.a = ox; g.b = gz;
        g.a.extent = (int32_t)wide_of(d_in);
        g.b.extent = (int32_t)wide_of(d_out);
        g.M = d_in; g.N = d_out; g.K = cap;
        g.d_K = d_n;
        joined(linear_product<T, false, false>(g, linear_plan(g.M, g.N, g.K, planes_of_type(TypeOf<T>::code)), LinearEnd{nullptr, {nullptr, 0}, {nullptr, 0}, grad_w, NO_ACT_NONE}, (float*)room.p, bias, st));
    }
    if (bias.grad_bias) hipLaunchKernelGGL(linear_bias_kernel, dim3((unsigned)ceil_div(d_out, 16)), dim3(256), 0, st, bias);
}

static int32_t linear_sizes(const char* who, no_dtype dt, int32_t act, int32_t cap, int32_t d_in, int32_t d_out) {
    NO_REQUIRE(dt == NO_F32 || dt == NO_BF16, NO_ERR_INVALID_ARG, "%s: values are NO_F32 or NO_BF16", who);
    NO_REQUIRE(act >= NO_ACT_NONE && act <= NO_ACT_SILU, NO_ERR_INVALID_ARG, "%s: unknown activation", who);
    NO_REQUIRE(cap >= 0 && d_in >= 1 && d_out >= 1, NO_ERR_INVALID_ARG, "%s: bad sizes", who);
    NO_REQUIRE(d_in <= NO_MAX_LINEAR_DIM && d_out <= NO_MAX_LINEAR_DIM && cap <= NO_MAX_LINEAR_ROWS, NO_ERR_UNSUPPORTED, "%s: a side of more than %d, or more than %d rows", who,
               NO_MAX_LINEAR_DIM, NO_MAX_LINEAR_ROWS);
    return NO_OK;
}

}  // namespace no

using namespace no;

extern "C" size_t no_linear_ws_bytes(no_dtype dt, int32_t n_rows_cap, int32_t d_in, int32_t d_out) {
    if ((dt != NO_F32 && dt != NO_BF16) || n_rows_cap < 0 || d_in < 1 || d_out < 1 || d_in > NO_MAX_LINEAR_DIM || d_out > NO_MAX_LINEAR_DIM || n_rows_cap > NO_MAX_LINEAR_ROWS) return 0;
    const int pieces = planes_of_type(dt);
    const int64_t n = n_rows_cap, least = n < LINEAR_FEW ? n : LINEAR_FEW;
    size_t parts = (size_t)linear_few_splits(d_in, d_out, least, dt == NO_F32 ? 4 : 2) * least * wide_of(d_out) * 4;        // (a call may have fewer rows than it is asked for)
    for (const size_t room : {linear_parts_room(n, d_out, d_in, pieces), linear_parts_room(n, d_in, d_out, pieces), linear_parts_room(d_in, d_out, n, pieces)})
        if (room > parts) parts = room;
    return 256 + operand_bytes(dt, n, d_in) + operand_bytes(dt, d_in, d_out) + operand_bytes(dt, n, d_out) + round_256((size_t)gz_blocks(n) * d_out * 4) + round_256(parts);
}

extern "C" int32_t no_linear_fwd(const void* d_x, no_dtype dt, int64_t x_stride_bytes, const void* d_w, int64_t w_stride_bytes, const float* d_bias, no_act act,
                                 const void* d_residual, int64_t residual_stride_bytes, const int32_t* d_n_rows, int32_t n_rows_cap, int32_t d_in, int32_t d_out,
                                 void* d_z, int64_t z_stride_bytes, void* d_y, int64_t y_stride_bytes, void* d_ws, size_t ws_bytes, void* stream) {
    clear_error();
    const char* who = "no_linear_fwd";
    NO_CHECK(linear_sizes(who, dt, act, n_rows_cap, d_in, d_out));
    NO_CHECK(check_rows(who, "x", d_x, dt, n_rows_cap, d_in, x_stride_bytes));
    NO_CHECK(check_rows(who, "w", d_w, dt, d_in, d_out, w_stride_bytes));
    if (d_residual) NO_CHECK(check_rows(who, "residual", d_residual, dt, n_rows_cap, d_out, residual_stride_bytes));
    if (d_z) NO_CHECK(check_rows(who, "z", d_z, dt, n_rows_cap, d_out, z_stride_bytes));
    NO_CHECK(check_rows(who, "y", d_y, dt, n_rows_cap, d_out, y_stride_bytes));
    NO_REQUIRE(d_ws && (uintptr_t)d_ws % 16 == 0, NO_ERR_INVALID_ARG, "%s: the workspace is NULL or misaligned", who);
    NO_REQUIRE(ws_bytes >= no_linear_ws_bytes(dt, n_rows_cap, d_in, d_out), NO_ERR_CAPACITY, "%s: workspace too small", who);
    if (n_rows_cap == 0) return NO_OK;
    const LinearEnd end{d_bias, rows_of(d_residual, residual_stride_bytes), rows_of(d_z, z_stride_bytes), rows_of(d_y, y_stride_bytes), (int32_t)act};
    const RowsOf x = rows_of(d_x, x_stride_bytes), w = rows_of(d_w, w_stride_bytes);
    if (dt == NO_F32) linear_fwd<float>(x, w, d_n_rows, n_rows_cap, d_in, d_out, end, (char*)d_ws, (hipStream_t)stream);
    else linear_fwd<bf16_t>(x, w, d_n_rows, n_rows_cap, d_in, d_out, end, (char*)d_ws, (hipStream_t)stream);
    return launch_status(who);
}

extern "C" int32_t no_linear_bwd(const void* d_x, no_dtype dt, int64_t x_stride_bytes, const void* d_w, int64_t w_stride_bytes, no_act act, const void* d_z,
                                 int64_t z_stride_bytes, const void* d_grad_y, int64_t grad_y_stride_bytes, const int32_t* d_n_rows, int32_t n_rows_cap, int32_t d_in,
                                 int32_t d_out, void* d_grad_x, int64_t grad_x_stride_bytes, void* d_grad_w, int64_t grad_w_stride_bytes, float* d_grad_bias, void* d_ws,
                                 size_t ws_bytes, void* stream) {
    clear_error();
    const char* who = "no_linear_bwd";
    NO_CHECK(linear_sizes(who, dt, act, n_rows_cap, d_in, d_out));
    if (d_grad_w) NO_CHECK(check_rows(who, "x", d_x, dt, n_rows_cap, d_in, x_stride_bytes));
    if (d_grad_x) NO_CHECK(check_rows(who, "w", d_w, dt, d_in, d_out, w_stride_bytes));
    if (act != NO_ACT_NONE) NO_CHECK(check_rows(who, "z", d_z, dt, n_rows_cap, d_out, z_stride_bytes));
    NO_CHECK(check_rows(who, "grad_y", d_grad_y, dt, n_rows_cap, d_out, grad_y_stride_bytes));
    if (d_grad_x) NO_CHECK(check_rows(who, "grad_x", d_grad_x, dt, n_rows_cap, d_in, grad_x_stride_bytes));
    if (d_grad_w) NO_CHECK(check_rows(who, "grad_w", d_grad_w, dt, d_in, d_out, grad_w_stride_bytes));
    NO_REQUIRE(d_ws && (uintptr_t)d_ws % 16 == 0, NO_ERR_INVALID_ARG, "%s: the workspace is NULL or misaligned", who);
    NO_REQUIRE(ws_bytes >= no_linear_ws_bytes(dt, n_rows_cap, d_in, d_out), NO_ERR_CAPACITY, "%s: workspace too small", who);
    const RowsOf x = rows_of(d_x, x_stride_bytes), w = rows_of(d_w, w_stride_bytes), z = rows_of(d_z, z_stride_bytes), gy = rows_of(d_grad_y, grad_y_stride_bytes),
                 gx = rows_of(d_grad_x, grad_x_stride_bytes), gw = rows_of(d_grad_w, grad_w_stride_bytes);
    if (dt == NO_F32) linear_bwd<float>(x, w, act, z, gy, d_n_rows, n_rows_cap, d_in, d_out, gx, gw, d_grad_bias, (char*)d_ws, (hipStream_t)stream);
    else linear_bwd<bf16_t>(x, w, act, z, gy, d_n_rows, n_rows_cap, d_in, d_out, gx, gw, d_grad_bias, (char*)d_ws, (hipStream_t)stream);
    return launch_status(who);
}
