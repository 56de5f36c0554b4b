// no_orthogonalise / no_muon_step: a matrix made nearly orthogonal by Newton-Schulz products, and the update of weights that uses it.
//
// X = U / |U|, then `steps` times G = X X^T (of the smaller side), P = b G + c G G, X <- a X + P X: every singular value s goes to a s + b s^3 + c s^5, which brings all of (0, 1] near
// 1, whatever the smallest, in five steps (0.0004 grows 485-fold). That growth is what the products' precision is for: values are held in two fp16 pieces, x = h + l with |l| <= 2^-11 |h| and what is left out
// below 2^-22 of x, and a product of two is the sum of three products of pieces (h h' + h l' + l h'; l l' is below 2^-22 of it), summed in fp32. Singular values stay below 1.21, so entries of X stay below 1.21,
// of G below 1.45 and of P below 2.81: pieces hold 2^14 times the value, below fp16's 65504, and what is 2^-17 of the largest still has all of its 22 bits.
// G and P are symmetric: only tiles on and above the diagonal are multiplied, and stored twice.
// Bound, when large, by the matrix pipes: a 4096 x 4096 update 3.43 ms, five times 190 us for G, 190 for P and 300 for the product with X (1.2 PFLOP/s of pieces); when small, by launches that follow one another:
// 602 x 256 111 us, five times 8.5, 6.7 and 6.5; four of 512 x 2048 267, five times 20, 9 and 23, where few tiles wait for what fills their LDS.
#include "dense.hpp"

namespace no {

constexpr float NS_A = 3.4445f, NS_B = -4.7750f, NS_C = 2.0315f;
constexpr float NS_HELD = 0x1p14f, NS_VALUE = 0x1p-14f;

// Eight values of one row in pieces.
__device__ __forceinline__ void ns_store(const float (&f)[8], char* to, int32_t plane) {
    f16x8 h, l;
#pragma unroll
    for (int w = 0; w < 8; ++w) {
        h[w] = (_Float16)f[w];
        l[w] = (_Float16)(f[w] - (float)h[w]);
    }
    *reinterpret_cast<f16x8*>(to) = h;
    *reinterpret_cast<f16x8*>(to + plane) = l;
}

// A matrix in pieces: rows of a multiple of 8 values, zeros past the columns, the second pieces of a row behind the first.
struct NsMatrix {
    char* p;
    int64_t pitch, matrix;
    int32_t plane;
};
struct NsRows {           // rows of the caller's matrices
    RowsOf rows;
    int64_t matrix;
    __device__ __forceinline__ RowsOf of(int64_t m) const { return RowsOf{rows.p + m * matrix, rows.stride}; }
};

// What follows the sums: own * from + by * sum, in pieces, or at the last step the result: stored as it is (out), or subtracted from weights (w <- keep w - step x).
enum { NS_PIECES, NS_OUT_F32, NS_OUT_BF16, NS_WEIGHTS };
template <bool SYMMETRIC>
struct NsEnd {
    struct Args {
        NsMatrix from, to;
        float own, by;
        int32_t kind;
        NsRows out;
        float keep, step;
        float* parts;           // not NULL: sums of a part of the reduction, [split][matrix][rows][pitch] of fp32, instead
        int32_t pitch;
        int64_t part;           // values from split to split
    };
    static constexpr bool MIRROR = SYMMETRIC;
    struct Ahead { f16x8 h, l; };
    __device__ static __forceinline__ Ahead ahead(const Args& e, int64_t z, int32_t m, int32_t n, int32_t) {
        Ahead a;
        if (e.from.p) {
            const char* from = e.from.p + z * e.from.matrix + m * e.from.pitch + n * 2;
            a.h = *reinterpret_cast<const f16x8*>(from);
            a.l = *reinterpret_cast<const f16x8*>(from + e.from.plane);
        }
        return a;
    }
    // a part's place; M is the side of a square where there are parts
    __device__ static __forceinline__ void keep_part(const Args& e, int64_t z, int32_t m, int32_t n, const float (&v)[8], int32_t M) {
        Run<float, 8> o;
        o.set(v);
        o.store(e.parts + blockIdx.y * e.part + (z * M + m) * e.pitch + n);
    }
    __device__ static __forceinline__ void pieces(const Args& e, int64_t z, int32_t m, int32_t n, const float (&v)[8]) {
        ns_store(v, e.to.p + z * e.to.matrix + m * e.to.pitch + n * 2, e.to.plane);
    }
    __device__ static __forceinline__ void put(const Args& e, int64_t z, int32_t m, int32_t n, int32_t here, float (&v)[8], const Ahead& a, int32_t M) {
        if (SYMMETRIC && e.parts) return keep_part(e, z, m, n, v, M);
#pragma unroll
        for (int w = 0; w < 8; ++w) {
            v[w] *= e.by;
            if (e.from.p) v[w] += e.own * ((float)a.h[w] + (float)a.l[w]);
            if (w >= here) v[w] = 0.0f;
        }
        if (SYMMETRIC || e.kind == NS_PIECES) return pieces(e, z, m, n, v);
#pragma unroll
        for (int w = 0; w < 8; ++w) v[w] *= NS_VALUE;
        const RowsOf out = e.out.of(z);
        if (e.kind == NS_OUT_BF16) {
            Run<bf16_t, 8> o;
            o.set(v);
            o.store(out.row<bf16_t>(m) + n, here);
            return;
        }
        Run<float, 8> o;
        if (e.kind == NS_WEIGHTS) {
            float f[8];
            o.load(out.row<float>(m) + n, here, 0.0f);
            o.get(f);
#pragma unroll
            for (int w = 0; w < 8; ++w) v[w] = f[w] * e.keep - v[w] * e.step;
        }
        o.set(v);
        o.store(out.row<float>(m) + n, here);
    }
    __device__ static __forceinline__ void mirror(const Args& e, int64_t z, int32_t m, int32_t n, const float (&v)[8], int32_t M) {
        if (e.parts) keep_part(e, z, m, n, v, M);
        else pieces(e, z, m, n, v);
    }
};

// The parts of Gram matrices added up in order, in pieces (an update of 117 x 3860 takes 168 us with whole reductions, 128 with split ones).
__global__ void __launch_bounds__(256) ns_join_kernel(const float* __restrict__ parts, int32_t splits, int64_t part, int32_t side, int32_t pitch, int32_t matrices, float by, NsMatrix to) {
    const int32_t units = pitch / 8;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / units;
    if (row >= (int64_t)matrices * side) return;
    const int32_t c = (int32_t)(i - row * units) * 8;
    float v[8] = {};
#pragma unroll 4
    for (int32_t s = 0; s < splits; ++s) {
        Run<float, 8> r;
        float f[8];
        r.load(parts + s * part + row * pitch + c);
        r.get(f);
#pragma unroll
        for (int w = 0; w < 8; ++w) v[w] += f[w];
    }
#pragma unroll
    for (int w = 0; w < 8; ++w) v[w] = c + w < side ? v[w] * by : 0.0f;
    const int64_t z = row / side;
    ns_store(v, to.p + z * to.matrix + (row - z * side) * to.pitch + c * 2, to.plane);
}

// ------------------------------------------------------------------------------------------------------- before the products

constexpr int NS_SUMS = 1024;       // blocks a matrix, at most, whose sums of squares make its norm

// U: the matrix itself, or the momentum after this step, m <- beta m + g, and U = g + beta m (nesterov) or m. First pass: the sums of squares in 64 bits (and the momentum stored);
// second: 2^14 U / |U| in pieces. A matrix of zeros stays one. Each reads a value once; 4096 x 4096 with a bf16 gradient and fp32 momentum 29 and 28 us (165 MB, 5.7 TB/s).
template <typename T>
struct NsSource {
    NsRows x, momentum;
    float beta;
    int32_t nesterov;
    // eight values of row r from column c on; DONE: the momentum is this step's already
    template <bool DONE>
    __device__ __forceinline__ void get(int64_t z, int64_t r, int32_t c, int32_t cols, float (&f)[8]) const {
        Run<T, 8> v;
        v.load_at(x.of(z).template row<T>(r), c, cols, from_f32<T>(0.0f));
        v.get(f);
        if (!momentum.rows.p) return;
        float* at = momentum.of(z).template row<float>(r);
        Run<float, 8> m;
        float k[8];
        m.load_at(at, c, cols, 0.0f);
        m.get(k);
        if (!DONE) {
#pragma unroll
            for (int w = 0; w < 8; ++w) k[w] = beta * k[w] + f[w];
            m.set(k);
            m.store(at + c, cols - c);
        }
#pragma unroll
        for (int w = 0; w < 8; ++w) f[w] = nesterov ? f[w] + beta * k[w] : k[w];
    }
};

template <typename T>
__global__ void __launch_bounds__(256) ns_norm_kernel(NsSource<T> u, int32_t rows, int32_t cols, double* sums) {
    __shared__ double share[4];
    const int64_t z = blockIdx.y;
    const int32_t units = (cols + 7) / 8;
    double sum = 0.0;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < (int64_t)rows * units; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / units;
        const int32_t c = (int32_t)(i - r * units) * 8;
        float f[8];
        u.template get<false>(z, r, c, cols, f);
#pragma unroll
        for (int w = 0; w < 8; ++w) if (c + w < cols) sum += (double)f[w] * (double)f[w];
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    if (lane_id() == 0) share[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) sums[z * NS_SUMS + blockIdx.x] = share[0] + share[1] + share[2] + share[3];
}

template <typename T>
__global__ void __launch_bounds__(256) ns_pieces_kernel(NsSource<T> u, int32_t rows, int32_t cols, const double* __restrict__ sums, int32_t n_sums, NsMatrix to) {
    __shared__ double share[4];
    const int64_t z = blockIdx.y;
    double sum = 0.0;
    for (int32_t i = threadIdx.x; i < n_sums; i += 256) sum += sums[z * NS_SUMS + i];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    if (lane_id() == 0) share[threadIdx.x >> 6] = sum;
    __syncthreads();
    sum = share[0] + share[1] + share[2] + share[3];
    const double by = sum == 0.0 ? 0.0 : (double)NS_HELD / sqrt(sum);
    const int32_t units = (cols + 7) / 8;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < (int64_t)rows * units; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / units;
        const int32_t c = (int32_t)(i - r * units) * 8;
        float f[8];
        u.template get<true>(z, r, c, cols, f);
#pragma unroll
        for (int w = 0; w < 8; ++w) f[w] = c + w < cols ? (float)((double)f[w] * by) : 0.0f;
        ns_store(f, to.p + z * to.matrix + r * to.pitch + c * 2, to.plane);
    }
}

// ------------------------------------------------------------------------------------------------------- products

template <bool AL, bool BL, bool HALF>
static void ns_product(const NsMatrix& a, int32_t a_extent, const NsMatrix& b, int32_t b_extent, int32_t M, int32_t N, int32_t K, int32_t matrices, const typename NsEnd<HALF>::Args& e,
                       const DensePlan& plan, hipStream_t st) {
    DenseArgs g{};
    g.a = DenseOperand{a.p, a.pitch, a.matrix, a.plane, a_extent};
    g.b = DenseOperand{b.p, b.pitch, b.matrix, b.plane, b_extent};
    g.M = M; g.N = N; g.K = K;
    dense_launch<_Float16, 2, AL, BL, NsEnd<HALF>>(g, e, plan, matrices, st);
}

constexpr size_t NS_PARTS_MOST = (size_t)64 << 20;       // bytes of a Gram matrix's parts, at most

struct NsRoom {
    NsMatrix x[2], gram, poly;
    double* sums;
    float* parts;
    DensePlan plan;         // of the Gram matrices
    size_t bytes;
};

static NsMatrix ns_matrix(char*& p, int64_t matrices, int64_t rows, int64_t cols) {
    const int32_t plane = (int32_t)wide_of(cols) * 2;
    const NsMatrix m{p, 2 * plane, 2 * plane * rows, plane};
    p += round_256((size_t)(matrices * m.matrix));
    return m;
}
static NsRoom ns_room(char* ws, int64_t matrices, int64_t rows, int64_t cols) {
    const int64_t side = rows < cols ? rows : cols;
    NsRoom r;
    char* p = ws;
    r.sums = (double*)p;
    p += round_256((size_t)matrices * NS_SUMS * 8);
    r.x[0] = ns_matrix(p, matrices, rows, cols);
    r.x[1] = ns_matrix(p, matrices, rows, cols);
    r.gram = ns_matrix(p, matrices, side, side);
    r.poly = ns_matrix(p, matrices, side, side);
    r.plan = dense_plan(side, side, rows < cols ? cols : rows, 2, matrices < 1 ? 1 : matrices, true, NS_PARTS_MOST);
    r.parts = (float*)p;
    p += round_256(dense_parts_room(side, side, rows < cols ? cols : rows, 2, matrices, NS_PARTS_MOST));       // (for matrices of smaller sides, too)
    r.bytes = (size_t)(p - ws);
    return r;
}

template <typename T>
static void newton_schulz(const NsSource<T>& u, int32_t matrices, int32_t rows, int32_t cols, int32_t steps, int32_t kind, const NsRows& out, float keep, float step, char* ws,
                          hipStream_t st) {
    const NsRoom room = ns_room(ws, matrices, rows, cols);
    const int64_t units = (int64_t)rows * ((cols + 7) / 8), blocks = ceil_div(units, 256);
    const int32_t n_sums = (int32_t)(blocks < NS_SUMS ? blocks : NS_SUMS);
    hipLaunchKernelGGL(ns_norm_kernel<T>, dim3((unsigned)n_sums, (unsigned)matrices), dim3(256), 0, st, u, rows, cols, room.sums);
    hipLaunchKernelGGL(ns_pieces_kernel<T>, dim3((unsigned)(blocks < 2048 ? blocks : 2048), (unsigned)matrices), dim3(256), 0, st, u, rows, cols, room.sums, n_sums, room.x[0]);
    const bool tall = rows > cols;
    const int32_t side = tall ? cols : rows, wide_c = (int32_t)wide_of(cols);
    const NsMatrix none{nullptr, 0, 0, 0};
    const NsRows nowhere{{nullptr, 0}, 0};
    for (int32_t s = 0; s < steps; ++s) {
        const NsMatrix &x = room.x[s & 1], &next = room.x[(s & 1) ^ 1];
        const int32_t pitch = (int32_t)wide_of(side);
        const int64_t part = (int64_t)matrices * side * pitch;
        const bool split = room.plan.splits > 1;
        const NsEnd<true>::Args gram{none, room.gram, 0.0f, NS_VALUE, NS_PIECES, nowhere, 0.0f, 0.0f, split ? room.parts : nullptr, pitch, part};
        if (tall) ns_product<false, false, true>(x, wide_c, x, wide_c, side, side, rows, matrices, gram, room.plan, st);
        else ns_product<true, true, true>(x, rows, x, rows, side, side, cols, matrices, gram, room.plan, st);
        if (split)
            hipLaunchKernelGGL(ns_join_kernel, dim3((unsigned)ceil_div(part / 8, 256)), dim3(256), 0, st, room.parts, room.plan.splits, part, side, pitch, matrices, NS_VALUE, room.gram);
        const NsEnd<true>::Args poly{room.gram, room.poly, NS_B, NS_C * NS_VALUE, NS_PIECES, nowhere, 0.0f, 0.0f, nullptr, 0, 0};
        ns_product<true, true, true>(room.gram, side, room.gram, side, side, side, side, matrices, poly, dense_plan(side, side, side, 2, matrices, true, 0), st);
        const bool last = s == steps - 1;
        const NsEnd<false>::Args to{x, next, NS_A, NS_VALUE, last ? kind : (int32_t)NS_PIECES, out, keep, step, nullptr, 0, 0};
        const DensePlan plan = dense_plan(rows, cols, side, 2, matrices, false, 0);
        if (tall) ns_product<true, true, false>(x, rows, room.poly, side, rows, cols, side, matrices, to, plan, st);
        else ns_product<true, false, false>(room.poly, side, x, wide_c, rows, cols, side, matrices, to, plan, st);
    }
}

static int32_t ns_sizes(const char* who, int32_t matrices, int32_t rows, int32_t cols, int32_t steps) {
    NO_REQUIRE(matrices >= 0 && rows >= 1 && cols >= 1 && steps >= 1 && steps <= 100, NO_ERR_INVALID_ARG, "%s: bad sizes or number of steps", who);
    NO_REQUIRE(rows <= NO_MAX_UPDATE_DIM && cols <= NO_MAX_UPDATE_DIM && matrices <= 65535, NO_ERR_UNSUPPORTED, "%s: a side of more than %d, or more than 65535 matrices", who,
               NO_MAX_UPDATE_DIM);
    return NO_OK;
}

static int32_t check_matrices(const char* who, const char* what, const void* p, no_dtype dt, int32_t matrices, int32_t rows, int32_t cols, int64_t stride, int64_t matrix) {
    NO_CHECK(check_rows(who, what, p, dt, matrices, cols, stride));
    NO_REQUIRE(matrices <= 1 || (matrix % size_of(dt) == 0 && matrix >= (rows - 1) * stride + (int64_t)cols * size_of(dt)), NO_ERR_INVALID_ARG, "%s: %s: matrices overlap or are misaligned", who, what);
    return NO_OK;
}

}  // namespace no

using namespace no;

extern "C" size_t no_orthogonalise_ws_bytes(int32_t n_matrices, int32_t rows, int32_t cols) {
    if (n_matrices < 0 || rows < 1 || cols < 1 || rows > NO_MAX_UPDATE_DIM || cols > NO_MAX_UPDATE_DIM || n_matrices > 65535) return 0;
    return 256 + ns_room(nullptr, n_matrices, rows, cols).bytes;
}

extern "C" int32_t no_orthogonalise(const void* d_x, no_dtype dt, int64_t x_stride_bytes, int64_t x_matrix_bytes, int32_t n_matrices, int32_t rows, int32_t cols, int32_t steps,
                                    void* d_out, no_dtype dt_out, int64_t out_stride_bytes, int64_t out_matrix_bytes, void* d_ws, size_t ws_bytes, void* stream) {
    clear_error();
    const char* who = "no_orthogonalise";
    NO_REQUIRE((dt == NO_F32 || dt == NO_BF16) && (dt_out == NO_F32 || dt_out == NO_BF16), NO_ERR_INVALID_ARG, "%s: matrices are NO_F32 or NO_BF16", who);
    NO_CHECK(ns_sizes(who, n_matrices, rows, cols, steps));
    NO_CHECK(check_matrices(who, "x", d_x, dt, n_matrices, rows, cols, x_stride_bytes, x_matrix_bytes));
    NO_CHECK(check_matrices(who, "out", d_out, dt_out, n_matrices, rows, cols, out_stride_bytes, out_matrix_bytes));
    NO_REQUIRE(d_ws && (uintptr_t)d_ws % 16 == 0, NO_ERR_INVALID_ARG, "%s: the workspace is NULL or misaligned", who);
    NO_REQUIRE(ws_bytes >= no_orthogonalise_ws_bytes(n_matrices, rows, cols), NO_ERR_CAPACITY, "%s: workspace too small", who);
    if (n_matrices == 0) return NO_OK;
    const NsRows x{rows_of(d_x, x_stride_bytes), x_matrix_bytes}, out{rows_of(d_out, out_stride_bytes), out_matrix_bytes}, none{{nullptr, 0}, 0};
    const int32_t kind = dt_out == NO_F32 ? NS_OUT_F32 : NS_OUT_BF16;
    if (dt == NO_F32) newton_schulz(NsSource<float>{x, none, 0.0f, 0}, n_matrices, rows, cols, steps, kind, out, 0.0f, 0.0f, (char*)d_ws, (hipStream_t)stream);
    else newton_schulz(NsSource<bf16_t>{x, none, 0.0f, 0}, n_matrices, rows, cols, steps, kind, out, 0.0f, 0.0f, (char*)d_ws, (hipStream_t)stream);
    return launch_status(who);
}

extern "C" int32_t no_muon_step(float* d_w, int64_t w_stride_bytes, int64_t w_matrix_bytes, float* d_momentum, int64_t momentum_stride_bytes, int64_t momentum_matrix_bytes,
                                const void* d_grad, no_dtype dt, int64_t grad_stride_bytes, int64_t grad_matrix_bytes, int32_t n_matrices, int32_t rows, int32_t cols, float lr,
                                float beta, int32_t nesterov, int32_t steps, float weight_decay, float scale, void* d_ws, size_t ws_bytes, void* stream) {
    clear_error();
    const char* who = "no_muon_step";
    NO_REQUIRE(dt == NO_F32 || dt == NO_BF16, NO_ERR_INVALID_ARG, "%s: gradients are NO_F32 or NO_BF16", who);
    NO_CHECK(ns_sizes(who, n_matrices, rows, cols, steps));
    NO_CHECK(check_matrices(who, "w", d_w, NO_F32, n_matrices, rows, cols, w_stride_bytes, w_matrix_bytes));
    NO_CHECK(check_matrices(who, "momentum", d_momentum, NO_F32, n_matrices, rows, cols, momentum_stride_bytes, momentum_matrix_bytes));
    NO_CHECK(check_matrices(who, "grad", d_grad, dt, n_matrices, rows, cols, grad_stride_bytes, grad_matrix_bytes));
    NO_REQUIRE(d_ws && (uintptr_t)d_ws % 16 == 0, NO_ERR_INVALID_ARG, "%s: the workspace is NULL or misaligned", who);
    NO_REQUIRE(ws_bytes >= no_orthogonalise_ws_bytes(n_matrices, rows, cols), NO_ERR_CAPACITY, "%s: workspace too small", who);
    if (n_matrices == 0) return NO_OK;
    const NsRows w{rows_of(d_w, w_stride_bytes), w_matrix_bytes}, m{rows_of(d_momentum, momentum_stride_bytes), momentum_matrix_bytes}, g{rows_of(d_grad, grad_stride_bytes), grad_matrix_bytes};
    const float keep = 1.0f - lr * weight_decay, step = lr * scale;
    if (dt == NO_F32) newton_schulz(NsSource<float>{g, m, beta, nesterov}, n_matrices, rows, cols, steps, NS_WEIGHTS, w, keep, step, (char*)d_ws, (hipStream_t)stream);
    else newton_schulz(NsSource<bf16_t>{g, m, beta, nesterov}, n_matrices, rows, cols, steps, NS_WEIGHTS, w, keep, step, (char*)d_ws, (hipStream_t)stream);
    return launch_status(who);
}
