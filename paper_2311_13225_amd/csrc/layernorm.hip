// no_layernorm_fwd / no_layernorm_bwd: layer norm of rows with the residual's addition, and its gradients.
#include "rows.hpp"

namespace no {

// y = (s - mean) rstd weight + bias of s = x + residual, rstd = 1 / sqrt(mean of (s - mean)^2 + eps). A team of lanes holds a row in registers, U runs of 16 bytes a
// lane, and goes over it three times (sum, squares of the differences, result), so that nothing cancels and memory sees the row once, up to 16384 fp32 values and 32768 of bf16 (above 16384 of which 12 to 24 registers are
// spilled); of wider rows 104 to 448 registers go to scratch.
// Bound by memory: 16384 x 4096 bf16 with residual and sum 94 us (537 MB, 5.7 TB/s), 50001 x 602 fp32 into bf16 38 (181 MB, 4.8 TB/s; arithmetic takes 73 % of its cycles), 3000 x 16384 fp32 with residual 143 and 3000 x 32768
// bf16 158 (786 MB, 5.5 and 5.0 TB/s), one row of 1024 3.0 in the kernel. By scratch: 1500 x 32768 fp32 202, 750 x 65536 fp32 428, 1500 x 65536 bf16 212 (786 MB each).
template <typename T, typename Y, int TEAM, int THREADS, int U>
__global__ void __launch_bounds__(THREADS) layernorm_fwd_kernel(RowsOf x, RowsOf residual, const float* __restrict__ weight, const float* __restrict__ bias, float eps,
                                                                const int32_t* d_n, int32_t cap, int32_t dim, RowsOf sum, RowsOf y, float* mean_out, float* rstd_out) {
    constexpr int W = 16 / (int)sizeof(T), PER_BLOCK = THREADS / TEAM;
    constexpr bool KEEP = U * W <= 16;          // weights and biases in registers
    __shared__ float smem[2 * THREADS / 64];
    Team<TEAM, THREADS> team(smem);
    const int32_t n = rows_here(d_n, cap), t = team.lane();
    const T zero = from_f32<T>(0.0f);
    RowRegs<float, W, KEEP ? U : 1, TEAM> wk, bk;
    if constexpr (KEEP) {
        if (weight) wk.load(weight, dim, t, 0.0f);
        if (bias) bk.load(bias, dim, t, 0.0f);
    }
    for (int64_t i = (int64_t)blockIdx.x * PER_BLOCK + team.index(); i < n; i += (int64_t)gridDim.x * PER_BLOCK) {
        RowRegs<T, W, U, TEAM> s, r;
        s.load(x.row<T>(i), dim, t, zero);
        float total = 0.0f;
        if (residual.p) {
            r.load(residual.row<T>(i), dim, t, zero);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float f[W], g[W];
                s.v[u].get(f);
                r.v[u].get(g);
#pragma unroll
                for (int w = 0; w < W; ++w) f[w] += g[w];
                s.v[u].set(f);
            }
        }
        s.renew();
#pragma unroll
        for (int u = 0; u < U; ++u) {       // (what lies past the row is 0)
            float f[W];
            s.v[u].get(f);
#pragma unroll
            for (int w = 0; w < W; ++w) total += f[w];
        }
        if (sum.p) {
            RowStore<T, W, true> store(sum.row<T>(i), dim);
#pragma unroll
            for (int u = 0; u < U; ++u) store.put(s.at(t, u), s.v[u]);
            store.finish();
        }
        const float mean = team.sum(total) / (float)dim;
        float ss = 0.0f;
        s.renew();
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float f[W];
            s.v[u].get(f);
            if ((u + 1) * TEAM * W <= dim) {        // every lane's run lies in the row
#pragma unroll
                for (int w = 0; w < W; ++w) ss += (f[w] - mean) * (f[w] - mean);
            } else {
                const int32_t here = dim - s.at(t, u);
#pragma unroll
                for (int w = 0; w < W; ++w) ss += w < here ? (f[w] - mean) * (f[w] - mean) : 0.0f;
            }
        }
        const float rstd = 1.0f / sqrtf(team.sum(ss) / (float)dim + eps);
        s.renew();
        RowStore<Y, W, true> store(y.row<Y>(i), dim);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float f[W], k[W], c[W];
            s.v[u].get(f);
            if constexpr (KEEP) {
                wk.v[u].get(k);
                bk.v[u].get(c);
            } else {
                Run<float, W> one;
                if (weight) { one.load_at(weight, s.at(t, u), dim, 0.0f); one.get(k); }
                if (bias) { one.load_at(bias, s.at(t, u), dim, 0.0f); one.get(c); }
            }
#pragma unroll
            for (int w = 0; w < W; ++w) {
                float v = (f[w] - mean) * rstd;
                if (weight) v *= k[w];
                f[w] = bias ? v + c[w] : v;
            }
            Run<Y, W> o;
            o.set(f);
            store.put(s.at(t, u), o);
        }
        store.finish();
        if (t == 0) {
            if (mean_out) mean_out[i] = mean;
            if (rstd_out) rstd_out[i] = rstd;
        }
    }
}

// ------------------------------------------------------------------------------------------------------- gradients
//
// The gradients of weight and bias are sums over rows for every column: a team adds its rows' terms in registers while it makes their input gradients, a block joins
// its teams' sums in LDS and stores one row of parts of each, and a second launch adds the blocks' parts in order.
// Bound by memory: 16384 x 2048 bf16 with grad_sum 59 us (268 MB, 4.6 TB/s) and 3 to 5 for the parts, of fp32 in all 94 (537 MB, 5.7 TB/s), 6000 x 8192 fp32 142 (5.5 TB/s); with the weights in LDS, or read again for every
// row, slower. Rows of 8193 to 16384 values, whose weights, sums and next row do not fit the registers (89 of fp32 and 42 of bf16 are spilled): 3000 x 16384 fp32 313 (786 MB, 2.5 TB/s), bf16 163 (393 MB).

constexpr int32_t LAYERNORM_PARTS = 512;     // rows of parts, at most

template <typename T, int TEAM, int THREADS, int U>
__global__ void __launch_bounds__(THREADS) layernorm_bwd_kernel(RowsOf s, const float* __restrict__ weight, const float* __restrict__ mean_in, const float* __restrict__ rstd,
                                                                RowsOf grad_y, RowsOf grad_sum, const int32_t* d_n, int32_t cap, int32_t dim, RowsOf grad_x, float* parts_w,
                                                                float* parts_b) {
    constexpr int W = 16 / (int)sizeof(T), PER_BLOCK = THREADS / TEAM;
    __shared__ float smem[4 * THREADS / 64];
    __shared__ float joined[PER_BLOCK > 1 ? U * TEAM * W : 1];
    Team<TEAM, THREADS> team(smem);
    const int32_t n = rows_here(d_n, cap), t = team.lane();
    const T zero = from_f32<T>(0.0f);
    RowRegs<float, W, U, TEAM> wk;
    float dw[U][W], db[U][W];
    if (weight) wk.load(weight, dim, t, 0.0f);
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int w = 0; w < W; ++w) dw[u][w] = db[u][w] = 0.0f;
        if (!weight) {
            const float one[4] = {1.0f, 1.0f, 1.0f, 1.0f};
#pragma unroll
            for (int k = 0; k < Run<float, W>::N; ++k) __builtin_memcpy(&wk.v[u].v[k], one, 16);
        }
    }
    const int64_t stride = (int64_t)gridDim.x * PER_BLOCK;
    int64_t i = (int64_t)blockIdx.x * PER_BLOCK + team.index();
    RowRegs<T, W, U, TEAM, U * TEAM >= 256> rs, rg, ra;
    float r = 0.0f, m = 0.0f;
    if (i < n) {
        r = rstd[i];
        m = mean_in[i];
        rs.load(s.row<T>(i), dim, t, zero);
        rg.load(grad_y.row<T>(i), dim, t, zero);
        if (grad_sum.p) ra.load(grad_sum.row<T>(i), dim, t, zero);
    }
    for (; i < n; i += stride) {
        // each run of the next row is requested when the gradient has no more use for this one's registers
        const int64_t next = i + stride, at = next < n ? next : i;
        const int32_t next_len = next < n ? dim : 0;
        const T *const next_s = s.row<T>(at), *const next_g = grad_y.row<T>(at), *const next_a = grad_sum.p ? grad_sum.row<T>(at) : nullptr;
        const float next_r = rstd[at], next_m = mean_in[at];
        float dot = 0.0f, flat = 0.0f;
#pragma unroll
        for (int u = 0; u < U; ++u) {       // (the gradient past the row is 0, and so is everything it meets)
            float v[W], g[W], k[W];
            rs.v[u].get(v);
            rg.v[u].get(g);
            wk.v[u].get(k);
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float gu = g[w] * ((v[w] - m) * r);
                dw[u][w] += gu;
                db[u][w] += g[w];
                dot += gu * k[w];
                flat += g[w] * k[w];
            }
        }
        team.sum_two(dot, flat);
        const float mean_dot = dot / (float)dim, mean_flat = flat / (float)dim;
        rs.renew();
        rg.renew();
        RowStore<T, W, TEAM != 64> store(grad_x.row<T>(i), dim);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[W], g[W], k[W], a[W];
            rs.v[u].get(v);
            rg.v[u].get(g);
            wk.v[u].get(k);
            if (grad_sum.p) ra.v[u].get(a);
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float dx = r * (g[w] * k[w] - mean_flat - (v[w] - m) * r * mean_dot);
                g[w] = grad_sum.p ? dx + a[w] : dx;
            }
            Run<T, W> o;
            o.set(g);
            store.put(rs.at(t, u), o);
            rs.load_run(next_s, next_len, t, u, zero);
            rg.load_run(next_g, next_len, t, u, zero);
            if (grad_sum.p) ra.load_run(next_a, next_len, t, u, zero);
        }
        store.finish();
        rs.load_end(next_s, next_len, t, zero);
        rg.load_end(next_g, next_len, t, zero);
        if (grad_sum.p) ra.load_end(next_a, next_len, t, zero);
        r = next_r;
        m = next_m;
    }
    auto put = [&](float (&d)[U][W], float* parts) {
        if (!parts) return;
        if constexpr (PER_BLOCK > 1) {      // the block's teams in turn
            for (int k = 0; k < PER_BLOCK; ++k) {
                if (team.index() == k)
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int w = 0; w < W; ++w) {
                            float& to = joined[((t + u * TEAM) * W) + w];
                            to = k ? to + d[u][w] : d[u][w];
                            if (k == PER_BLOCK - 1) d[u][w] = to;
                        }
                __syncthreads();
            }
            if (team.index() != PER_BLOCK - 1) return;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int32_t c = (t + u * TEAM) * W;
            if (c < dim) {
                Run<float, W> o;
                o.set(d[u]);
                o.store(parts + (int64_t)blockIdx.x * dim + c, dim - c);
            }
        }
    };
    put(dw, parts_w);
    if (PER_BLOCK > 1) __syncthreads();
    put(db, parts_b);
}

// Rows too wide for registers: an element a lane, read twice, and a third time for the parameters' gradients (1500 x 32768 fp32 323 us, 750 x 65536 377, 3000 x 32768 bf16 484, 1500 x 65536 510, 786 MB each at one reading).
template <typename T>
__global__ void __launch_bounds__(1024) layernorm_bwd_wide_kernel(RowsOf s, const float* __restrict__ weight, const float* __restrict__ mean_in, const float* __restrict__ rstd,
                                                                  RowsOf grad_y, RowsOf grad_sum, const int32_t* d_n, int32_t cap, int32_t dim, RowsOf grad_x) {
    __shared__ float smem[64];
    Team<1024, 1024> team(smem);
    const int32_t n = rows_here(d_n, cap);
    for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
        const float r = rstd[i], m = mean_in[i];
        float dot = 0.0f, flat = 0.0f;
        for (int32_t c = threadIdx.x; c < dim; c += 1024) {
            const float g = to_f32(grad_y.row<T>(i)[c]) * (weight ? weight[c] : 1.0f);
            dot += g * ((to_f32(s.row<T>(i)[c]) - m) * r);
            flat += g;
        }
        team.sum_two(dot, flat);
        const float mean_dot = dot / (float)dim, mean_flat = flat / (float)dim;
        for (int32_t c = threadIdx.x; c < dim; c += 1024) {
            const float g = to_f32(grad_y.row<T>(i)[c]) * (weight ? weight[c] : 1.0f);
            const float dx = r * (g - mean_flat - (to_f32(s.row<T>(i)[c]) - m) * r * mean_dot);
            grad_x.row<T>(i)[c] = from_f32<T>(grad_sum.p ? dx + to_f32(grad_sum.row<T>(i)[c]) : dx);
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(256) layernorm_wide_parts_kernel(RowsOf s, const float* __restrict__ mean_in, const float* __restrict__ rstd, RowsOf grad_y, const int32_t* d_n,
                                                                   int32_t cap, int32_t dim, float* parts_w, float* parts_b) {
    const int32_t n = rows_here(d_n, cap), c = (int32_t)(blockIdx.x * 256 + threadIdx.x);
    if (c >= dim) return;
    float w = 0.0f, b = 0.0f;
    for (int64_t i = blockIdx.y; i < n; i += gridDim.y) {
        const float g = to_f32(grad_y.row<T>(i)[c]);
        w += g * ((to_f32(s.row<T>(i)[c]) - mean_in[i]) * rstd[i]);
        b += g;
    }
    if (parts_w) parts_w[(int64_t)blockIdx.y * dim + c] = w;
    if (parts_b) parts_b[(int64_t)blockIdx.y * dim + c] = b;
}

// Sixteen columns a block, 64 lanes to a column, so that a lane has eight parts at most and asks for them at once. blockIdx.y: the weight's gradient or the bias's.
__global__ void __launch_bounds__(1024) layernorm_join_kernel(const float* __restrict__ parts_w, const float* __restrict__ parts_b, int32_t n_parts, int32_t dim,
                                                              float* grad_weight, float* grad_bias) {
    __shared__ float share[64][16];
    const float* parts = blockIdx.y ? parts_b : parts_w;
    float* to = blockIdx.y ? grad_bias : grad_weight;
    if (!to) return;
    const int32_t col = (int32_t)threadIdx.x & 15, row = (int32_t)threadIdx.x >> 4, c = (int32_t)blockIdx.x * 16 + col;
    float sum = 0.0f;
    if (c < dim) {
#pragma unroll
        for (int k = 0; k < LAYERNORM_PARTS / 64; ++k) {
            const int32_t p = row + k * 64;
            sum += p < n_parts ? parts[(int64_t)p * dim + c] : 0.0f;
        }
    }
    share[row][col] = sum;
    __syncthreads();
    if (threadIdx.x >= 64) return;
    sum = 0.0f;
#pragma unroll
    for (int k = 0; k < 16; ++k) sum += share[(lane_id() >> 4) * 16 + k][col];
    sum += __shfl_xor(sum, 16, 64);
    sum += __shfl_xor(sum, 32, 64);
    if (threadIdx.x < 16 && c < dim) to[c] = sum;
}

// Blocks for n rows, `most` at most, behind which a team walks several rows.
static inline int64_t layernorm_blocks(int64_t n, int per_block, int64_t most) {
    const int64_t b = ceil_div(n, per_block);
    return b < most ? b : most;
}

// The forward pass's most blocks. A block that walks several rows reads weights and biases (twice the bytes of a bf16 row) once: 50001 x 602 fp32 into bf16 40.3 us with 1024 blocks, 54.7 with one for every four rows;
// 16384 x 4096 bf16 with residual 95.4 with 8192, 97 with 4096 and 101 with 16384; 8000 x 8192 62.4 with 4096, 75.6 with 1024; 4000 x 16384 101 with 1024, 109 with all. Rows of 512 or 1024 values are no faster so (30000 x
// 1024 bf16 42.8, 43.5 with 1024; 100000 x 256 fp32 71.5 and 79.1).
static inline int64_t layernorm_most(int team, int u) {
    if (team == 1024) return 256;
    if (team < 64) return 2048;
    if (team == 64) return u >= 3 ? 1024 : 1 << 20;
    return u == 2 ? 8192 : u == 4 ? 4096 : 1024;
}

}  // namespace no

using namespace no;

extern "C" int32_t no_layernorm_fwd(const void* d_x, no_dtype dt, int64_t x_stride_bytes, const void* d_residual, int64_t residual_stride_bytes,
                                    const float* d_weight, const float* d_bias, float eps, const int32_t* d_n_rows, int32_t n_rows_cap, int32_t dim,
                                    void* d_sum, int64_t sum_stride_bytes, void* d_y, no_dtype dt_y, int64_t y_stride_bytes, float* d_mean,
                                    float* d_rstd, void* stream) {
    clear_error();
    const char* who = "no_layernorm_fwd";
    NO_REQUIRE(dt == NO_F32 || dt == NO_BF16, NO_ERR_INVALID_ARG, "%s: rows are NO_F32 or NO_BF16", who);
    NO_REQUIRE(dt_y == NO_F32 || dt_y == NO_BF16, NO_ERR_INVALID_ARG, "%s: results are NO_F32 or NO_BF16", who);
    NO_REQUIRE(n_rows_cap >= 0 && dim >= 1 && eps >= 0.0f, NO_ERR_INVALID_ARG, "%s: bad sizes or eps", who);
    NO_REQUIRE(dim <= NO_MAX_NORM_DIM, NO_ERR_UNSUPPORTED, "%s: rows of more than %d values", who, NO_MAX_NORM_DIM);
    NO_CHECK(check_rows(who, "x", d_x, dt, n_rows_cap, dim, x_stride_bytes));
    if (d_residual) NO_CHECK(check_rows(who, "residual", d_residual, dt, n_rows_cap, dim, residual_stride_bytes));
    if (d_sum) NO_CHECK(check_rows(who, "sum", d_sum, dt, n_rows_cap, dim, sum_stride_bytes));
    NO_CHECK(check_rows(who, "y", d_y, dt_y, n_rows_cap, dim, y_stride_bytes));
    if (n_rows_cap == 0) return NO_OK;
    const RowsOf x = rows_of(d_x, x_stride_bytes), r = rows_of(d_residual, residual_stride_bytes), s = rows_of(d_sum, sum_stride_bytes), y = rows_of(d_y, y_stride_bytes);
    hipStream_t st = (hipStream_t)stream;
#define NO_NORM_AS(T, Y, TEAM, THREADS, U)                                                                                                                           \
    hipLaunchKernelGGL((layernorm_fwd_kernel<T, Y, TEAM, THREADS, U>), dim3((unsigned)layernorm_blocks(n_rows_cap, THREADS / TEAM, layernorm_most(TEAM, U))), \
                       dim3(THREADS), 0, st, x, r, d_weight, d_bias, eps, d_n_rows, n_rows_cap, dim, s, y, d_mean, d_rstd)
#define NO_NORM(T, Y)                                              \
    do {                                                           \
        const int64_t units = ceil_div(dim, 16 / (int)sizeof(T));  \
        if (units <= 8) NO_NORM_AS(T, Y, 8, 256, 1);               \
        else if (units <= 16) NO_NORM_AS(T, Y, 16, 256, 1);        \
        else if (units <= 32) NO_NORM_AS(T, Y, 32, 256, 1);        \
        else if (units <= 64) NO_NORM_AS(T, Y, 64, 256, 1);        \
        else if (units <= 128) NO_NORM_AS(T, Y, 64, 256, 2);       \
        else if (units <= 192) NO_NORM_AS(T, Y, 64, 256, 3);       \
        else if (units <= 256) NO_NORM_AS(T, Y, 64, 256, 4);       \
        else if (units <= 512) NO_NORM_AS(T, Y, 256, 256, 2);      \
        else if (units <= 1024) NO_NORM_AS(T, Y, 256, 256, 4);     \
        else if (units <= 2048) NO_NORM_AS(T, Y, 256, 256, 8);     \
        else if (units <= 4096) NO_NORM_AS(T, Y, 1024, 1024, 4);   \
        else if (units <= 8192) NO_NORM_AS(T, Y, 1024, 1024, 8);   \
        else NO_NORM_AS(T, Y, 1024, 1024, sizeof(T) == 4 ? 16 : 8); \
    } while (0)
    if (dt == NO_F32) { if (dt_y == NO_F32) NO_NORM(float, float); else NO_NORM(float, bf16_t); }
    else { if (dt_y == NO_F32) NO_NORM(bf16_t, float); else NO_NORM(bf16_t, bf16_t); }
#undef NO_NORM
#undef NO_NORM_AS
    return launch_status(who);
}

extern "C" size_t no_layernorm_ws_bytes(int32_t n_rows_cap, int32_t dim) {
    if (n_rows_cap < 0 || dim < 1 || dim > NO_MAX_NORM_DIM) return 0;
    return 16 + (size_t)(n_rows_cap < LAYERNORM_PARTS ? n_rows_cap : LAYERNORM_PARTS) * (size_t)dim * 8;
}

extern "C" int32_t no_layernorm_bwd(const void* d_s, no_dtype dt, int64_t s_stride_bytes, const float* d_weight, const float* d_mean, const float* d_rstd,
                                    const void* d_grad_y, int64_t grad_y_stride_bytes, const void* d_grad_sum, int64_t grad_sum_stride_bytes,
                                    const int32_t* d_n_rows, int32_t n_rows_cap, int32_t dim, void* d_grad_x, int64_t grad_x_stride_bytes,
                                    float* d_grad_weight, float* d_grad_bias, void* d_ws, size_t ws_bytes, void* stream) {
    clear_error();
    const char* who = "no_layernorm_bwd";
    NO_REQUIRE(dt == NO_F32 || dt == NO_BF16, NO_ERR_INVALID_ARG, "%s: rows are NO_F32 or NO_BF16", who);
    NO_REQUIRE(n_rows_cap >= 0 && dim >= 1, NO_ERR_INVALID_ARG, "%s: bad sizes", who);
    NO_REQUIRE(dim <= NO_MAX_NORM_DIM, NO_ERR_UNSUPPORTED, "%s: rows of more than %d values", who, NO_MAX_NORM_DIM);
    NO_CHECK(check_rows(who, "s", d_s, dt, n_rows_cap, dim, s_stride_bytes));
    NO_CHECK(check_rows(who, "grad_y", d_grad_y, dt, n_rows_cap, dim, grad_y_stride_bytes));
    if (d_grad_sum) NO_CHECK(check_rows(who, "grad_sum", d_grad_sum, dt, n_rows_cap, dim, grad_sum_stride_bytes));
    NO_CHECK(check_rows(who, "grad_x", d_grad_x, dt, n_rows_cap, dim, grad_x_stride_bytes));
    NO_REQUIRE((d_mean && d_rstd) || n_rows_cap == 0, NO_ERR_INVALID_ARG, "%s: mean or rstd is NULL", who);
    NO_REQUIRE(d_ws && (uintptr_t)d_ws % 16 == 0, NO_ERR_INVALID_ARG, "%s: the workspace is NULL or misaligned", who);
    NO_REQUIRE(ws_bytes >= no_layernorm_ws_bytes(n_rows_cap, dim), NO_ERR_CAPACITY, "%s: workspace too small", who);
    const RowsOf s = rows_of(d_s, s_stride_bytes), gy = rows_of(d_grad_y, grad_y_stride_bytes), gs = rows_of(d_grad_sum, grad_sum_stride_bytes), gx = rows_of(d_grad_x, grad_x_stride_bytes);
    hipStream_t st = (hipStream_t)stream;
    int64_t n_parts = 0;
    float *parts_w = nullptr, *parts_b = nullptr;
    // one block's sums are the gradients
    auto room = [&](int64_t blocks, bool direct) {
        n_parts = blocks;
        float* p = (float*)d_ws;
        parts_w = !d_grad_weight ? nullptr : direct && blocks == 1 ? d_grad_weight : p;
        parts_b = !d_grad_bias ? nullptr : direct && blocks == 1 ? d_grad_bias : p + blocks * dim;
    };
    bool direct = true;
#define NO_NORM_AS(T, TEAM, THREADS, U)                                                                                                              \
    do {                                                                                                                                             \
        room(layernorm_blocks(n_rows_cap, THREADS / TEAM, THREADS >= 512 ? 256 : LAYERNORM_PARTS), true);                                           \
        hipLaunchKernelGGL((layernorm_bwd_kernel<T, TEAM, THREADS, U>), dim3((unsigned)n_parts), dim3(THREADS), 0, st, s, d_weight, d_mean, d_rstd, gy, gs, d_n_rows, \
                           n_rows_cap, dim, gx, parts_w, parts_b);                                                                                   \
    } while (0)
#define NO_NORM(T)                                                                                                                                   \
    do {                                                                                                                                             \
        const int64_t units = ceil_div(dim, 16 / (int)sizeof(T));                                                                                    \
        if (units <= 8) NO_NORM_AS(T, 8, 256, 1);                                                                                                    \
        else if (units <= 16) NO_NORM_AS(T, 16, 256, 1);                                                                                             \
        else if (units <= 32) NO_NORM_AS(T, 32, 256, 1);                                                                                             \
        else if (units <= 64) NO_NORM_AS(T, 64, 256, 1);                                                                                             \
        else if (units <= 128) NO_NORM_AS(T, 64, 256, 2);                                                                                            \
        else if (units <= 192) NO_NORM_AS(T, 64, 256, 3);                                                                                            \
        /* (16384 x 2048 bf16 with grad_sum 63.0 us by a block a row, 66.2 by a wavefront, whose sums leave no registers for the next row; fp32 rows of as many bytes, 16384 x 1024, by a wavefront 48.4) */ \
        else if (units <= 256) NO_NORM_AS(T, (sizeof(T) == 2 ? 256 : 64), 256, (sizeof(T) == 2 ? 1 : 4));                                            \
        else if (units <= 512) NO_NORM_AS(T, 256, 256, 2);                                                                                           \
        else if (units <= 1024) NO_NORM_AS(T, 256, 256, 4);                                                                                          \
        /* (3000 x 16384 bf16 with grad_sum 165 us; 1024 lanes, whose registers do not hold it, 260) */                                             \
        else if (units <= 2048) NO_NORM_AS(T, 512, 512, 4);                                                                                          \
        else if (sizeof(T) == 4 && units <= 4096) NO_NORM_AS(float, 1024, 1024, 4);                                                                  \
        else {                                                                                                                                       \
            direct = false;                                                                                                                          \
            room(n_rows_cap < 64 ? n_rows_cap : 64, false);                                                                                          \
            /* before the input gradient, which may overwrite what this reads */                                                                     \
            if (parts_w || parts_b)                                                                                                                  \
                hipLaunchKernelGGL(layernorm_wide_parts_kernel<T>, dim3((unsigned)ceil_div(dim, 256), (unsigned)n_parts), dim3(256), 0, st, s, d_mean, d_rstd, gy, d_n_rows, \
                                   n_rows_cap, dim, parts_w, parts_b);                                                                               \
            hipLaunchKernelGGL(layernorm_bwd_wide_kernel<T>, dim3((unsigned)layernorm_blocks(n_rows_cap, 1, 512)), dim3(1024), 0, st, s, d_weight, d_mean, d_rstd, gy, gs, \
                               d_n_rows, n_rows_cap, dim, gx);                                                                                       \
        }                                                                                                                                            \
    } while (0)
    if (n_rows_cap > 0) { if (dt == NO_F32) NO_NORM(float); else NO_NORM(bf16_t); }
    else room(0, true);
#undef NO_NORM
#undef NO_NORM_AS
    if ((d_grad_weight || d_grad_bias) && !(direct && n_parts == 1))
        hipLaunchKernelGGL(layernorm_join_kernel, dim3((unsigned)ceil_div(dim, 16), 2), dim3(1024), 0, st, parts_w, parts_b, (int32_t)n_parts, dim, d_grad_weight, d_grad_bias);
    return launch_status(who);
}
