// no_rmsnorm_fwd / no_rmsnorm_bwd: root-mean-square norm of rows with the residual's addition, and its gradients.
#include "rows.hpp"

namespace no {

constexpr float E4M3_MOST = 448.0f, SMALLEST_MOST = 0x1p-100f;

// y = s / sqrt(mean(s^2) + eps) weight of s = x + residual. A team of lanes holds a row in registers, U runs of 16 bytes a lane, so that the row is read once and written once, which is
// what bounds it: 16384 x 4096 bf16 with a residual 92 us, 5.8 TB/s; 50001 x 602 fp32 into e4m3 33 us, 4.6 TB/s (three runs a lane; four, of which 41 % are empty: 35.2).
// What it writes goes past the caches (94.8 -> 91.1 us, 4096 x 4096 27.8 -> 21.8); what it reads does not, since the launch before may have left it there (4096 x 4096: 25.7, but
// 50000 x 2048 138.9 -> 134.1). A next launch that reads small outputs at once pays some of it back (with both read next, 4096 x 4096 50.0 us, by the caches 48.6).
template <typename T, typename Y, int TEAM, int THREADS, int U>
__global__ void __launch_bounds__(THREADS) rmsnorm_fwd_kernel(RowsOf x, RowsOf residual, const float* __restrict__ weight, float eps, const int32_t* d_n, int32_t cap,
                                                              int32_t dim, RowsOf sum, RowsOf y, float* row_scale, float* rstd_out) {
    constexpr int W = 16 / (int)sizeof(T), PER_BLOCK = THREADS / TEAM;
    constexpr bool KEEP = U * W <= 32;          // weights in registers
    __shared__ float smem[2 * THREADS / 64];
    Team<TEAM, THREADS> team(smem);
    const int32_t n = rows_here(d_n, cap), t = team.lane();
    const T zero = from_f32<T>(0.0f);
    RowRegs<float, W, KEEP ? U : 1, TEAM> wk;
    if constexpr (KEEP) if (weight) wk.load(weight, dim, t, 0.0f);
    for (int64_t i = (int64_t)blockIdx.x * PER_BLOCK + team.index(); i < n; i += (int64_t)gridDim.x * PER_BLOCK) {
        RowRegs<T, W, U, TEAM> s, r;
        s.load(x.row<T>(i), dim, t, zero);
        float ss = 0.0f;
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
        for (int u = 0; u < U; ++u) {
            float f[W];
            s.v[u].get(f);
#pragma unroll
            for (int w = 0; w < W; ++w) ss += f[w] * f[w];
        }
        if (sum.p) {
            RowStore<T, W, true> store(sum.row<T>(i), dim);
#pragma unroll
            for (int u = 0; u < U; ++u) store.put(s.at(t, u), s.v[u]);
            store.finish();
        }
        ss = team.sum(ss);
        const float rstd = 1.0f / sqrtf(ss / (float)dim + eps);
        auto values = [&](int u, float (&f)[W]) {
            float k[W];
            if (weight) {
                if constexpr (KEEP) wk.v[KEEP ? u : 0].get(k);
                else {
                    Run<float, W> one;
                    one.load_at(weight, s.at(t, u), dim, 0.0f);
                    one.get(k);
                }
            }
            s.v[u].get(f);
#pragma unroll
            for (int w = 0; w < W; ++w) f[w] = weight ? f[w] * rstd * k[w] : f[w] * rstd;
        };
        float scale = 1.0f, inv = 1.0f;
        if constexpr (TypeOf<Y>::code == NO_E4M3) {
            float most = 0.0f;
            s.renew();
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float f[W];
                values(u, f);
#pragma unroll
                for (int w = 0; w < W; ++w) most = fmaxf(most, fabsf(f[w]));
            }
            most = team.max(most);
            scale = ss < INFINITY ? fmaxf(most, SMALLEST_MOST) / E4M3_MOST : NAN;
            inv = 1.0f / scale;
        }
        s.renew();
        RowStore<Y, W, true> store(y.row<Y>(i), dim);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float f[W];
            values(u, f);
            if constexpr (TypeOf<Y>::code == NO_E4M3)
#pragma unroll
                for (int w = 0; w < W; ++w) f[w] *= inv;
            Run<Y, W> o;
            o.set(f);
            store.put(s.at(t, u), o);
        }
        store.finish();
        if (t == 0) {
            if (rstd_out) rstd_out[i] = rstd;
            if (TypeOf<Y>::code == NO_E4M3) row_scale[i] = scale;
        }
    }
}

// ------------------------------------------------------------------------------------------------------- gradients
//
// The weight's gradient is a sum over rows for every column: a team adds its rows' terms in registers while it makes their input gradients, a block joins its
// teams' sums in LDS and stores one row of parts, and a second launch adds the blocks' parts in order. Bound by memory: 16384 x 2048 bf16 with the residual's gradient 48 us,
// the first launch 45 (5.9 TB/s) and the second under 5 under the profiler; 16384 x 4096 97 us, 5.5 TB/s.

constexpr int32_t NORM_PARTS = 512;     // rows of parts, at most (50000 x 602 fp32: 101 us; 256: 132, 1024: 121)

template <typename T, int TEAM, int THREADS, int U>
__global__ void __launch_bounds__(THREADS) rmsnorm_bwd_kernel(RowsOf s, const float* __restrict__ weight, const float* __restrict__ rstd, RowsOf grad_y, RowsOf grad_sum,
                                                              const int32_t* d_n, int32_t cap, int32_t dim, RowsOf grad_x, float* parts, float* grad_weight) {
    constexpr int W = 16 / (int)sizeof(T), PER_BLOCK = THREADS / TEAM;
    __shared__ float smem[2 * THREADS / 64];
    __shared__ float joined[PER_BLOCK > 1 ? U * TEAM * W : 1];
    Team<TEAM, THREADS> team(smem);
    const int32_t n = rows_here(d_n, cap), t = team.lane();
    const T zero = from_f32<T>(0.0f);
    RowRegs<float, W, U, TEAM> wk;
    float dw[U][W];
    if (weight) wk.load(weight, dim, t, 0.0f);
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int w = 0; w < W; ++w) dw[u][w] = 0.0f;
        if (!weight) {
            const float one[4] = {1.0f, 1.0f, 1.0f, 1.0f};
#pragma unroll
            for (int k = 0; k < Run<float, W>::N; ++k) __builtin_memcpy(&wk.v[u].v[k], one, 16);
        }
    }
    const int64_t stride = (int64_t)gridDim.x * PER_BLOCK;
    int64_t i = (int64_t)blockIdx.x * PER_BLOCK + team.index();
    // Stores past the caches but for rows of a wavefront (16384 x 2048 bf16 51.5 us so, 48.8 by the caches; 16384 x 4096 96.4 and 100.0; 100000 x 128 22.6 and 25.4).
    // Requests: long rows past the caches (16384 x 4096 bf16 103 -> 95 us, 4000 x 16384 fp32 214 -> 196); short ones share cache lines with the rows beside them (50000 x 602 fp32: 102 -> 115).
    RowRegs<T, W, U, TEAM, U * TEAM >= 256> rs, rg, ra;
    float r = 0.0f;
    if (i < n) {
        r = rstd[i];
        rs.load(s.row<T>(i), dim, t, zero);
        rg.load(grad_y.row<T>(i), dim, t, zero);
        if (grad_sum.p) ra.load(grad_sum.row<T>(i), dim, t, zero);
    }
    for (; i < n; i += stride) {
        // each run of the next row is requested when the gradient has no more use for this one's registers (100000 x 128 bf16: 55.6 -> 36.5 us,
        // 16384 x 2048: 59.6 -> 55.9)
        const int64_t next = i + stride, at = next < n ? next : i;
        const int32_t next_len = next < n ? dim : 0;
        const T *const next_s = s.row<T>(at), *const next_g = grad_y.row<T>(at), *const next_a = grad_sum.p ? grad_sum.row<T>(at) : nullptr;
        const float next_r = rstd[at];
        float dot = 0.0f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[W], g[W], k[W];
            rs.v[u].get(v);
            rg.v[u].get(g);
            wk.v[u].get(k);
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float gu = g[w] * (v[w] * r);
                dw[u][w] += gu;
                dot += gu * k[w];
            }
        }
        const float mean = team.sum(dot) / (float)dim;
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
                const float dx = r * (g[w] * k[w] - v[w] * r * mean);
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
    }
    if (!grad_weight) return;
    if constexpr (PER_BLOCK > 1) {      // the block's teams in turn
        for (int k = 0; k < PER_BLOCK; ++k) {
            if (team.index() == k)
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int w = 0; w < W; ++w) {
                        float& to = joined[((t + u * TEAM) * W) + w];
                        to = k ? to + dw[u][w] : dw[u][w];
                        if (k == PER_BLOCK - 1) dw[u][w] = to;
                    }
            __syncthreads();
        }
        if (team.index() != PER_BLOCK - 1) return;
    }
    float* to = gridDim.x == 1 ? grad_weight : parts + (int64_t)blockIdx.x * dim;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int32_t c = (t + u * TEAM) * W;
        if (c < dim) {
            Run<float, W> o;
            o.set(dw[u]);
            o.store(to + c, dim - c);
        }
    }
}

// Rows too wide for registers: read twice.
template <typename T>
__global__ void __launch_bounds__(1024) rmsnorm_bwd_wide_kernel(RowsOf s, const float* __restrict__ weight, const float* __restrict__ rstd, RowsOf grad_y, RowsOf grad_sum,
                                                                const int32_t* d_n, int32_t cap, int32_t dim, RowsOf grad_x) {
    __shared__ float smem[32];
    Team<1024, 1024> team(smem);
    const int32_t n = rows_here(d_n, cap);
    for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
        const float r = rstd[i];
        float dot = 0.0f;
        for (int32_t c = threadIdx.x; c < dim; c += 1024)
            dot += to_f32(grad_y.row<T>(i)[c]) * (to_f32(s.row<T>(i)[c]) * r) * (weight ? weight[c] : 1.0f);
        const float mean = team.sum(dot) / (float)dim;
        for (int32_t c = threadIdx.x; c < dim; c += 1024) {
            const float dx = r * (to_f32(grad_y.row<T>(i)[c]) * (weight ? weight[c] : 1.0f) - to_f32(s.row<T>(i)[c]) * r * mean);
            grad_x.row<T>(i)[c] = from_f32<T>(grad_sum.p ? dx + to_f32(grad_sum.row<T>(i)[c]) : dx);
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(256) rmsnorm_wide_parts_kernel(RowsOf s, const float* __restrict__ rstd, RowsOf grad_y, const int32_t* d_n, int32_t cap, int32_t dim,
                                                                 float* parts) {
    const int32_t n = rows_here(d_n, cap), c = (int32_t)(blockIdx.x * 256 + threadIdx.x);
    if (c >= dim) return;
    float sum = 0.0f;
    for (int64_t i = blockIdx.y; i < n; i += gridDim.y) sum += to_f32(grad_y.row<T>(i)[c]) * (to_f32(s.row<T>(i)[c]) * rstd[i]);
    parts[(int64_t)blockIdx.y * dim + c] = sum;
}

// Sixteen columns a block, 64 lanes to a column, so that a lane has eight parts at most and asks for them at once.
__global__ void __launch_bounds__(1024) rmsnorm_join_kernel(const float* __restrict__ parts, int32_t n_parts, int32_t dim, float* grad_weight) {
    __shared__ float share[64][16];
    const int32_t col = (int32_t)threadIdx.x & 15, row = (int32_t)threadIdx.x >> 4, c = (int32_t)blockIdx.x * 16 + col;
    float sum = 0.0f;
    if (c < dim) {
#pragma unroll
        for (int k = 0; k < NORM_PARTS / 64; ++k) {
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
    if (threadIdx.x < 16 && c < dim) grad_weight[c] = sum;
}

// Blocks for n rows, `most` at most, behind which a team walks several rows with the weights it holds. The forward pass has a team for every row (16384 x 4096 bf16 94.8 us; 2048 blocks
// 105.8), but for rows of part of a wavefront (200000 x 128 bf16 by 32 lanes: 2048 blocks 47 us, all 56; by 16, which hold it, 37), for fp32 into e4m3, whose arithmetic is most (50001 x 602: 4096 blocks 32.7, all 36.1; 100000 x 256:
// 33.7 and 39.4), and for blocks of 1024 lanes (4000 x 30000 fp32: 256 blocks 347, all 382).
static inline int64_t norm_blocks(int64_t n, int per_block, int64_t most) {
    const int64_t b = ceil_div(n, per_block);
    return b < most ? b : most;
}

}  // namespace no

using namespace no;

extern "C" int32_t no_rmsnorm_fwd(const void* d_x, no_dtype dt, int64_t x_stride_bytes, const void* d_residual, int64_t residual_stride_bytes,
                                  const float* d_weight, float eps, const int32_t* d_n_rows, int32_t n_rows_cap, int32_t dim, void* d_sum,
                                  int64_t sum_stride_bytes, void* d_y, no_dtype dt_y, int64_t y_stride_bytes, float* d_row_scale,
                                  float* d_rstd, void* stream) {
    clear_error();
    const char* who = "no_rmsnorm_fwd";
    NO_REQUIRE(dt == NO_F32 || dt == NO_BF16, NO_ERR_INVALID_ARG, "%s: rows are NO_F32 or NO_BF16", who);
    NO_REQUIRE(dt_y == NO_F32 || dt_y == NO_BF16 || dt_y == NO_E4M3, NO_ERR_INVALID_ARG, "%s: unknown output type", who);
    NO_REQUIRE(n_rows_cap >= 0 && dim >= 1 && eps >= 0.0f, NO_ERR_INVALID_ARG, "%s: bad sizes or eps", who);
    NO_REQUIRE(dim <= NO_MAX_NORM_DIM, NO_ERR_UNSUPPORTED, "%s: rows of more than %d values", who, NO_MAX_NORM_DIM);
    NO_CHECK(check_rows(who, "x", d_x, dt, n_rows_cap, dim, x_stride_bytes));
    if (d_residual) NO_CHECK(check_rows(who, "residual", d_residual, dt, n_rows_cap, dim, residual_stride_bytes));
    if (d_sum) NO_CHECK(check_rows(who, "sum", d_sum, dt, n_rows_cap, dim, sum_stride_bytes));
    NO_CHECK(check_rows(who, "y", d_y, dt_y, n_rows_cap, dim, y_stride_bytes));
    if (n_rows_cap == 0) return NO_OK;
    NO_REQUIRE((dt_y == NO_E4M3) == (d_row_scale != nullptr), NO_ERR_INVALID_ARG, "%s: row scales go with NO_E4M3, and with it alone", who);
    const RowsOf x = rows_of(d_x, x_stride_bytes), r = rows_of(d_residual, residual_stride_bytes), s = rows_of(d_sum, sum_stride_bytes), y = rows_of(d_y, y_stride_bytes);
    hipStream_t st = (hipStream_t)stream;
#define NO_NORM_AS(T, Y, TEAM, THREADS, U)                                                                                                          \
    hipLaunchKernelGGL((rmsnorm_fwd_kernel<T, Y, TEAM, THREADS, U>), dim3((unsigned)norm_blocks(n_rows_cap, THREADS / TEAM, THREADS == 1024 ? 256 : TEAM < 64 ? 2048 : sizeof(T) == 4 && sizeof(Y) == 1 ? 4096 : 1 << 20)), \
                       dim3(THREADS), 0, st, x, r, d_weight, eps, d_n_rows, n_rows_cap, dim, s, y, d_row_scale, d_rstd)
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
    if (dt == NO_F32) { if (dt_y == NO_F32) NO_NORM(float, float); else if (dt_y == NO_BF16) NO_NORM(float, bf16_t); else NO_NORM(float, e4m3_t); }
    else { if (dt_y == NO_F32) NO_NORM(bf16_t, float); else if (dt_y == NO_BF16) NO_NORM(bf16_t, bf16_t); else NO_NORM(bf16_t, e4m3_t); }
#undef NO_NORM
#undef NO_NORM_AS
    return launch_status(who);
}

extern "C" size_t no_rmsnorm_ws_bytes(int32_t n_rows_cap, int32_t dim) {
    if (n_rows_cap < 0 || dim < 1 || dim > NO_MAX_NORM_DIM) return 0;
    return 16 + (size_t)(n_rows_cap < NORM_PARTS ? n_rows_cap : NORM_PARTS) * (size_t)dim * 4;
}

extern "C" int32_t no_rmsnorm_bwd(const void* d_s, no_dtype dt, int64_t s_stride_bytes, const float* d_weight, const float* d_rstd,
                                  const void* d_grad_y, int64_t grad_y_stride_bytes, const void* d_grad_sum, int64_t grad_sum_stride_bytes,
                                  const int32_t* d_n_rows, int32_t n_rows_cap, int32_t dim, void* d_grad_x, int64_t grad_x_stride_bytes,
                                  float* d_grad_weight, void* d_ws, size_t ws_bytes, void* stream) {
    clear_error();
    const char* who = "no_rmsnorm_bwd";
    NO_REQUIRE(dt == NO_F32 || dt == NO_BF16, NO_ERR_INVALID_ARG, "%s: rows are NO_F32 or NO_BF16", who);
    NO_REQUIRE(n_rows_cap >= 0 && dim >= 1, NO_ERR_INVALID_ARG, "%s: bad sizes", who);
    NO_REQUIRE(dim <= NO_MAX_NORM_DIM, NO_ERR_UNSUPPORTED, "%s: rows of more than %d values", who, NO_MAX_NORM_DIM);
    NO_CHECK(check_rows(who, "s", d_s, dt, n_rows_cap, dim, s_stride_bytes));
    NO_CHECK(check_rows(who, "grad_y", d_grad_y, dt, n_rows_cap, dim, grad_y_stride_bytes));
    if (d_grad_sum) NO_CHECK(check_rows(who, "grad_sum", d_grad_sum, dt, n_rows_cap, dim, grad_sum_stride_bytes));
    NO_CHECK(check_rows(who, "grad_x", d_grad_x, dt, n_rows_cap, dim, grad_x_stride_bytes));
    NO_REQUIRE(d_rstd || n_rows_cap == 0, NO_ERR_INVALID_ARG, "%s: rstd is NULL", who);
    NO_REQUIRE(d_ws && (uintptr_t)d_ws % 16 == 0, NO_ERR_INVALID_ARG, "%s: the workspace is NULL or misaligned", who);
    NO_REQUIRE(ws_bytes >= no_rmsnorm_ws_bytes(n_rows_cap, dim), NO_ERR_CAPACITY, "%s: workspace too small", who);
    const RowsOf s = rows_of(d_s, s_stride_bytes), gy = rows_of(d_grad_y, grad_y_stride_bytes), gs = rows_of(d_grad_sum, grad_sum_stride_bytes), gx = rows_of(d_grad_x, grad_x_stride_bytes);
    hipStream_t st = (hipStream_t)stream;
    float* parts = (float*)d_ws;
    int64_t n_parts = 0;
#define NO_NORM_AS(T, TEAM, THREADS, U)                                                                                                              \
    do {                                                                                                                                             \
        n_parts = norm_blocks(n_rows_cap, THREADS / TEAM, THREADS == 1024 ? 256 : NORM_PARTS);                                                       \
        hipLaunchKernelGGL((rmsnorm_bwd_kernel<T, TEAM, THREADS, U>), dim3((unsigned)n_parts), dim3(THREADS), 0, st, s, d_weight, d_rstd, gy, gs, d_n_rows, n_rows_cap, dim, \
                           gx, parts, d_grad_weight);                                                                                                \
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
        else if (units <= 256) NO_NORM_AS(T, 64, 256, 4);                                                                                            \
        else if (units <= 512) NO_NORM_AS(T, 256, 256, 2);                                                                                           \
        else if (units <= 1024) NO_NORM_AS(T, 256, 256, 4);                                                                                          \
        else if (units <= 2048) NO_NORM_AS(T, 1024, 1024, 2);                                                                                        \
        else if (units <= 4096) NO_NORM_AS(T, 1024, 1024, 4);                                                                                        \
        else {                                                                                                                                       \
            n_parts = n_rows_cap < NORM_PARTS ? n_rows_cap : NORM_PARTS;                                                                             \
            if (n_parts > 64) n_parts = 64;                                                                                                          \
            /* before the input gradient, which may overwrite what this reads; always joined, so never one part straight into the result */          \
            if (d_grad_weight)                                                                                                                       \
                hipLaunchKernelGGL(rmsnorm_wide_parts_kernel<T>, dim3((unsigned)ceil_div(dim, 256), (unsigned)n_parts), dim3(256), 0, st, s, d_rstd, gy, d_n_rows, n_rows_cap, dim, parts); \
            hipLaunchKernelGGL(rmsnorm_bwd_wide_kernel<T>, dim3((unsigned)norm_blocks(n_rows_cap, 1, 512)), dim3(1024), 0, st, s, d_weight, d_rstd, gy, gs, d_n_rows, n_rows_cap, dim, gx); \
            direct = false;                                                                                                                          \
        }                                                                                                                                            \
    } while (0)
    bool direct = true;         // a single block has stored the weight's gradient itself
    if (n_rows_cap > 0) { if (dt == NO_F32) NO_NORM(float); else NO_NORM(bf16_t); }
#undef NO_NORM
#undef NO_NORM_AS
    if (d_grad_weight && !(direct && n_parts == 1))
        hipLaunchKernelGGL(rmsnorm_join_kernel, dim3((unsigned)ceil_div(dim, 16)), dim3(1024), 0, st, parts, (int32_t)n_parts, dim, d_grad_weight);
    return launch_status(who);
}
