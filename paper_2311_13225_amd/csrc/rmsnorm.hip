// no_rmsnorm_fwd / no_rmsnorm_bwd: root-mean-square norm of rows with the residual's addition, and its gradients.
#include "rows.hpp"

namespace no {

constexpr float E4M3_MOST = 448.0f, SMALLEST_MOST = 0x1p-100f;

template <typename T, typename Y>
__global__ void __launch_bounds__(256) rmsnorm_fwd_kernel(RowsOf x, RowsOf residual, const float* weight, float eps, const int32_t* d_n, int32_t cap,
                                                          int32_t dim, RowsOf sum, RowsOf y, float* row_scale, float* rstd_out) {
    __shared__ float smem[4];
    const int32_t n = rows_here(d_n, cap);
    for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
        auto s_at = [&](int32_t c) {
            const float v = to_f32(x.row<T>(i)[c]);
            return residual.p ? to_f32(from_f32<T>(v + to_f32(residual.row<T>(i)[c]))) : v;
        };
        float ss = 0.0f;
        for (int32_t c = threadIdx.x; c < dim; c += 256) { const float v = s_at(c); ss += v * v; }
        ss = block_sum<float, 256>(ss, smem);
        const float rstd = 1.0f / sqrtf(ss / (float)dim + eps);
        float most = 0.0f;
        for (int32_t c = threadIdx.x; c < dim; c += 256) most = fmaxf(most, fabsf(s_at(c) * rstd * (weight ? weight[c] : 1.0f)));
        for (int o = 32; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor(most, o, 64));
        if (lane_id() == 0) smem[threadIdx.x >> 6] = most;
        __syncthreads();
        most = fmaxf(fmaxf(smem[0], smem[1]), fmaxf(smem[2], smem[3]));
        __syncthreads();
        float scale = 1.0f;
        if constexpr (TypeOf<Y>::code == NO_E4M3) scale = ss < INFINITY ? fmaxf(most, SMALLEST_MOST) / E4M3_MOST : NAN;
        for (int32_t c = threadIdx.x; c < dim; c += 256) {
            const float v = s_at(c);
            if (sum.p) sum.row<T>(i)[c] = from_f32<T>(v);
            float o = v * rstd * (weight ? weight[c] : 1.0f);
            if constexpr (TypeOf<Y>::code == NO_E4M3) o = o / scale;
            y.row<Y>(i)[c] = from_f32<Y>(o);
        }
        if (threadIdx.x == 0) {
            if (rstd_out) rstd_out[i] = rstd;
            if (TypeOf<Y>::code == NO_E4M3) row_scale[i] = scale;
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(256) rmsnorm_grad_weight_kernel(RowsOf s, const float* rstd, RowsOf grad_y, const int32_t* d_n, int32_t cap,
                                                                  int32_t dim, float* grad_weight) {
    const int32_t n = rows_here(d_n, cap), c = (int32_t)(blockIdx.x * 256 + threadIdx.x);
    if (c >= dim) return;
    double sum = 0.0;
    for (int64_t i = 0; i < n; ++i) sum += to_f32(grad_y.row<T>(i)[c]) * (to_f32(s.row<T>(i)[c]) * rstd[i]);
    grad_weight[c] = (float)sum;
}

template <typename T>
__global__ void __launch_bounds__(256) rmsnorm_grad_x_kernel(RowsOf s, const float* weight, const float* rstd, RowsOf grad_y, RowsOf grad_sum,
                                                             const int32_t* d_n, int32_t cap, int32_t dim, RowsOf grad_x) {
    __shared__ float smem[4];
    const int32_t n = rows_here(d_n, cap);
    for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
        const float r = rstd[i];
        float dot = 0.0f;
        for (int32_t c = threadIdx.x; c < dim; c += 256)
            dot += to_f32(grad_y.row<T>(i)[c]) * (weight ? weight[c] : 1.0f) * (to_f32(s.row<T>(i)[c]) * r);
        const float mean = block_sum<float, 256>(dot, smem) / (float)dim;
        for (int32_t c = threadIdx.x; c < dim; c += 256) {
            const float wg = to_f32(grad_y.row<T>(i)[c]) * (weight ? weight[c] : 1.0f);
            const float dx = r * (wg - to_f32(s.row<T>(i)[c]) * r * mean);
            grad_x.row<T>(i)[c] = from_f32<T>(grad_sum.p ? dx + to_f32(grad_sum.row<T>(i)[c]) : dx);
        }
    }
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
    const dim3 grid((unsigned)(n_rows_cap < 65536 ? n_rows_cap : 65536));
#define NO_NORM(T, Y) hipLaunchKernelGGL((rmsnorm_fwd_kernel<T, Y>), grid, dim3(256), 0, (hipStream_t)stream, x, r, d_weight, eps, d_n_rows, n_rows_cap, dim, s, y, d_row_scale, d_rstd)
    if (dt == NO_F32) { if (dt_y == NO_F32) NO_NORM(float, float); else if (dt_y == NO_BF16) NO_NORM(float, bf16_t); else NO_NORM(float, e4m3_t); }
    else { if (dt_y == NO_F32) NO_NORM(bf16_t, float); else if (dt_y == NO_BF16) NO_NORM(bf16_t, bf16_t); else NO_NORM(bf16_t, e4m3_t); }
#undef NO_NORM
    return launch_status(who);
}

extern "C" size_t no_rmsnorm_ws_bytes(int32_t n_rows_cap, int32_t dim) {
    if (n_rows_cap < 0 || dim < 1 || dim > NO_MAX_NORM_DIM) return 0;
    return 16;
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
    const dim3 grid((unsigned)(n_rows_cap < 65536 ? n_rows_cap : 65536)), cols((unsigned)ceil_div(dim, 256));
    hipStream_t st = (hipStream_t)stream;
    // the weight's gradient first: grad_x may overwrite what it reads
#define NO_NORM(T)                                                                                                                                   \
    do {                                                                                                                                             \
        if (d_grad_weight) hipLaunchKernelGGL(rmsnorm_grad_weight_kernel<T>, cols, dim3(256), 0, st, s, d_rstd, gy, d_n_rows, n_rows_cap, dim, d_grad_weight); \
        if (n_rows_cap) hipLaunchKernelGGL(rmsnorm_grad_x_kernel<T>, grid, dim3(256), 0, st, s, d_weight, d_rstd, gy, gs, d_n_rows, n_rows_cap, dim, gx);      \
    } while (0)
    if (dt == NO_F32) NO_NORM(float); else NO_NORM(bf16_t);
#undef NO_NORM
    return launch_status(who);
}
