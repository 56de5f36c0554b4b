// no_embed_fwd / no_embed_bwd: rows of a table by id, scaled, and the gradient of the table.
#include "rows.hpp"

namespace no {

template <typename T, typename O>
__global__ void __launch_bounds__(256) embed_fwd_kernel(RowsOf table, int64_t n_rows, int32_t dim, const float* row_scale, const int32_t* ids,
                                                        const int32_t* d_n, int32_t cap, float scale, RowsOf out) {
    const int32_t n = rows_here(d_n, cap);
    for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
        const int32_t id = ids[i];
        const bool there = id >= 0 && id < n_rows;
        const float by = there ? (row_scale ? scale * row_scale[id] : scale) : 0.0f;
        for (int32_t c = threadIdx.x; c < dim; c += 256) out.row<O>(i)[c] = there ? from_f32<O>(to_f32(table.row<T>(id)[c]) * by) : from_f32<O>(0.0f);
    }
}

// A block a table row: walks all ids.
template <typename T>
__global__ void __launch_bounds__(256) embed_bwd_kernel(RowsOf grad, const int32_t* ids, const int32_t* d_n, int32_t cap, float scale, bool accumulate,
                                                        RowsOf table, int64_t n_rows, int32_t dim) {
    const int32_t n = rows_here(d_n, cap);
    for (int64_t v = blockIdx.x; v < n_rows; v += gridDim.x)
        for (int32_t c = threadIdx.x; c < dim; c += 256) {
            float sum = 0.0f;
            bool any = false;
            for (int32_t i = 0; i < n; ++i)
                if (ids[i] == v) { sum += to_f32(grad.row<T>(i)[c]); any = true; }
            float* to = table.row<float>(v) + c;
            if (accumulate) { if (any) *to += scale * sum; }
            else *to = scale * sum;
        }
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
    NO_CHECK(check_rows("no_embed_fwd", "table", d_table, dt, n_rows, dim, table_stride_bytes));
    NO_CHECK(check_rows("no_embed_fwd", "out", d_out, dt_out, n_ids_cap, dim, out_stride_bytes));
    if (n_ids_cap == 0) return NO_OK;
    NO_REQUIRE(d_ids, NO_ERR_INVALID_ARG, "no_embed_fwd: ids are NULL");
    const RowsOf table = rows_of(d_table, table_stride_bytes), out = rows_of(d_out, out_stride_bytes);
    const dim3 grid((unsigned)(n_ids_cap < 65536 ? n_ids_cap : 65536));
#define NO_EMBED(T, O) hipLaunchKernelGGL((embed_fwd_kernel<T, O>), grid, dim3(256), 0, (hipStream_t)stream, table, n_rows, dim, d_row_scale, d_ids, d_n_ids, n_ids_cap, scale, out)
    if (dt_out == NO_F32) { if (dt == NO_F32) NO_EMBED(float, float); else if (dt == NO_BF16) NO_EMBED(bf16_t, float); else NO_EMBED(e4m3_t, float); }
    else { if (dt == NO_F32) NO_EMBED(float, bf16_t); else if (dt == NO_BF16) NO_EMBED(bf16_t, bf16_t); else NO_EMBED(e4m3_t, bf16_t); }
#undef NO_EMBED
    return launch_status("no_embed_fwd");
}

extern "C" size_t no_embed_ws_bytes(int32_t n_ids_cap, int32_t dim) {
    if (n_ids_cap < 0 || dim < 1) return 0;
    return 16;
}

extern "C" int32_t no_embed_bwd(const void* d_grad_out, no_dtype dt, int64_t grad_stride_bytes, const int32_t* d_ids, const int32_t* d_n_ids,
                                int32_t n_ids_cap, float scale, int32_t accumulate, float* d_grad_table, int64_t n_rows, int32_t dim,
                                int64_t table_stride_bytes, void* d_ws, size_t ws_bytes, void* stream) {
    clear_error();
    NO_REQUIRE(dt == NO_F32 || dt == NO_BF16, NO_ERR_INVALID_ARG, "no_embed_bwd: gradients are NO_F32 or NO_BF16");
    NO_REQUIRE(n_rows >= 1 && n_rows <= INT32_MAX && dim >= 1 && n_ids_cap >= 0, NO_ERR_INVALID_ARG, "no_embed_bwd: bad sizes");
    NO_CHECK(check_rows("no_embed_bwd", "grad_out", d_grad_out, dt, n_ids_cap, dim, grad_stride_bytes));
    NO_CHECK(check_rows("no_embed_bwd", "grad_table", d_grad_table, NO_F32, n_rows, dim, table_stride_bytes));
    NO_REQUIRE(d_ids || n_ids_cap == 0, NO_ERR_INVALID_ARG, "no_embed_bwd: ids are NULL");
    NO_REQUIRE(d_ws && (uintptr_t)d_ws % 16 == 0, NO_ERR_INVALID_ARG, "no_embed_bwd: the workspace is NULL or misaligned");
    NO_REQUIRE(ws_bytes >= no_embed_ws_bytes(n_ids_cap, dim), NO_ERR_CAPACITY, "no_embed_bwd: workspace too small");
    const dim3 grid((unsigned)(n_rows < 65536 ? n_rows : 65536));
    const RowsOf grad = rows_of(d_grad_out, grad_stride_bytes), table = rows_of(d_grad_table, table_stride_bytes);
#define NO_EMBED(T) hipLaunchKernelGGL(embed_bwd_kernel<T>, grid, dim3(256), 0, (hipStream_t)stream, grad, d_ids, d_n_ids, n_ids_cap, scale, accumulate != 0, table, n_rows, dim)
    if (dt == NO_F32) NO_EMBED(float); else NO_EMBED(bf16_t);
#undef NO_EMBED
    return launch_status("no_embed_bwd");
}
