// no_distill_* and no_logprobs_*: one pass or two over rows of logits.
#include "rows.hpp"

namespace no {

__device__ __forceinline__ float block_max(float v, float* smem) {
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    if (lane_id() == 0) smem[threadIdx.x >> 6] = v;
    __syncthreads();
    v = fmaxf(fmaxf(smem[0], smem[1]), fmaxf(smem[2], smem[3]));
    __syncthreads();
    return v;
}

// Largest logit (0 where there is none above -inf), sum of exponentials, sum of e * (z - m).
struct RowSums { float m, s, h; bool none; };

template <typename T>
__device__ RowSums row_sums(const T* z, int32_t classes, float inv_t, float* smem) {
    RowSums r;
    float m = -INFINITY;
    for (int32_t c = threadIdx.x; c < classes; c += 256) m = fmaxf(m, to_f32(z[c]));
    m = block_max(m, smem);
    float s = 0.0f, h = 0.0f;
    const float from = m == -INFINITY ? 0.0f : m;
    for (int32_t c = threadIdx.x; c < classes; c += 256) {
        const float d = (to_f32(z[c]) - from) * inv_t, e = expf(d);
        s += e;
        if (e != 0.0f) h += e * d;
    }
    r.s = block_sum<float, 256>(s, smem);
    r.h = block_sum<float, 256>(h, smem);
    r.none = r.s == 0.0f;
    r.m = from;
    return r;
}

// The teacher's shares of a row into p[k] (0 for entries that are left out); ids_out[k] = -1 for those. Returns whether there are any.
__device__ bool teacher_shares(const int32_t* ids, const float* logits, int32_t k, int32_t classes, float inv_t, float* p, float* log_p, int32_t* ids_out,
                               float* smem) {
    const int j = threadIdx.x;
    const int32_t id = j < k ? ids[j] : -1;
    const bool there = id >= 0 && id < classes;
    const float t = there ? logits[j] * inv_t : -INFINITY;
    const float m = block_max(t, smem), from = m == -INFINITY ? 0.0f : m;
    const float e = there ? expf(t - from) : 0.0f, s = block_sum<float, 256>(e, smem);
    if (j < k) {
        p[j] = s == 0.0f ? 0.0f : e / s;
        log_p[j] = t - from - logf(s);
        ids_out[j] = there ? id : -1;
    }
    __syncthreads();
    return s != 0.0f;
}

template <typename T>
__global__ void __launch_bounds__(256) distill_kernel(RowsOf z, const int32_t* d_n, int32_t cap, int32_t classes, const int32_t* t_ids, const float* t_logits,
                                                      int32_t k, float temperature, const float* weight, float* loss, const float* lse_in, float* lse_out, RowsOf grad) {
    __shared__ float smem[4], p[256], log_p[256], at[256];
    __shared__ int32_t ids[256];
    const int32_t n = rows_here(d_n, cap);
    const float inv_t = 1.0f / temperature;
    for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
        const T* row = z.row<T>(i);
        const float w = weight ? weight[i] : 1.0f;
        const bool any = teacher_shares(t_ids + i * k, t_logits + i * k, k, classes, inv_t, p, log_p, ids, smem);
        if ((int)threadIdx.x < k) at[threadIdx.x] = ids[threadIdx.x] >= 0 ? to_f32(row[ids[threadIdx.x]]) : 0.0f;
        RowSums r{0, 0, 0, false};
        float log_s = 0.0f;
        if (!lse_in) {
            r = row_sums(row, classes, inv_t, smem);
            log_s = logf(r.s);
            if (threadIdx.x == 0 && lse_out) lse_out[i] = r.m * inv_t + log_s;
        }
        __syncthreads();
        if (loss) {
            const int j = threadIdx.x;
            float term = 0.0f;
            if (j < k && p[j] != 0.0f) term = p[j] * (log_p[j] - (r.none ? -INFINITY : (at[j] - r.m) * inv_t - log_s));
            const float sum = block_sum<float, 256>(term, smem);
            if (j == 0) loss[i] = w == 0.0f || !any ? 0.0f : w * temperature * temperature * sum;
        }
        if (grad.p) {
            T* out = grad.row<T>(i);
            const float by = w * temperature, lse = lse_in ? lse_in[i] : 0.0f, inv_s = 1.0f / r.s;
            auto q_of = [&](float v) { return v == -INFINITY ? 0.0f : lse_in ? expf(v * inv_t - lse) : expf((v - r.m) * inv_t) * inv_s; };
            for (int32_t c = threadIdx.x; c < classes; c += 256) out[c] = from_f32<T>(w == 0.0f || !any ? 0.0f : by * q_of(to_f32(row[c])));
            __syncthreads();
            const int j = threadIdx.x;
            if (j < k && ids[j] >= 0 && w != 0.0f && any) {
                float share = 0.0f;
                for (int32_t o = 0; o < k; ++o) if (ids[o] == ids[j]) share += p[o];
                out[ids[j]] = from_f32<T>(by * (q_of(at[j]) - share));
            }
        }
        __syncthreads();
    }
}

// Order of alternatives: larger value first, then the lower class.
__device__ __forceinline__ uint64_t order_key(float v, int32_t c) {
    const uint32_t b = __float_as_uint(v + 0.0f);                    // (-0 counts as 0)
    return (uint64_t)((b & 0x80000000u) ? ~b : b | 0x80000000u) << 32 | (uint32_t)~c;
}

template <typename T>
__global__ void __launch_bounds__(256) logprobs_fwd_kernel(RowsOf z, const int32_t* d_n, int32_t cap, int32_t classes, const int32_t* tokens, float temperature,
                                                           float* logprob, float* entropy, float* lse, int32_t k, int32_t* top_ids, float* top_logprobs) {
    __shared__ float smem[4];
    __shared__ uint64_t keys[4];
    const int32_t n = rows_here(d_n, cap);
    const float inv_t = 1.0f / temperature;
    for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
        const T* row = z.row<T>(i);
        const RowSums r = row_sums(row, classes, inv_t, smem);
        const float log_s = logf(r.s);
        auto log_of = [&](float v) { return v == -INFINITY && !(r.s != r.s) ? -INFINITY : (v - r.m) * inv_t - log_s; };
        if (threadIdx.x == 0) {
            const int32_t t = tokens[i];
            logprob[i] = t >= 0 && t < classes ? log_of(to_f32(row[t])) : 0.0f;
            entropy[i] = r.none ? 0.0f : log_s - r.h / r.s;
            lse[i] = r.m * inv_t + log_s;
        }
        uint64_t before = ~0ull;
        for (int32_t j = 0; j < k; ++j) {
            uint64_t best = 0;
            for (int32_t c = threadIdx.x; c < classes; c += 256) {
                const float v = to_f32(row[c]);
                const uint64_t key = v > -INFINITY ? order_key(v, c) : 0;
                if (key < before && key > best) best = key;
            }
            for (int o = 32; o > 0; o >>= 1) best = max(best, (uint64_t)__shfl_xor((unsigned long long)best, o, 64));
            if (lane_id() == 0) keys[threadIdx.x >> 6] = best;
            __syncthreads();
            best = max(max(keys[0], keys[1]), max(keys[2], keys[3]));
            __syncthreads();
            if (threadIdx.x == 0) {
                const int32_t c = best ? (int32_t)~(uint32_t)best : -1;
                top_ids[i * k + j] = r.s != r.s ? -1 : c;
                top_logprobs[i * k + j] = r.s != r.s ? NAN : c < 0 ? -INFINITY : log_of(to_f32(row[c]));
            }
            before = best ? best : 0;
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(256) logprobs_bwd_kernel(RowsOf z, const int32_t* d_n, int32_t cap, int32_t classes, const int32_t* tokens, float temperature,
                                                           const float* lse, const float* entropy, const float* g_logprob, const float* g_entropy, RowsOf grad) {
    const int32_t n = rows_here(d_n, cap);
    const float inv_t = 1.0f / temperature;
    for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
        const int32_t t = tokens[i];
        const float l = lse[i], h = entropy[i], gl = g_logprob && t >= 0 && t < classes ? g_logprob[i] : 0.0f, gh = g_entropy ? g_entropy[i] : 0.0f;
        for (int32_t c = threadIdx.x; c < classes; c += 256) {
            const float v = to_f32(z.row<T>(i)[c]);
            const float log_p = v * inv_t - l, p = v == -INFINITY ? 0.0f : expf(log_p);
            const float d = (c == t ? gl : 0.0f) - (p == 0.0f ? 0.0f : p * (gl + gh * (log_p + h)));
            grad.row<T>(i)[c] = from_f32<T>(d * inv_t);
        }
    }
}

static int32_t check_logits(const char* who, const void* z, no_dtype dt, int64_t stride, int32_t n, int32_t classes, float temperature) {
    NO_REQUIRE(dt == NO_F32 || dt == NO_BF16, NO_ERR_INVALID_ARG, "%s: logits are NO_F32 or NO_BF16", who);
    NO_REQUIRE(n >= 0 && classes >= 1, NO_ERR_INVALID_ARG, "%s: bad sizes", who);
    NO_REQUIRE(classes <= NO_MAX_CLASSES, NO_ERR_UNSUPPORTED, "%s: more than %d classes", who, NO_MAX_CLASSES);
    NO_REQUIRE(temperature > 0.0f && temperature < INFINITY, NO_ERR_INVALID_ARG, "%s: the temperature must be positive and finite", who);
    return check_rows(who, "z", z, dt, n, classes, stride);
}

static int32_t check_ws(const char* who, const void* ws, size_t bytes, size_t needed) {
    NO_REQUIRE(ws && (uintptr_t)ws % 16 == 0, NO_ERR_INVALID_ARG, "%s: the workspace is NULL or misaligned", who);
    NO_REQUIRE(bytes >= needed, NO_ERR_CAPACITY, "%s: workspace too small", who);
    return NO_OK;
}

static int32_t check_teacher(const char* who, int32_t n, const int32_t* ids, const float* logits, int32_t k) {
    NO_REQUIRE(k >= 1, NO_ERR_INVALID_ARG, "%s: a row has at least one teacher entry", who);
    NO_REQUIRE(k <= NO_MAX_TEACHER, NO_ERR_UNSUPPORTED, "%s: more than %d teacher entries a row", who, NO_MAX_TEACHER);
    NO_REQUIRE((ids && logits) || n == 0, NO_ERR_INVALID_ARG, "%s: the teacher's entries are NULL", who);
    return NO_OK;
}

static int32_t distill(const char* who, const void* z, no_dtype dt, int64_t stride, const int32_t* d_n, int32_t cap, int32_t classes, const int32_t* ids,
                       const float* logits, int32_t k, float temperature, const float* weight, float* loss, const float* lse_in, float* lse_out, void* grad,
                       int64_t grad_stride, hipStream_t st) {
    if (cap == 0) return NO_OK;
    const dim3 grid((unsigned)(cap < 65536 ? cap : 65536));
    const RowsOf rows = rows_of(z, stride), out = rows_of(grad, grad_stride);
    if (dt == NO_F32) hipLaunchKernelGGL(distill_kernel<float>, grid, dim3(256), 0, st, rows, d_n, cap, classes, ids, logits, k, temperature, weight, loss, lse_in, lse_out, out);
    else hipLaunchKernelGGL(distill_kernel<bf16_t>, grid, dim3(256), 0, st, rows, d_n, cap, classes, ids, logits, k, temperature, weight, loss, lse_in, lse_out, out);
    return launch_status(who);
}

}  // namespace no

using namespace no;

extern "C" size_t no_distill_ws_bytes(int32_t n_rows_cap, int32_t n_classes) {
    if (n_rows_cap < 0 || n_classes < 1 || n_classes > NO_MAX_CLASSES) return 0;
    return 16;
}

extern "C" int32_t no_distill_fwd(const void* d_z, no_dtype dt, int64_t z_stride_bytes, const int32_t* d_n_rows, int32_t n_rows_cap, int32_t n_classes,
                                  const int32_t* d_teacher_ids, const float* d_teacher_logits, int32_t k, float temperature,
                                  const float* d_row_weight, float* d_loss, float* d_lse, void* d_ws, size_t ws_bytes, void* stream) {
    clear_error();
    const char* who = "no_distill_fwd";
    NO_CHECK(check_logits(who, d_z, dt, z_stride_bytes, n_rows_cap, n_classes, temperature));
    NO_CHECK(check_teacher(who, n_rows_cap, d_teacher_ids, d_teacher_logits, k));
    NO_REQUIRE((d_loss && d_lse) || n_rows_cap == 0, NO_ERR_INVALID_ARG, "%s: NULL output", who);
    NO_CHECK(check_ws(who, d_ws, ws_bytes, no_distill_ws_bytes(n_rows_cap, n_classes)));
    return distill(who, d_z, dt, z_stride_bytes, d_n_rows, n_rows_cap, n_classes, d_teacher_ids, d_teacher_logits, k, temperature, d_row_weight, d_loss, nullptr,
                   d_lse, nullptr, 0, (hipStream_t)stream);
}

extern "C" int32_t no_distill_bwd(const void* d_z, no_dtype dt, int64_t z_stride_bytes, const int32_t* d_n_rows, int32_t n_rows_cap, int32_t n_classes,
                                  const int32_t* d_teacher_ids, const float* d_teacher_logits, int32_t k, float temperature,
                                  const float* d_row_weight, const float* d_lse, void* d_grad_z, int64_t grad_stride_bytes, void* stream) {
    clear_error();
    const char* who = "no_distill_bwd";
    NO_CHECK(check_logits(who, d_z, dt, z_stride_bytes, n_rows_cap, n_classes, temperature));
    NO_CHECK(check_teacher(who, n_rows_cap, d_teacher_ids, d_teacher_logits, k));
    NO_CHECK(check_rows(who, "grad_z", d_grad_z, dt, n_rows_cap, n_classes, grad_stride_bytes));
    NO_REQUIRE(d_lse || n_rows_cap == 0, NO_ERR_INVALID_ARG, "%s: lse is NULL", who);
    return distill(who, d_z, dt, z_stride_bytes, d_n_rows, n_rows_cap, n_classes, d_teacher_ids, d_teacher_logits, k, temperature, d_row_weight, nullptr, d_lse,
                   nullptr, d_grad_z, grad_stride_bytes, (hipStream_t)stream);
}

extern "C" int32_t no_distill_fwd_bwd(const void* d_z, no_dtype dt, int64_t z_stride_bytes, const int32_t* d_n_rows, int32_t n_rows_cap,
                                      int32_t n_classes, const int32_t* d_teacher_ids, const float* d_teacher_logits, int32_t k,
                                      float temperature, const float* d_row_weight, float* d_loss, float* d_lse, void* d_grad_z,
                                      int64_t grad_stride_bytes, void* d_ws, size_t ws_bytes, void* stream) {
    clear_error();
    const char* who = "no_distill_fwd_bwd";
    NO_CHECK(check_logits(who, d_z, dt, z_stride_bytes, n_rows_cap, n_classes, temperature));
    NO_CHECK(check_teacher(who, n_rows_cap, d_teacher_ids, d_teacher_logits, k));
    NO_CHECK(check_rows(who, "grad_z", d_grad_z, dt, n_rows_cap, n_classes, grad_stride_bytes));
    NO_REQUIRE(d_loss || n_rows_cap == 0, NO_ERR_INVALID_ARG, "%s: loss is NULL", who);
    NO_CHECK(check_ws(who, d_ws, ws_bytes, no_distill_ws_bytes(n_rows_cap, n_classes)));
    return distill(who, d_z, dt, z_stride_bytes, d_n_rows, n_rows_cap, n_classes, d_teacher_ids, d_teacher_logits, k, temperature, d_row_weight, d_loss, nullptr,
                   d_lse, d_grad_z, grad_stride_bytes, (hipStream_t)stream);
}

extern "C" size_t no_logprobs_ws_bytes(int32_t n_rows_cap, int32_t n_classes, int32_t k) {
    if (n_rows_cap < 0 || n_classes < 1 || n_classes > NO_MAX_CLASSES || k < 0 || k > NO_MAX_ALTERNATIVES) return 0;
    return 16;
}

extern "C" int32_t no_logprobs_fwd(const void* d_z, no_dtype dt, int64_t z_stride_bytes, const int32_t* d_n_rows, int32_t n_rows_cap, int32_t n_classes,
                                   const int32_t* d_tokens, float temperature, float* d_logprob, float* d_entropy, float* d_lse, int32_t k,
                                   int32_t* d_top_ids, float* d_top_logprobs, void* d_ws, size_t ws_bytes, void* stream) {
    clear_error();
    const char* who = "no_logprobs_fwd";
    NO_CHECK(check_logits(who, d_z, dt, z_stride_bytes, n_rows_cap, n_classes, temperature));
    NO_REQUIRE(k >= 0, NO_ERR_INVALID_ARG, "%s: k < 0", who);
    NO_REQUIRE(k <= NO_MAX_ALTERNATIVES, NO_ERR_UNSUPPORTED, "%s: more than %d alternatives", who, NO_MAX_ALTERNATIVES);
    NO_REQUIRE((d_tokens && d_logprob && d_entropy && d_lse) || n_rows_cap == 0, NO_ERR_INVALID_ARG, "%s: NULL argument", who);
    NO_REQUIRE((d_top_ids && d_top_logprobs) || n_rows_cap == 0 || k == 0, NO_ERR_INVALID_ARG, "%s: the alternatives' arrays are NULL", who);
    NO_CHECK(check_ws(who, d_ws, ws_bytes, no_logprobs_ws_bytes(n_rows_cap, n_classes, k)));
    if (n_rows_cap == 0) return NO_OK;
    const dim3 grid((unsigned)(n_rows_cap < 65536 ? n_rows_cap : 65536));
    const RowsOf z = rows_of(d_z, z_stride_bytes);
    if (dt == NO_F32) hipLaunchKernelGGL(logprobs_fwd_kernel<float>, grid, dim3(256), 0, (hipStream_t)stream, z, d_n_rows, n_rows_cap, n_classes, d_tokens, temperature, d_logprob, d_entropy, d_lse, k, d_top_ids, d_top_logprobs);
    else hipLaunchKernelGGL(logprobs_fwd_kernel<bf16_t>, grid, dim3(256), 0, (hipStream_t)stream, z, d_n_rows, n_rows_cap, n_classes, d_tokens, temperature, d_logprob, d_entropy, d_lse, k, d_top_ids, d_top_logprobs);
    return launch_status(who);
}

extern "C" int32_t no_logprobs_bwd(const void* d_z, no_dtype dt, int64_t z_stride_bytes, const int32_t* d_n_rows, int32_t n_rows_cap, int32_t n_classes,
                                   const int32_t* d_tokens, float temperature, const float* d_lse, const float* d_entropy, const float* d_grad_logprob,
                                   const float* d_grad_entropy, void* d_grad_z, int64_t grad_stride_bytes, void* stream) {
    clear_error();
    const char* who = "no_logprobs_bwd";
    NO_CHECK(check_logits(who, d_z, dt, z_stride_bytes, n_rows_cap, n_classes, temperature));
    NO_CHECK(check_rows(who, "grad_z", d_grad_z, dt, n_rows_cap, n_classes, grad_stride_bytes));
    NO_REQUIRE((d_tokens && d_lse && d_entropy) || n_rows_cap == 0, NO_ERR_INVALID_ARG, "%s: NULL argument", who);
    if (n_rows_cap == 0) return NO_OK;
    const dim3 grid((unsigned)(n_rows_cap < 65536 ? n_rows_cap : 65536));
    const RowsOf z = rows_of(d_z, z_stride_bytes), g = rows_of(d_grad_z, grad_stride_bytes);
    if (dt == NO_F32) hipLaunchKernelGGL(logprobs_bwd_kernel<float>, grid, dim3(256), 0, (hipStream_t)stream, z, d_n_rows, n_rows_cap, n_classes, d_tokens, temperature, d_lse, d_entropy, d_grad_logprob, d_grad_entropy, g);
    else hipLaunchKernelGGL(logprobs_bwd_kernel<bf16_t>, grid, dim3(256), 0, (hipStream_t)stream, z, d_n_rows, n_rows_cap, n_classes, d_tokens, temperature, d_lse, d_entropy, d_grad_logprob, d_grad_entropy, g);
    return launch_status(who);
}
