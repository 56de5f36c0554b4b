// Rows of fp32, bf16 or e4m3 values for the operators on learned inputs and large answers (embed.hip, rmsnorm.hip, logits.hip): types,
// 16-byte units of a row at any alignment, reductions over the lanes that share a row.
#pragma once
#include "primitives.hpp"

namespace no {

typedef __bf16 bf16_t;
struct e4m3_t { uint8_t bits; };

template <typename T> struct TypeOf;
template <> struct TypeOf<float> { static constexpr no_dtype code = NO_F32; };
template <> struct TypeOf<bf16_t> { static constexpr no_dtype code = NO_BF16; };
template <> struct TypeOf<e4m3_t> { static constexpr no_dtype code = NO_E4M3; };

static inline int32_t size_of(no_dtype dt) { return dt == NO_F32 ? 4 : dt == NO_BF16 ? 2 : 1; }

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(bf16_t v) { return (float)v; }
__device__ __forceinline__ float to_f32(e4m3_t v) { return __builtin_amdgcn_cvt_f32_fp8((int)v.bits, 0); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16_t from_f32<bf16_t>(float v) { return (bf16_t)v; }
template <> __device__ __forceinline__ e4m3_t from_f32<e4m3_t>(float v) {
    return e4m3_t{(uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(v, 0.0f, 0, false)};
}

// Rows that are there: min(*d_n, cap), or cap.
__device__ __forceinline__ int32_t rows_here(const int32_t* d_n, int32_t cap) { return d_n ? min(*d_n, cap) : cap; }

// One pointer and stride of a row matrix.
struct RowsOf {
    char* p;
    int64_t stride;
    template <typename T> __device__ __forceinline__ T* row(int64_t i) const { return reinterpret_cast<T*>(p + i * stride); }
};
static inline RowsOf rows_of(const void* p, int64_t stride) { return RowsOf{(char*)p, stride}; }

// What every call checks of a row matrix. The stride counts from the second row on.
static inline int32_t check_rows(const char* who, const char* what, const void* p, no_dtype dt, int64_t n, int64_t dim, int64_t stride) {
    const int32_t es = size_of(dt);
    NO_REQUIRE(p || n == 0, NO_ERR_INVALID_ARG, "%s: %s is NULL", who, what);
    NO_REQUIRE((uintptr_t)p % es == 0 && stride % es == 0, NO_ERR_INVALID_ARG, "%s: %s: address and stride must be multiples of the element size", who, what);
    NO_REQUIRE(stride >= dim * es, NO_ERR_INVALID_ARG, "%s: %s: stride smaller than a row", who, what);
    return NO_OK;
}

}  // namespace no
