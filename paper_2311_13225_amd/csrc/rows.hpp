// Rows of fp32, bf16 or e4m3 values for the operators on learned inputs and large answers (embed.hip, rmsnorm.hip, logits.hip): types,
// 16-byte units of a row at any alignment, reductions over the lanes that share a row.
#pragma once
#include "primitives.hpp"

#include <type_traits>

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
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16_t from_f32<bf16_t>(float v) { return (bf16_t)v; }
template <> __device__ __forceinline__ e4m3_t from_f32<e4m3_t>(float v) {
    return e4m3_t{(uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(v, 0.0f, 0, false)};
}

// Rows that are there: *d_n within [0, cap], or cap.
__device__ __forceinline__ int32_t rows_here(const int32_t* d_n, int32_t cap) { return d_n ? min(max(*d_n, 0), cap) : cap; }

// One pointer and stride of a row matrix.
struct RowsOf {
    char* p;
    int64_t stride;
    template <typename T> __device__ __forceinline__ T* row(int64_t i) const { return reinterpret_cast<T*>(p + i * stride); }
};
static inline RowsOf rows_of(const void* p, int64_t stride) { return RowsOf{(char*)p, stride}; }

// W consecutive values of a row, `here` of which are there (the others read as `fill` and are not written). A whole run goes in 16-byte (or
// narrower, for short runs) requests at any alignment of an element: global memory takes unaligned requests on this chip, so that odd row
// widths, whose rows begin anywhere, take the same path.
template <int BYTES> struct Chunk;
template <> struct Chunk<4> { typedef uint32_t raw __attribute__((aligned(1), may_alias)); typedef uint32_t val; };
template <> struct Chunk<8> { typedef uint32_t val __attribute__((ext_vector_type(2))); typedef val raw __attribute__((aligned(1), may_alias)); };
template <> struct Chunk<16> { typedef uint32_t val __attribute__((ext_vector_type(4))); typedef val raw __attribute__((aligned(1), may_alias)); };

template <typename T, int W>
struct Run {
    static constexpr int BYTES = W * (int)sizeof(T), REQ = BYTES < 16 ? BYTES : 16, N = BYTES / REQ, WORDS = BYTES / 4, BITS = 8 * (int)sizeof(T);
    typedef typename Chunk<REQ>::val val;
    typedef typename Chunk<REQ>::raw raw;
    val v[N];
    __device__ __forceinline__ void load(const T* p) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = reinterpret_cast<const raw*>(p)[i];
    }
    // the same past the caches' usual order: values that are used once
    __device__ __forceinline__ void load_once(const T* p) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = __builtin_nontemporal_load(reinterpret_cast<const raw*>(p) + i);
    }
    // `here` values and no more, one at a time, in a loop that shifts the run (written out, a branch a value, it costs the kernels more registers than the rest of
    // them needs). Each waits for memory by itself: for rows shorter than a run.
    __device__ __forceinline__ void load(const T* p, int here, T fill) {
        if (here >= W) return load(p);
        uint32_t w[WORDS], f = bits(fill);
        if constexpr (BITS == 8) f |= f << 8;
        if constexpr (BITS <= 16) f |= f << 16;
#pragma unroll
        for (int j = 0; j < WORDS; ++j) w[j] = f;
#pragma unroll 1
        for (int i = here - 1; i >= 0; --i) {
#pragma unroll
            for (int j = WORDS - 1; j > 0; --j) w[j] = BITS == 32 ? w[j - 1] : w[j] << (BITS & 31) | w[j - 1] >> (32 - BITS & 31);
            w[0] = BITS == 32 ? bits(p[i]) : w[0] << (BITS & 31) | bits(p[i]);
        }
        __builtin_memcpy(v, w, BYTES);
    }
    // The same from the W values that end at p + here, one request, shifted into place: the end of a row of W values and more. (What it reads of the run before
    // is shifted out, so that it may be overwritten meanwhile.)
    __device__ __forceinline__ void load_to_end(const T* p, int here, T fill) {
        load(p + here - W);
        uint32_t w[WORDS];
        __builtin_memcpy(w, v, BYTES);
#pragma unroll 1
        for (int i = here; i < W; ++i) {
#pragma unroll
            for (int j = 0; j < WORDS; ++j) {
                const uint32_t up = j + 1 < WORDS ? w[j + 1 < WORDS ? j + 1 : 0] : bits(fill);
                w[j] = BITS == 32 ? up : w[j] >> (BITS & 31) | up << (32 - BITS & 31);
            }
        }
        __builtin_memcpy(v, w, BYTES);
    }
    // values [c, c + W) of a row of `dim`
    __device__ __forceinline__ void load_at(const T* row, int32_t c, int32_t dim, T fill) {
        if (c + W <= dim) load(row + c);
        else if (dim >= W && c < dim) load_to_end(row + c, dim - c, fill);
        else load(row + (c < dim ? c : 0), dim - c, fill);
    }
    __device__ __forceinline__ void store(T* p) const {
#pragma unroll
        for (int i = 0; i < N; ++i) reinterpret_cast<raw*>(p)[i] = v[i];
    }
    __device__ __forceinline__ void store_once(T* p) const {
#pragma unroll
        for (int i = 0; i < N; ++i) __builtin_nontemporal_store(v[i], reinterpret_cast<raw*>(p) + i);
    }
    __device__ __forceinline__ void store(T* p, int here) const {
        if (here >= W) return store(p);
        uint32_t w[WORDS];
        __builtin_memcpy(w, v, BYTES);
#pragma unroll 1
        for (int i = 0; i < here; ++i) {
            T e;
            __builtin_memcpy(&e, w, sizeof(T));
            p[i] = e;
#pragma unroll
            for (int j = 0; j < WORDS; ++j) {
                const uint32_t up = j + 1 < WORDS ? w[j + 1 < WORDS ? j + 1 : 0] : 0u;
                w[j] = BITS == 32 ? up : w[j] >> (BITS & 31) | up << (32 - BITS & 31);
            }
        }
    }
    __device__ __forceinline__ static uint32_t bits(T e) {
        if constexpr (BITS == 32) return __builtin_bit_cast(uint32_t, e);
        else if constexpr (BITS == 16) return __builtin_bit_cast(uint16_t, e);
        else return __builtin_bit_cast(uint8_t, e);
    }
    __device__ __forceinline__ void get(float (&f)[W]) const {
        uint32_t w[WORDS];
        __builtin_memcpy(w, v, BYTES);
        if constexpr (BITS == 8) {
            typedef float f2 __attribute__((ext_vector_type(2)));
#pragma unroll
            for (int i = 0; i < W / 4; ++i) {
                const f2 a = __builtin_amdgcn_cvt_pk_f32_fp8(w[i], false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w[i], true);
                f[4 * i] = a.x; f[4 * i + 1] = a.y; f[4 * i + 2] = b.x; f[4 * i + 3] = b.y;
            }
        } else if constexpr (BITS == 16) {
#pragma unroll
            for (int i = 0; i < W / 2; ++i) {
                f[2 * i] = __uint_as_float(w[i] << 16);
                f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int i = 0; i < W; ++i) f[i] = __uint_as_float(w[i]);
        }
    }
    __device__ __forceinline__ void set(const float (&f)[W]) {
        uint32_t w[WORDS];
        if constexpr (BITS == 8) {
#pragma unroll
            for (int i = 0; i < W / 4; ++i)
                w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i + 2], f[4 * i + 3], __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i], f[4 * i + 1], 0, false), true);
        } else if constexpr (BITS == 16) {
            typedef float f2 __attribute__((ext_vector_type(2)));
            typedef __bf16 b2 __attribute__((ext_vector_type(2)));
#pragma unroll
            for (int i = 0; i < W / 2; ++i) w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{f[2 * i], f[2 * i + 1]}), b2));
        } else {
#pragma unroll
            for (int i = 0; i < W; ++i) w[i] = __float_as_uint(f[i]);
        }
        __builtin_memcpy(v, w, BYTES);
    }
};

// Where a lane's run of a row begins: at its own columns [c, c + W), or W values before the row's end, so that the requests of every lane are whole and nothing branches; the
// last two lanes of such a row hold some values twice. Rows shorter than a run (SHORT) go value by value.
template <int W, bool SHORT>
struct Place {
    int32_t at, skip;       // skip: values of the run that are the lane before's
    int32_t dim;
    __device__ __forceinline__ Place(int32_t c, int32_t dim_) : at(SHORT ? c : min(c, dim_ - W)), skip(c - at), dim(dim_) {}
    template <typename T>
    __device__ __forceinline__ void load(Run<T, W>& r, const T* row) const {
        if constexpr (SHORT) r.load_at(row, at, dim, from_f32<T>(0.0f));
        else r.load(row + at);
    }
    __device__ __forceinline__ void store(const float (&f)[W], float* row) const {      // of a lane inside the row
        if (SHORT || skip == 0) {
            Run<float, W> o;
            o.set(f);
            if constexpr (SHORT) o.store(row + at, dim - at);
            else o.store(row + at);
        } else {
#pragma unroll
            for (int w = 1; w < W; ++w) if (w >= skip) row[at + w] = f[w];
        }
    }
};

// p + c for a row's address, the same in all lanes, and a place in it: 32 bits of offset, which a request takes beside a scalar address (as 64-bit
// addresses the places of all of a lane's runs would be kept in registers).
template <typename T>
__device__ __forceinline__ T* offset(T* p, int32_t c) {
    typedef typename std::conditional<std::is_const<T>::value, const char, char>::type byte;
    return reinterpret_cast<T*>(reinterpret_cast<byte*>(p) + (uint32_t)c * (uint32_t)sizeof(T));
}

// A row (or a piece of one) of `len` values in the registers of TEAM lanes: run u of lane t covers values [(t + u TEAM) W, + W). ONCE: by requests that leave the caches
// to others. Measured kernel by kernel: sums of 16384 x 32768 bf16 logits 198 -> 178 us, their gradient from an lse 403 -> 373, the gradient of log probabilities 101 -> 95, rows
// of 131072 bf16 logits in a block 426 -> 410, of 20000 fp32 ones 242 -> 215; but short rows of logits slower (100000 x 600 fp32 99 -> 152), and what fits the caches (see the norms).
template <typename T, int W, int U, int TEAM, bool ONCE = false>
struct RowRegs {
    Run<T, W> v[U];
    __device__ __forceinline__ static int32_t at(int t, int u) { return (t + u * TEAM) * W; }
    // run u, if all of it is there (else `fill`)
    __device__ __forceinline__ void load_run(const T* p, int32_t len, int t, int u, T fill) {
        if (at(t, u) + W <= len) {
            if constexpr (ONCE) v[u].load_once(offset(p, at(t, u)));
            else v[u].load(offset(p, at(t, u)));
        } else v[u].load(p, 0, fill);
    }
    // the run that the row ends in, by the lane that has it
    __device__ __forceinline__ void load_end(const T* p, int32_t len, int t, T fill) {
        if (len % W == 0) return;
        const int32_t c = len / W * W;
        if (len / W % TEAM != t) return;
        Run<T, W> r;
        if (c > 0) r.load_to_end(p + c, len - c, fill);
        else r.load(p, len, fill);
#pragma unroll
        for (int u = 0; u < U; ++u) if (c == at(t, u)) v[u] = r;
    }
    __device__ __forceinline__ void load(const T* p, int32_t len, int t, T fill) {
#pragma unroll
        for (int u = 0; u < U; ++u) load_run(p, len, t, u, fill);
        load_end(p, len, t, fill);
    }
    // Between two passes over the values: without it the compiler keeps what the first one converted to fp32 (twice the registers of bf16 rows, spilled in
    // the largest kernels) instead of converting again, one instruction a value.
    __device__ __forceinline__ void renew() {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < Run<T, W>::N; ++i) asm volatile("" : "+v"(v[u].v[i]));
    }
};

// Stores a row run by run; the run that the row ends in is kept until the others are stored.
template <typename T, int W, bool ONCE = false>
struct RowStore {
    T* p;
    int32_t len, end = -1;
    Run<T, W> last;
    __device__ __forceinline__ RowStore(T* p_, int32_t len_) : p(p_), len(len_) {}
    __device__ __forceinline__ void put(int32_t c, const Run<T, W>& r) {
        if (c + W <= len) {
            if constexpr (ONCE) r.store_once(offset(p, c));
            else r.store(offset(p, c));
        } else if (c < len) { last = r; end = c; }
    }
    __device__ __forceinline__ void finish() { if (end >= 0) last.store(p + end, len - end); }
};

// TEAM lanes that share a row: a part of a wavefront, a wavefront, or a block. Sums and maxima reach every lane. Across wavefronts they cost one
// barrier each: two slots take turns, and a wavefront that writes a slot again has passed the barrier behind its last reads.
template <int TEAM, int THREADS>
struct Team {
    static_assert(TEAM <= 64 || TEAM == THREADS, "a team is a part of a wavefront or the block");
    static constexpr int WAVES = TEAM <= 64 ? 1 : TEAM / 64, PER_BLOCK = THREADS / TEAM;
    float* smem;        // [2][WAVES] where a team spans wavefronts
    int turn = 0;
    __device__ __forceinline__ explicit Team(float* s) : smem(s) {}
    __device__ __forceinline__ static int lane() { return (int)threadIdx.x & (TEAM - 1); }
    __device__ __forceinline__ static int index() { return (int)threadIdx.x / TEAM; }
    template <typename Op>
    __device__ __forceinline__ float reduce(float v, Op op) {
#pragma unroll
        for (int o = (TEAM < 64 ? TEAM : 64) / 2; o > 0; o >>= 1) v = op(v, __shfl_xor(v, o, 64));
        if constexpr (TEAM > 64) {
            float* s = smem + turn * WAVES;
            turn ^= 1;
            if (lane_id() == 0) s[threadIdx.x >> 6] = v;
            __syncthreads();
            v = s[0];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) v = op(v, s[w]);
        }
        return v;
    }
    // what the team's lanes wrote before, its lanes see after
    __device__ __forceinline__ static void sync() {
        if constexpr (TEAM > 64) __syncthreads();
        else {
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        }
    }
    __device__ __forceinline__ float sum(float v) { return reduce(v, [](float a, float b) { return a + b; }); }
    __device__ __forceinline__ float max(float v) { return reduce(v, [](float a, float b) { return fmaxf(a, b); }); }
};

// What every call checks of a row matrix. The stride counts from the second row on.
static inline int32_t check_rows(const char* who, const char* what, const void* p, no_dtype dt, int64_t n, int64_t dim, int64_t stride) {
    const int32_t es = size_of(dt);
    NO_REQUIRE(p || n == 0, NO_ERR_INVALID_ARG, "%s: %s is NULL", who, what);
    NO_REQUIRE((uintptr_t)p % es == 0 && stride % es == 0, NO_ERR_INVALID_ARG, "%s: %s: address and stride must be multiples of the element size", who, what);
    NO_REQUIRE(stride >= dim * es, NO_ERR_INVALID_ARG, "%s: %s: stride smaller than a row", who, what);
    return NO_OK;
}

}  // namespace no
