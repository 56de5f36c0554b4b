// no_distill_* and no_logprobs_*: rows of logits, read once.
//
// A team of lanes (a wavefront or a block) holds a row, or a piece of one, in registers, U runs of 16 bytes a lane, and takes the maximum, the sum of
// exponentials and whatever follows from there. Rows that are longer than a team's registers, and rows that are too few to fill the chip, are cut into pieces whose sums a
// second launch joins. Exponentials are 2^x with x = (z - m) c, c = log2(e) / T, m the row's maximum, the difference taken first: it is exact next to the maximum,
// where the exponentials are large, so that its rounding costs nothing there; where x leaves fp32 its exponential is 0 long since, and log p itself is made in natural units.
// (fma(z, c, -mc) saves one instruction of twelve, but is off by the rounding of mc = m c, which is no smaller than the result where |m c| passes 2^24: logits of 1e8, or a small T.)
#include "rows.hpp"

namespace no {

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

__device__ __forceinline__ float above(float m) { return m == -INFINITY ? 0.0f : m; }      // what differences are taken from

// x of a logit under a maximum.
struct Exponent {
    float from, c;
    __device__ __forceinline__ Exponent(float m, float c_) : from(above(m)), c(c_) {}
    __device__ __forceinline__ float operator()(float z) const { return (z - from) * c; }
};

// Sums of a row, a piece or a lane's values: largest logit (-inf: there is none above), sum of 2^x, sum of x 2^x.
struct Sums {
    float m, s, h;
    // s and h as they are under another maximum, no smaller than m. Where d lies below -1000 the exponential is 0, and d held there keeps its product with s, and so h, finite:
    // under masks of a type's lowest value d itself is about -3e38, or -inf (and +inf of a lane without values, whose s is 0).
    template <bool ENTROPY>
    __device__ __forceinline__ void move(const Exponent& to) {
        const float d = to(above(m)), e = s == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(d);
        if constexpr (ENTROPY) h = e * (h + __builtin_amdgcn_fmed3f(d, -1000.0f, 0.0f) * s);
        s *= e;
    }
};

// log p of a logit from its row's sums and the logarithm (to base 2) of their s. In natural units: to base 2 the difference of a masked class (a type's lowest value) leaves
// fp32 where log p itself does not. A difference that leaves it before its division by T is taken after that; its two parts have one sign then, so that nothing cancels.
__device__ __forceinline__ float log_ratio(const Sums& r, float inv_t, float log_s, float z) {
    const float from = above(r.m), d = z - from;
    return (fabsf(d) < INFINITY ? d * inv_t : z * inv_t - from * inv_t) - log_s * LN2;
}

template <typename T, int U, int TEAM, bool ONCE = false>
struct Piece : RowRegs<T, 16 / (int)sizeof(T), U, TEAM, ONCE> {      // logits of a row or a piece of one, in a lane's registers; -inf behind its end
    static constexpr int W = 16 / (int)sizeof(T);
    using RowRegs<T, W, U, TEAM, ONCE>::v;
    __device__ __forceinline__ void load(const T* z, int32_t len, int t) { RowRegs<T, W, U, TEAM, ONCE>::load(z, len, t, from_f32<T>(-INFINITY)); }
    // Sums of the lane's values, run by run with the maximum so far, so that the first runs are added while later ones are still on their way; what was added under a smaller
    // maximum is scaled down, one exponential a run.
    template <bool ENTROPY>
    __device__ __forceinline__ Sums lane_sums(float c) {
        Sums r{-INFINITY, 0.0f, 0.0f};
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float f[W], m = r.m;
            v[u].get(f);
#pragma unroll
            for (int w = 0; w < W; ++w) m = fmaxf(m, f[w]);
            const Exponent x(m, c);
            if (u > 0) r.move<ENTROPY>(x);
            r.m = m;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float d = x(f[w]), e = __builtin_amdgcn_exp2f(d);
                r.s += e;
                if constexpr (ENTROPY) r.h += e * fmaxf(d, -3.0e38f);     // (-inf counts as 0)
            }
            // The next run waits for this one's sums: taken ahead for their maximum, or put off until h is asked for, all runs' values or exponentials
            // would stand in registers at once.
            asm volatile("" : "+v"(v[u + 1 < U ? u + 1 : u].v[0]), "+v"(r.s), "+v"(r.h));
        }
        return r;
    }
};

// Sums of a team's lanes, or of a lane's share of a row's pieces, each with its own maximum, as the team's.
template <bool ENTROPY, int TEAM, int THREADS>
__device__ __forceinline__ Sums team_sums(Sums r, float c, Team<TEAM, THREADS>& team) {
    const float m = team.max(r.m);
    r.move<ENTROPY>(Exponent(m, c));
    return Sums{m, team.sum(r.s), ENTROPY ? team.sum(r.h) : 0.0f};
}

// Joins the sums of a row's pieces, each with its own maximum: a lane takes pieces t, t + TEAM, ...
template <int TEAM, int THREADS>
__device__ __forceinline__ Sums join_sums(const Sums* parts, int32_t pieces, float c, Team<TEAM, THREADS>& team) {
    Sums r{-INFINITY, 0.0f, 0.0f};
    for (int32_t p = team.lane(); p < pieces; p += TEAM) {
        Sums q = parts[p];
        const Exponent x(fmaxf(r.m, q.m), c);
        r.move<true>(x);
        q.move<true>(x);
        r = Sums{fmaxf(r.m, q.m), r.s + q.s, r.h + q.h};
    }
    return team_sums<true>(r, c, team);
}

// ------------------------------------------------------------------------------------------------------- teacher

// The teacher's entries of a row in LDS: class (-1: left out) and share side by side, the share's logarithm, and the student's logit there. One wavefront makes them, up to four
// entries a lane, without a barrier; in blocks of several the others take the row's sums meanwhile.
struct Entry { int32_t id; float p; };
struct Teacher {
    Entry of[NO_MAX_TEACHER];
    float log_p[NO_MAX_TEACHER], z[NO_MAX_TEACHER];
    int32_t any;        // whether an entry is above -inf
};
constexpr int TEACHER_Q = NO_MAX_TEACHER / 64;
static_assert(TEACHER_Q * 64 == NO_MAX_TEACHER, "entries go evenly over a wavefront");

struct Distill {
    RowsOf z;
    const int32_t* d_n;
    int64_t row0;                   // the launch's first row
    int32_t cap, classes;
    const int32_t* ids;
    const float* logits;
    int32_t k;
    float temperature, inv_t, c;    // 1 / T, log2(e) / T
    const float* weight;
    float* loss;
    const float* lse_in;
    float* lse_out;
    RowsOf grad;
    Sums* parts;                    // [cap][pieces] where rows are cut
    int32_t pieces, piece;          // pieces a row, values a piece (a multiple of a run)
};

typedef Team<64, 64> Wave;

struct Entries {        // a lane's entries as they come from memory
    int32_t id[TEACHER_Q];
    float x[TEACHER_Q], z[TEACHER_Q], w;
    __device__ __forceinline__ void load(const Distill& a, int64_t i) {
        w = a.weight ? a.weight[i] : 1.0f;
#pragma unroll
        for (int q = 0; q < TEACHER_Q; ++q) {
            const int j = lane_id() + q * 64;
            id[q] = j < a.k ? a.ids[i * a.k + j] : -1;
            x[q] = j < a.k ? a.logits[i * a.k + j] : -INFINITY;
        }
    }
    // the student's logits at those in [lo, hi)
    template <typename T>
    __device__ __forceinline__ void load_logits(const T* row, int32_t classes, int32_t lo, int32_t hi) {
#pragma unroll
        for (int q = 0; q < TEACHER_Q; ++q) {
            if (id[q] < 0 || id[q] >= classes) id[q] = -1;
            z[q] = id[q] >= lo && id[q] < hi ? to_f32(row[id[q]]) : 0.0f;
        }
    }
    // softmax(logits / T) over the entries inside the classes
    __device__ __forceinline__ void shares(const Distill& a, Teacher& to) const {
        Wave wave(nullptr);
        float m = -INFINITY, s = 0.0f, e[TEACHER_Q];
#pragma unroll
        for (int q = 0; q < TEACHER_Q; ++q) if (id[q] >= 0) m = fmaxf(m, x[q]);
        const float from = above(wave.max(m));
#pragma unroll
        for (int q = 0; q < TEACHER_Q; ++q) {
            e[q] = id[q] < 0 ? 0.0f : expf((x[q] - from) * a.inv_t);
            s += e[q];
        }
        s = wave.sum(s);
        const float log_s = logf(s);
#pragma unroll
        for (int q = 0; q < TEACHER_Q; ++q) {
            const int j = lane_id() + q * 64;
            if (j < a.k) {
                to.of[j] = Entry{id[q], s == 0.0f ? 0.0f : e[q] / s};
                to.log_p[j] = (x[q] - from) * a.inv_t - log_s;
                to.z[j] = z[q];
            }
        }
        if (lane_id() == 0) to.any = s != 0.0f;
    }
};

// Loss and lse of a row whose sums are known, by one wavefront. The terms are T p (log p - log q) with T log q = (z - m) - T log s, so that masked classes (a type's lowest
// value) that the teacher names leave the loss finite, where z / T, z - m or the sum of terms would leave fp32: halves of the terms do not.
__device__ __forceinline__ void distill_loss(const Distill& a, int64_t i, const Sums& r, float w, const Teacher& te) {
    const float from = above(r.m), ln_s = log2f(r.s) * LN2;
    float term = 0.0f;
    for (int j = lane_id(); j < a.k; j += 64)
        if (te.of[j].p != 0.0f) term += te.of[j].p * (r.s == 0.0f ? INFINITY : 0.5f * a.temperature * (te.log_p[j] + ln_s) - (0.5f * te.z[j] - 0.5f * from));
    term = Wave(nullptr).sum(term);
    if (lane_id() == 0) {
        a.loss[i] = w == 0.0f || !te.any ? 0.0f : 2.0f * (w * a.temperature * term);
        if (a.lse_out) a.lse_out[i] = from * a.inv_t + ln_s;
    }
}

// A class's share in the student's row, times `by`: from the row's sums, or from its lse. (A row of -inf alone has no share anywhere: the factor is 0
// then, or the lse counts as +inf.)
struct ShareBySums {
    Exponent x;
    float by;
    __device__ __forceinline__ ShareBySums(const Sums& r, float c, float by_) : x(r.m, c), by(r.s == 0.0f ? 0.0f : by_ / r.s) {}
    __device__ __forceinline__ float operator()(float z) const { return __builtin_amdgcn_exp2f(x(z)) * by; }
};
// (An lse is rounded, which may be more than a share's logarithm where a row is masked throughout, by -1e9 or less: no share is larger than 1, so no exponent is above 0. The
// minimum drops a NaN; a row whose lse is one takes it from the factor.)
struct ShareByLse {
    float inv_t, lse, by;
    __device__ __forceinline__ ShareByLse(float inv_t_, float lse_, float by_) : inv_t(inv_t_), lse(lse_ == -INFINITY ? INFINITY : lse_), by(lse_ != lse_ ? NAN : by_) {}
    __device__ __forceinline__ float operator()(float z) const { return __builtin_amdgcn_exp2f(fminf(z * inv_t - lse, 0.0f) * LOG2E) * by; }
};

// The gradient of values [first, first + len) of a row, held in `v`: w T q everywhere, then the classes that the teacher names once more with
// their shares taken off (the barrier orders the two stores; an entry that stands twice stores the same value twice).
template <typename T, int U, int TEAM, int THREADS, bool ONCE, typename Q>
__device__ __forceinline__ void distill_grad(const Distill& a, int64_t i, int32_t first, int32_t len, Piece<T, U, TEAM, ONCE>& v, const Q& q, float w, const Teacher& te,
                                             Team<TEAM, THREADS>& team) {
    constexpr int W = Piece<T, U, TEAM>::W;
    int t = team.lane();
    asm volatile("" : "+v"(t));
    T* const out = a.grad.row<T>(i) + first;
    RowStore<T, W, ONCE> store(out, len);
    const bool live = w != 0.0f && te.any;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        Run<T, W> o;
        if (live) {
            float f[W];
            v.v[u].get(f);
#pragma unroll
            for (int x = 0; x < W; ++x) f[x] = q(f[x]);
            o.set(f);
        } else o.v[0] = 0;
        store.put(v.at(t, u), o);
    }
    store.finish();
    team.sync();
    if (live)
        for (int j = t; j < a.k; j += TEAM) {
            const int32_t id = te.of[j].id, at = id - first;
            if (id < 0 || at < 0 || at >= len) continue;
            float share = 0.0f;         // of all entries with this class
#pragma unroll 8
            for (int o = 0; o < a.k; ++o) {
                const Entry other = te.of[o];
                share += other.id == id ? other.p : 0.0f;
            }
            out[at] = from_f32<T>(q(te.z[j]) - w * a.temperature * share);
        }
}

// Whole rows in a team's registers: everything in one read and one write, which bound it; the largest take a compute unit's register file. 1024 x 172 fp32 with 8 entries: 5.6 us, a row's
// round trips; 16384 x 32768 bf16: 403 us, 5.3 TB/s; 4096 x 131072 bf16 with 64 entries: 410 us, 5.2 TB/s (sums and gradients in two launches: 554; a block that walks rows and
// asks for each run of the next one as soon as the gradient has no more use for its registers: 452).
template <typename T, int TEAM, int THREADS, int U>
__global__ void __launch_bounds__(THREADS) distill_row_kernel(Distill a) {
    __shared__ float smem[2 * THREADS / 64];
    __shared__ Teacher teachers[THREADS / TEAM];
    Team<TEAM, THREADS> team(smem);
    Teacher& te = teachers[team.index()];
    const int64_t i = a.row0 + (int64_t)blockIdx.x * (THREADS / TEAM) + team.index();
    if (i >= rows_here(a.d_n, a.cap)) return;
    const T* z = a.z.row<T>(i);
    const bool first_wave = TEAM == 64 || threadIdx.x < 64;
    Entries e;
    if (first_wave) e.load(a, i);
    Piece<T, U, TEAM, (TEAM == 1024 && U > 4)> v;
    v.load(z, a.classes, team.lane());
    const float w = a.weight ? a.weight[i] : 1.0f;
    if (first_wave) {
        e.load_logits(z, a.classes, 0, a.classes);
        e.shares(a, te);
    }
    if constexpr (TEAM == 64)       // (longer rows go in pieces where an lse is given)
        if (a.lse_in) {
            team.sync();
            distill_grad(a, i, 0, a.classes, v, ShareByLse(a.inv_t, a.lse_in[i], w * a.temperature), w, te, team);
            return;
        }
    const Sums r = team_sums<false>(v.template lane_sums<false>(a.c), a.c, team);
    v.renew();
    if constexpr (TEAM == 64) team.sync();      // (the entries; in larger teams a sum's barrier stood between)
    if (first_wave) distill_loss(a, i, r, w, te);
    if (a.grad.p) distill_grad(a, i, 0, a.classes, v, ShareBySums(r, a.c, w * a.temperature), w, te, team);
}

// Sums of one piece of a row. 16384 x 32768 bf16: 174 us, 6.2 TB/s.
template <typename T, int THREADS, int U>
__global__ void __launch_bounds__(THREADS) distill_sums_kernel(Distill a) {
    __shared__ float smem[2 * THREADS / 64];
    Team<THREADS, THREADS> team(smem);
    const int64_t i = a.row0 + blockIdx.x / (uint32_t)a.pieces;
    const int32_t p = (int32_t)(blockIdx.x % (uint32_t)a.pieces);
    if (i >= rows_here(a.d_n, a.cap)) return;
    Piece<T, U, THREADS, true> v;
    v.load(a.z.row<T>(i) + (int64_t)p * a.piece, min(a.piece, a.classes - p * a.piece), team.lane());
    const Sums r = team_sums<false>(v.template lane_sums<false>(a.c), a.c, team);
    if (threadIdx.x == 0) a.parts[i * a.pieces + p] = r;
}

// One piece of a row's gradient, from the sums of the row's pieces or from a given lse (4096 x 131072 bf16: 367 us, 5.9 TB/s). The gradient may go over the logits, so the loss, which
// reads them all over the row, is made by a launch before this one (distill_loss_kernel).
template <typename T, int THREADS, int U>
__global__ void __launch_bounds__(THREADS) distill_grad_kernel(Distill a) {
    __shared__ float smem[2 * THREADS / 64];
    __shared__ Teacher te;
    Team<THREADS, THREADS> team(smem);
    const int64_t i = a.row0 + blockIdx.x / (uint32_t)a.pieces;
    const int32_t p = (int32_t)(blockIdx.x % (uint32_t)a.pieces), first = p * a.piece, len = min(a.piece, a.classes - first);
    if (i >= rows_here(a.d_n, a.cap)) return;
    const T* z = a.z.row<T>(i);
    Entries e;
    if (threadIdx.x < 64) e.load(a, i);
    Piece<T, U, THREADS, true> v;
    v.load(z + first, len, team.lane());
    const float w = a.weight ? a.weight[i] : 1.0f;
    if (threadIdx.x < 64) {
        e.load_logits(z, a.classes, first, first + len);
        e.shares(a, te);
    }
    if (a.lse_in) {
        team.sync();
        distill_grad(a, i, first, len, v, ShareByLse(a.inv_t, a.lse_in[i], w * a.temperature), w, te, team);
    } else {
        const Sums r = join_sums(a.parts + i * a.pieces, a.pieces, a.c, team);      // (its barriers stand behind the entries)
        distill_grad(a, i, first, len, v, ShareBySums(r, a.c, w * a.temperature), w, te, team);
    }
}

// Loss and lse from the sums of a row's pieces.
template <typename T>
__global__ void __launch_bounds__(256) distill_loss_kernel(Distill a) {
    __shared__ Teacher teachers[4];
    Team<64, 256> team(nullptr);
    Teacher& te = teachers[team.index()];
    const int64_t i = a.row0 + (int64_t)blockIdx.x * 4 + team.index();
    if (i >= rows_here(a.d_n, a.cap)) return;
    const T* z = a.z.row<T>(i);
    Entries e;
    e.load(a, i);
    e.load_logits(z, a.classes, 0, a.classes);
    e.shares(a, te);
    const Sums r = join_sums(a.parts + i * a.pieces, a.pieces, a.c, team);
    team.sync();
    distill_loss(a, i, r, a.weight ? a.weight[i] : 1.0f, te);
}

// ------------------------------------------------------------------------------------------------------- log probabilities

// Order of alternatives: larger value first, then the lower class; -0 counts as 0.
__device__ __forceinline__ uint32_t order_of(float v) {
    const uint32_t b = __float_as_uint(v + 0.0f);
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o); }
__device__ __forceinline__ uint64_t order_key(float v, int32_t c) { return (uint64_t)order_of(v) << 32 | (uint32_t)~c; }

template <int TEAM>
struct TopSpace {
    static constexpr int CAP = 512;         // candidates that are ranked against each other
    uint64_t key[CAP];
    int32_t count;
    uint32_t bound[TEAM / 64];
};

// The k largest values of a piece, as order keys in `to.key[0 .. min(count, CAP))`, in no order, with others that are smaller among them perhaps: all that reach a bound which
// k values at least reach, and few others as a rule. Where n wavefronts share the piece, the ceil(k / n)-th largest of a wavefront's 64 lane maxima is reached by that many
// of its values, and the least of the n such values by k of the piece. Where that is -inf, since a wavefront holds next to nothing else, the k-th largest lane maximum of any one
// wavefront will do as well, and the largest of those is taken. Where more reach the bound than there is room for (equal values, large ones that sit in few lanes, or finite masks, which are
// values like others), it is raised bit by bit, first by value, then among equal ones by class (4096 x 50001 fp32 of which ten classes are left: 139 us masked with -inf, 1890 with the lowest value).
template <typename T, int U, int TEAM, int THREADS>
__device__ __forceinline__ void top_candidates(Piece<T, U, TEAM, true>& v, float lane_max, int32_t first, int32_t k, TopSpace<TEAM>& to, Team<TEAM, THREADS>& team) {
    constexpr int W = Piece<T, U, TEAM>::W;
    const int t = team.lane();
    const int32_t base = first + t * W;     // class of a lane's first value; those of run u follow at u TEAM W (classes written out would be kept in registers)
    // The values that `in` takes go to the list. (Counted first and given their places by the wavefront, with one addition instead of one a value, it took
    // longer: 288 us for 264 on 4096 x 131072 bf16 logits, 20 alternatives.)
    auto collect = [&](auto in) {
        v.renew();
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float f[W];
            v.v[u].get(f);
#pragma unroll
            for (int w = 0; w < W; ++w)
                if (in(f[w], u * TEAM * W + w)) {
                    const int32_t at = atomicAdd(&to.count, 1);
                    if (at < TopSpace<TEAM>::CAP) to.key[at] = order_key(f[w], base + u * TEAM * W + w);
                }
        }
    };
    // the `need`-th largest lane maximum of the wavefront, its upper 16 bits (so a little less than it is), bit by bit
    const uint32_t o = order_of(lane_max), lowest = order_of(-3.4028234663852886e38f);
    auto largest = [&](int need) {
        uint32_t most = 0;
        for (int b = 31; b >= 16; --b)
            if (__popcll(__ballot(o >= (most | 1u << b))) >= need) most |= 1u << b;
        return most;
    };
    constexpr int WAVES = TEAM / 64;
    uint32_t most = largest((k + WAVES - 1) / WAVES);
    if (t == 0) to.count = 0;
    if constexpr (WAVES > 1) {
        if (lane_id() == 0) to.bound[threadIdx.x >> 6] = most;
        team.sync();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) most = min(most, to.bound[w]);
        if (most < lowest) {            // a wavefront with next to nothing: each by itself
            team.sync();
            most = largest(k);
            if (lane_id() == 0) to.bound[threadIdx.x >> 6] = most;
            team.sync();
#pragma unroll
            for (int w = 0; w < WAVES; ++w) most = max(most, to.bound[w]);
        }
    } else team.sync();
    const float bound = value_of(max(most, lowest));       // (-inf is no candidate)
    if (lane_max >= bound) collect([&](float f, int32_t) { return f >= bound; });
    team.sync();
    if (to.count <= TopSpace<TEAM>::CAP) return;
    // how many values are at least x, or are larger than x or equal to it with a class below c
    auto count = [&](float x, bool ties, int32_t c) {
        int here = 0;
        v.renew();
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float f[W];
            v.v[u].get(f);
#pragma unroll
            for (int w = 0; w < W; ++w) here += ties ? f[w] > x || (f[w] == x && u * TEAM * W + w < c - base) : f[w] >= x;
        }
        return (int)team.sum((float)here);          // (exact: a piece has fewer than 2^24 values)
    };
    uint32_t best = 0;
    bool fits = false;
    for (int b = 31; b >= 0 && !fits; --b) {        // the largest value that k values reach (finite: -inf is no candidate, and a row with +inf has none)
        const uint32_t cand = best | 1u << b;
        const float x = value_of(cand);
        if (!(x <= 3.4028234663852886e38f)) continue;
        const int here = count(x, false, 0);
        if (here >= k) { best = cand; fits = here <= TopSpace<TEAM>::CAP; }
    }
    const float x = value_of(best);
    int32_t below = 0x7fffffff;
    if (!fits) {                                    // more than fit reach it: the lowest classes of those equal to it
        int32_t c = 0;
        for (int b = 22; b >= 0; --b)
            if (count(x, true, c | 1 << b) < k) c |= 1 << b;
        below = c + 1;                              // (k values with a class below c + 1)
    }
    team.sync();
    if (t == 0) to.count = 0;
    team.sync();
    collect([&](float f, int32_t k) { return f > x || (f == x && k < below - base); });
    team.sync();
}

struct Logprobs {
    RowsOf z;
    const int32_t* d_n;
    int64_t row0;
    int32_t cap, classes;
    const int32_t* tokens;
    float inv_t, c;
    float *logprob, *entropy, *lse;
    int32_t k;
    int32_t* top_ids;
    float* top_logprobs;
    Sums* parts;                    // [cap][pieces]
    uint64_t* keys;                 // [cap][pieces][k], each piece's in order, 0: none
    int32_t pieces, piece;
};

__device__ __forceinline__ float log_share(const Logprobs& a, const Sums& r, float log_s, float z) {
    if (r.s != r.s) return NAN;
    return z == -INFINITY ? -INFINITY : log_ratio(r, a.inv_t, log_s, z);
}

// A row's answer and its logit, requested before the sums that they wait for.
template <typename T>
struct Answer {
    bool there;
    float z;
    __device__ __forceinline__ Answer(const Logprobs& a, int64_t i) {
        const int32_t tok = a.tokens[i];
        there = tok >= 0 && tok < a.classes;
        z = there ? to_f32(a.z.row<T>(i)[tok]) : 0.0f;
    }
};

template <typename T>
__device__ __forceinline__ void store_row(const Logprobs& a, int64_t i, const Answer<T>& answer, const Sums& r, float log_s) {
    a.logprob[i] = answer.there ? log_share(a, r, log_s, answer.z) : 0.0f;
    a.entropy[i] = r.s == 0.0f ? 0.0f : (log_s - r.h / r.s) * LN2;
    a.lse[i] = above(r.m) * a.inv_t + log_s * LN2;
}

__device__ __forceinline__ void store_top(const Logprobs& a, int64_t i, int32_t at, uint64_t key, const Sums& r, float log_s) {
    const bool none = key == 0 || r.s != r.s;
    a.top_ids[i * a.k + at] = none ? -1 : (int32_t)~(uint32_t)key;
    a.top_logprobs[i * a.k + at] = r.s != r.s ? NAN : none ? -INFINITY : log_share(a, r, log_s, value_of((uint32_t)(key >> 32)));
}

// A row, or a piece of one: sums, and the largest values. 4096 x 50001 fp32 with 20 alternatives: 148 us, 5.5 TB/s, the join in it 13 to 15; one row of 131072 bf16
// in 64 pieces 5 us and 5, the round trips of either launch; 4096 x 131072 bf16 204 us without alternatives (5.3 TB/s), 259 with 20, whose search holds a block's place longer than
// its share of memory takes.
template <typename T, int TEAM, int THREADS, int U, bool SPLIT>
__global__ void __launch_bounds__(THREADS, U == 8 ? 5 : U == 4 ? 7 : 8) logprobs_kernel(Logprobs a) {
    __shared__ float smem[2 * THREADS / 64];
    __shared__ TopSpace<TEAM> tops[THREADS / TEAM];
    Team<TEAM, THREADS> team(smem);
    const int t = team.lane();
    int64_t i = a.row0 + (int64_t)blockIdx.x * (THREADS / TEAM) + team.index();
    int32_t p = 0;
    if constexpr (SPLIT) {
        p = (int32_t)(blockIdx.x % (uint32_t)a.pieces);
        i = a.row0 + blockIdx.x / (uint32_t)a.pieces;
    }
    if (i >= rows_here(a.d_n, a.cap)) return;
    const int32_t first = SPLIT ? p * a.piece : 0, len = SPLIT ? min(a.piece, a.classes - first) : a.classes;
    Piece<T, U, TEAM, true> v;
    v.load(a.z.row<T>(i) + first, len, t);
    const Sums mine = v.template lane_sums<true>(a.c), r = team_sums<true>(mine, a.c, team);
    const float log_s = log2f(r.s);
    if (t == 0) {
        if constexpr (SPLIT) a.parts[i * a.pieces + p] = r;
        else store_row<T>(a, i, Answer<T>(a, i), r, log_s);
    }
    if (a.k == 0) return;
    TopSpace<TEAM>& top = tops[team.index()];
    top_candidates(v, mine.m, first, a.k, top, team);
    const int32_t count = min(top.count, TopSpace<TEAM>::CAP);
    auto put = [&](int32_t at, uint64_t key) {
        if constexpr (SPLIT) a.keys[(i * a.pieces + p) * a.k + at] = key;
        else store_top(a, i, at, key, r, log_s);
    };
    for (int32_t j = t; j < count; j += TEAM) {
        const uint64_t key = top.key[j];
        int32_t rank = 0;
#pragma unroll 8
        for (int32_t o = 0; o < count; ++o) rank += top.key[o] > key;
        if (rank < a.k) put(rank, key);
    }
    for (int32_t j = count + t; j < a.k; j += TEAM) put(j, 0);
}

// A row from its pieces. Of every piece's list the j-th key is looked at, j the least with j pieces >= k: r = ceil(k / j) lists whose j-th key reaches a bound hold k keys
// that do, so the r-th largest of those keys is a bound; the keys that reach it are ranked against each other. (With more lists than lanes a lane
// takes the largest of several lists' first keys.) Where large values stand in few pieces more keys than there is room for may reach the bound: then
// every key is ranked by a search in every other list.
template <typename T, int TEAM>
__global__ void __launch_bounds__(256) logprobs_join_kernel(Logprobs a) {
    constexpr int CAP = TEAM * 4, ROWS = 256 / TEAM;
    __shared__ float smem[8];
    __shared__ uint64_t lane_key[256], cands[ROWS][CAP], bounds[ROWS];
    __shared__ int32_t counts[ROWS];
    Team<TEAM, 256> team(smem);
    const int64_t i = a.row0 + (int64_t)blockIdx.x * ROWS + team.index();
    if (i >= rows_here(a.d_n, a.cap)) return;
    const int32_t t = team.lane(), all = a.pieces * a.k;
    const Answer<T> answer(a, i);
    const uint64_t* const keys = a.keys + i * all;
    uint64_t *const first = lane_key + team.index() * TEAM, *const cand = cands[team.index()], &bound = bounds[team.index()];
    int32_t& count = counts[team.index()];
    if (a.k > 0) {
        const int32_t j = (a.k + a.pieces - 1) / a.pieces, need = (a.k + j - 1) / j, lanes = min(a.pieces, TEAM);
        uint64_t mine = 0;
        for (int32_t p = t; p < a.pieces; p += TEAM) mine = max(mine, keys[p * a.k + j - 1]);
        first[t] = mine;
        if (t == 0) { bound = 1; count = 0; }
        team.sync();
        int32_t rank = 0;
#pragma unroll 8
        for (int32_t o = 0; o < lanes; ++o) rank += first[o] > mine;
        if (rank == need - 1 && mine != 0) bound = mine;        // (keys are all different; fewer than `need` above 0: all of them)
    }
    const Sums r = join_sums(a.parts + i * a.pieces, a.pieces, a.c, team);
    const float log_s = log2f(r.s);
    if (t == 0) store_row(a, i, answer, r, log_s);
    if (a.k == 0) return;
    team.sync();
    for (int32_t e = t; e < all; e += TEAM) {
        const uint64_t key = keys[e];
        if (key >= bound) {
            const int32_t at = atomicAdd(&count, 1);
            if (at < CAP) cand[at] = key;
        }
    }
    team.sync();
    if (count <= CAP) {
        for (int32_t e = t; e < count; e += TEAM) {
            const uint64_t key = cand[e];
            int32_t rank = 0;
#pragma unroll 8
            for (int32_t o = 0; o < count; ++o) rank += cand[o] > key;
            if (rank < a.k) store_top(a, i, rank, key, r, log_s);
        }
    } else {
        for (int32_t e = t; e < all; e += TEAM) {
            const uint64_t key = keys[e];
            if (key < bound) continue;
            const int32_t own = e / a.k;
            int32_t rank = e - own * a.k;                       // larger ones in its own list
            for (int32_t o = 0; o < a.pieces && rank < a.k; ++o) {
                if (o == own) continue;
                const uint64_t* l = keys + o * a.k;
                int32_t lo = 0, hi = a.k;
                while (lo < hi) {
                    const int32_t mid = (lo + hi) >> 1;
                    if (l[mid] > key) lo = mid + 1; else hi = mid;
                }
                rank += lo;
            }
            if (rank < a.k) store_top(a, i, rank, key, r, log_s);
        }
    }
    for (int32_t e = count + t; e < a.k; e += TEAM) store_top(a, i, e, 0, r, log_s);
}

// The gradient of log probability and entropy: one read, one write. 4096 x 32000 bf16: 91 us, 5.8 TB/s.
template <typename T, int TEAM, int U>
__global__ void __launch_bounds__(256) logprobs_grad_kernel(RowsOf z, const int32_t* d_n, int64_t row0, int32_t cap, int32_t classes, int32_t pieces, const int32_t* __restrict__ tokens,
                                                            float inv_t, const float* __restrict__ lse, const float* __restrict__ entropy, const float* __restrict__ g_logprob,
                                                            const float* __restrict__ g_entropy, RowsOf grad) {
    constexpr int W = Piece<T, U, TEAM>::W, PIECE = W * U * TEAM;
    const int t = Team<TEAM, 256>::lane();
    const int64_t i = row0 + (TEAM == 256 ? blockIdx.x / (uint32_t)pieces : (int64_t)blockIdx.x * (256 / TEAM) + Team<TEAM, 256>::index());
    const int32_t first = TEAM == 256 ? (int32_t)(blockIdx.x % (uint32_t)pieces) * PIECE : 0, len = min(PIECE, classes - first);
    if (i >= rows_here(d_n, cap)) return;
    Piece<T, U, TEAM, true> v;
    v.load(z.row<T>(i) + first, len, t);
    const int32_t tok = tokens[i];
    // A row's lse is rounded: where that is more than a share's logarithm (rows masked throughout, by -1e9 or less) z / T - lse may come out far above 0, and beyond fp32 as inf - inf. No
    // share is larger than 1, so no logarithm is above 0; an lse of -inf leaves no share. (The minimum drops a NaN: a row whose lse is one takes it from gl.)
    const float given = lse[i], l = given == -INFINITY ? INFINITY : given, gh = g_entropy ? g_entropy[i] : 0.0f;
    const float gl = given != given ? NAN : g_logprob && tok >= 0 && tok < classes ? g_logprob[i] : 0.0f;
    const float h = g_entropy ? entropy[i] : 0.0f;      // (0 times an entropy that is not finite would be NaN)
    RowStore<T, W, true> store(grad.row<T>(i) + first, len);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int32_t c = v.at(t, u);
        float f[W];
        v.v[u].get(f);
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float log_p = fminf(f[w] * inv_t - l, 0.0f), p = __builtin_amdgcn_exp2f(log_p * LOG2E);
            const float d = p == 0.0f ? 0.0f : -(p * (gl + gh * (log_p + h)));
            f[w] = (first + c + w == tok ? gl + d : d) * inv_t;
        }
        Run<T, W> o;
        o.set(f);
        store.put(c, o);
    }
    store.finish();
}

static int32_t check_logits(const char* who, const void* z, no_dtype dt, int64_t stride, int32_t n, int32_t classes, float temperature) {
    NO_REQUIRE(dt == NO_F32 || dt == NO_BF16, NO_ERR_INVALID_ARG, "%s: logits are NO_F32 or NO_BF16", who);
    NO_REQUIRE(n >= 0 && classes >= 1, NO_ERR_INVALID_ARG, "%s: bad sizes", who);
    NO_REQUIRE(classes <= NO_MAX_CLASSES, NO_ERR_UNSUPPORTED, "%s: more than %d classes", who, NO_MAX_CLASSES);
    NO_REQUIRE(temperature > 0.0f && temperature < INFINITY && LOG2E / temperature < INFINITY, NO_ERR_INVALID_ARG,
               "%s: the temperature must be positive and finite, and so must its inverse", who);
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

// Rows in pieces: as many as fill the chip while rows are few, of a multiple of a block's runs. (100 x 50001 fp32, log probabilities: at least 1024 blocks 14.8 us, 512 or 2048 16.1.)
struct Cut {
    int32_t u, piece, pieces;
    Cut(int32_t n, int32_t classes, int32_t w, int32_t most_u) {
        u = most_u;
        while (u > 1 && (int64_t)n * ceil_div(classes, 256 * w * u) < 1024) u >>= 1;
        piece = 256 * w * u;
        pieces = (int32_t)ceil_div(classes, piece);
    }
};
static int32_t most_pieces(int32_t n, int32_t classes) { return Cut(n, classes, 4, 8).pieces; }      // (of either type: bf16 pieces of 4 runs are as long)

// Rows of more values than MANY, whose arithmetic takes one block long, and fewer than FEW_ROWS of them: in pieces all over the chip (48 x 131072 bf16: 17.0 us, a block a row 19.3; 64: 19.0 and 19.8;
// 96: 22.1 and 21.2; but 20 x 50000 bf16 13.5 and 10.9, 48 x 50000 fp32 15.5 and 11.5). For the loss alone pieces do where there are rows for the chip (16384 x 32768 bf16:
// 6.2 TB/s), and a block a row where there are not (200 x 30000 fp32: 8.1 us, pieces 10.9).
constexpr int64_t FEW_ROWS = 64;
constexpr int32_t MANY = 65536;

// A launch holds fewer than 2^32 threads, 2^21 blocks of 1024 among them: more rows go in several.
template <typename F>
static void in_slabs(int64_t rows, int64_t rows_per_launch, F launch) {
    for (int64_t r = 0; r < rows; r += rows_per_launch) launch(r, rows - r < rows_per_launch ? rows - r : rows_per_launch);
}
constexpr int64_t MOST_BLOCKS = 1 << 21;

template <typename T>
static int32_t distill(const char* who, Distill a, void* ws, hipStream_t st) {
    constexpr int W = 16 / (int)sizeof(T);
    const int64_t units = ceil_div(a.classes, W);
#define NO_ROW(TEAM, THREADS, U)                                                                                                                  \
    in_slabs(a.cap, MOST_BLOCKS * (THREADS / TEAM), [&](int64_t row0, int64_t rows) {                                                             \
        a.row0 = row0;                                                                                                                            \
        hipLaunchKernelGGL((distill_row_kernel<T, TEAM, THREADS, U>), dim3((unsigned)ceil_div(rows, THREADS / TEAM)), dim3(THREADS), 0, st, a);   \
    })
    // (from a given lse every piece of a row goes by itself, but short rows by wavefronts, which share the work on the teacher's entries)
    // Runs a lane: as few as hold the row, where a step less was measured to pay (50000 x 602 fp32: three runs 59.3 us, four 62.1; 32000 x 10000 bf16: three runs of 512 lanes 246, four 263;
    // 8000 x 80000 bf16: ten of 1024 lanes 518, sixteen 596).
    const bool row = a.lse_in ? units <= 256 : units <= 2048 || (units <= 16384 && (a.grad.p ? a.classes <= MANY || a.cap >= FEW_ROWS : a.classes <= MANY && a.cap < 256));
    if (row) {
        if (units <= 64) NO_ROW(64, 256, 1);
        else if (units <= 128) NO_ROW(64, 256, 2);
        else if (units <= 192) NO_ROW(64, 256, 3);
        else if (units <= 256) NO_ROW(64, 256, 4);
        else if (units <= 512) NO_ROW(256, 256, 2);
        else if (units <= 768) NO_ROW(256, 256, 3);
        else if (units <= 1024) NO_ROW(256, 256, 4);
        else if (units <= 1536) NO_ROW(512, 512, 3);
        else if (units <= 2048) NO_ROW(512, 512, 4);
        else if (units <= 4096) NO_ROW(1024, 1024, 4);
        else if (units <= 8192) NO_ROW(1024, 1024, 8);
        else if (units <= 10240) NO_ROW(1024, 1024, 10);
        else if (units <= 12288) NO_ROW(1024, 1024, 12);
        else if (units <= 14336) NO_ROW(1024, 1024, 14);
        else NO_ROW(1024, 1024, 16);
        return launch_status(who);
    }
#undef NO_ROW
    // (from a given lse, which needs no sums of the pieces, of four runs a lane: 4096 x 50001 fp32 286 us, of eight 304)
    const Cut cut(a.cap, a.classes, W, a.lse_in ? 4 : 8);
    a.piece = cut.piece;
    a.pieces = cut.pieces;
    a.parts = (Sums*)ws;
#define NO_PIECES(KERNEL)                                                                                              \
    in_slabs(a.cap, MOST_BLOCKS / a.pieces, [&](int64_t row0, int64_t rows) {                                          \
        const dim3 grid((unsigned)(rows * a.pieces));                                                                  \
        a.row0 = row0;                                                                                                 \
        if (cut.u == 8) hipLaunchKernelGGL((KERNEL<T, 256, 8>), grid, dim3(256), 0, st, a);                            \
        else if (cut.u == 4) hipLaunchKernelGGL((KERNEL<T, 256, 4>), grid, dim3(256), 0, st, a);                       \
        else if (cut.u == 2) hipLaunchKernelGGL((KERNEL<T, 256, 2>), grid, dim3(256), 0, st, a);                       \
        else hipLaunchKernelGGL((KERNEL<T, 256, 1>), grid, dim3(256), 0, st, a);                                       \
    })
    if (!a.lse_in) {
        NO_PIECES(distill_sums_kernel);
        in_slabs(a.cap, MOST_BLOCKS * 4, [&](int64_t row0, int64_t rows) {
            a.row0 = row0;
            hipLaunchKernelGGL(distill_loss_kernel<T>, dim3((unsigned)ceil_div(rows, 4)), dim3(256), 0, st, a);
        });
    }
    if (a.grad.p) NO_PIECES(distill_grad_kernel);
#undef NO_PIECES
    return launch_status(who);
}

static int32_t distill(const char* who, const void* z, no_dtype dt, int64_t stride, const int32_t* d_n, int32_t cap, int32_t classes, const int32_t* ids,
                       const float* logits, int32_t k, float temperature, const float* weight, float* loss, const float* lse_in, float* lse_out, void* grad,
                       int64_t grad_stride, void* ws, hipStream_t st) {
    const float inv_t = 1.0f / temperature;
    const Distill a{rows_of(z, stride), d_n, 0, cap, classes, ids, logits, k, temperature, inv_t, inv_t * LOG2E, weight, loss, lse_in, lse_out, rows_of(grad, grad_stride),
                    nullptr, 1, classes};
    return dt == NO_F32 ? distill<float>(who, a, ws, st) : distill<bf16_t>(who, a, ws, st);
}

// Pieces of these rows, or of any that are fewer or shorter (whose pieces may be more: they are made shorter until there are 1024 blocks for them, so that short ones are fewer than 2048).
static int64_t pieces_room(int32_t n, int32_t classes) {
    const int64_t longest = (int64_t)n * ceil_div(classes, 256 * 4 * 8), shortest = (int64_t)n * ceil_div(classes, 256 * 4), brief = shortest < 2048 ? shortest : 2048;
    return longest > brief ? longest : brief;
}
static size_t parts_room(int32_t n, int32_t classes) { return ((size_t)pieces_room(n, classes) * sizeof(Sums) + 15) / 16 * 16; }
static size_t parts_bytes(int32_t n, int32_t classes) { return ((size_t)n * (size_t)most_pieces(n, classes) * sizeof(Sums) + 15) / 16 * 16; }

template <typename T>
static int32_t logprobs(const char* who, Logprobs a, void* ws, hipStream_t st) {
    constexpr int W = 16 / (int)sizeof(T);
    const int64_t units = ceil_div(a.classes, W);
#define NO_ROW(TEAM, U)                                                                                                                        \
    in_slabs(a.cap, MOST_BLOCKS * (256 / TEAM), [&](int64_t row0, int64_t rows) {                                                              \
        a.row0 = row0;                                                                                                                         \
        hipLaunchKernelGGL((logprobs_kernel<T, TEAM, 256, U, false>), dim3((unsigned)ceil_div(rows, 256 / TEAM)), dim3(256), 0, st, a);        \
    })
    if (units <= 64) NO_ROW(64, 1);
    else if (units <= 128) NO_ROW(64, 2);
    else if (units <= 192) NO_ROW(64, 3);
    else if (units <= 256) NO_ROW(64, 4);
    else if (units <= 512) NO_ROW(256, 2);
    else if (units <= 768) NO_ROW(256, 3);
    else if (units <= 1024) NO_ROW(256, 4);
    else if (W == 4 && units <= 2048) NO_ROW(256, W == 4 ? 8 : 4);
#undef NO_ROW
    else {
        const Cut cut(a.cap, a.classes, W, 32 / W);
        a.piece = cut.piece;
        a.pieces = cut.pieces;
        a.parts = (Sums*)ws;
        a.keys = (uint64_t*)((char*)ws + parts_bytes(a.cap, a.classes));
        in_slabs(a.cap, MOST_BLOCKS / a.pieces, [&](int64_t row0, int64_t rows) {
            const dim3 grid((unsigned)(rows * a.pieces));
            a.row0 = row0;
            if (cut.u == 8) hipLaunchKernelGGL((logprobs_kernel<T, 256, 256, W == 4 ? 8 : 4, true>), grid, dim3(256), 0, st, a);
            else if (cut.u == 4) hipLaunchKernelGGL((logprobs_kernel<T, 256, 256, 4, true>), grid, dim3(256), 0, st, a);
            else if (cut.u == 2) hipLaunchKernelGGL((logprobs_kernel<T, 256, 256, 2, true>), grid, dim3(256), 0, st, a);
            else hipLaunchKernelGGL((logprobs_kernel<T, 256, 256, 1, true>), grid, dim3(256), 0, st, a);
            // many rows of few pieces: a wavefront each, without barriers (4096 x 50001: 149.1 us in all, by blocks 151.1; one row of 64 pieces 10.3 and 10.0)
            if (rows >= 256 && a.pieces <= 64) hipLaunchKernelGGL((logprobs_join_kernel<T, 64>), dim3((unsigned)ceil_div(rows, 4)), dim3(256), 0, st, a);
            else hipLaunchKernelGGL((logprobs_join_kernel<T, 256>), dim3((unsigned)rows), dim3(256), 0, st, a);
        });
    }
    return launch_status(who);
}

template <typename T>
static int32_t logprobs_grad(const char* who, const RowsOf& z, const int32_t* d_n, int32_t cap, int32_t classes, const int32_t* tokens, float inv_t, const float* lse,
                             const float* entropy, const float* g_logprob, const float* g_entropy, const RowsOf& grad, hipStream_t st) {
    const int64_t units = ceil_div(classes, 16 / (int)sizeof(T));
    // (pieces of four runs a lane: 4096 x 32000 bf16 91 us, 4096 x 50001 fp32 287, 20000 x 3000 fp32 85; of eight 95, 313 and 85; of two 91, 278 and 94)
    const Cut cut(cap, classes, 16 / (int)sizeof(T), 4);
#define NO_GRAD(TEAM, U) hipLaunchKernelGGL((logprobs_grad_kernel<T, TEAM, U>), grid, dim3(256), 0, st, z, d_n, row0, cap, classes, cut.pieces, tokens, inv_t, lse, entropy, g_logprob, g_entropy, grad)
    if (units <= 256) {
        in_slabs(cap, MOST_BLOCKS * 4, [&](int64_t row0, int64_t rows) {
            const dim3 grid((unsigned)ceil_div(rows, 4));
            if (units <= 64) NO_GRAD(64, 1); else if (units <= 128) NO_GRAD(64, 2); else NO_GRAD(64, 4);
        });
        return launch_status(who);
    }
    in_slabs(cap, MOST_BLOCKS / cut.pieces, [&](int64_t row0, int64_t rows) {
        const dim3 grid((unsigned)(rows * cut.pieces));
        if (cut.u == 4) NO_GRAD(256, 4); else if (cut.u == 2) NO_GRAD(256, 2); else NO_GRAD(256, 1);
    });
#undef NO_GRAD
    return launch_status(who);
}

}  // namespace no

using namespace no;

extern "C" size_t no_distill_ws_bytes(int32_t n_rows_cap, int32_t n_classes) {
    if (n_rows_cap < 0 || n_classes < 1 || n_classes > NO_MAX_CLASSES) return 0;
    return 16 + parts_room(n_rows_cap, n_classes);
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
                   d_lse, nullptr, 0, d_ws, (hipStream_t)stream);
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
                   nullptr, d_grad_z, grad_stride_bytes, nullptr, (hipStream_t)stream);
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
                   d_lse, d_grad_z, grad_stride_bytes, d_ws, (hipStream_t)stream);
}

extern "C" size_t no_logprobs_ws_bytes(int32_t n_rows_cap, int32_t n_classes, int32_t k) {
    if (n_rows_cap < 0 || n_classes < 1 || n_classes > NO_MAX_CLASSES || k < 0 || k > NO_MAX_ALTERNATIVES) return 0;
    return 16 + parts_room(n_rows_cap, n_classes) + (size_t)pieces_room(n_rows_cap, n_classes) * (size_t)k * 8;
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
    const float inv_t = 1.0f / temperature;
    const Logprobs a{rows_of(d_z, z_stride_bytes), d_n_rows, 0, n_rows_cap, n_classes, d_tokens, inv_t, inv_t * LOG2E, d_logprob, d_entropy, d_lse, k, d_top_ids, d_top_logprobs,
                     nullptr, nullptr, 1, n_classes};
    return dt == NO_F32 ? logprobs<float>(who, a, d_ws, (hipStream_t)stream) : logprobs<bf16_t>(who, a, d_ws, (hipStream_t)stream);
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
    const RowsOf z = rows_of(d_z, z_stride_bytes), g = rows_of(d_grad_z, grad_stride_bytes);
    const float inv_t = 1.0f / temperature;
    hipStream_t st = (hipStream_t)stream;
    return dt == NO_F32 ? logprobs_grad<float>(who, z, d_n_rows, n_rows_cap, n_classes, d_tokens, inv_t, d_lse, d_entropy, d_grad_logprob, d_grad_entropy, g, st)
                        : logprobs_grad<bf16_t>(who, z, d_n_rows, n_rows_cap, n_classes, d_tokens, inv_t, d_lse, d_entropy, d_grad_logprob, d_grad_entropy, g, st);
}
