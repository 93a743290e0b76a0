// Log probabilities of labels under a row's softmax, with entropy, normaliser and the most likely classes, in one pass
// over the logits; and their gradient.  Bound by memory: the forward pass reads every logit once (a row's top classes
// cost reads of the few vectors that can hold them), the gradient reads and writes every logit once.
//
// Forward.  A thread keeps, over the vectors of 16 bytes that it reads, the largest value m so far, s = sum 2^((x-m) L) and
// t = sum 2^((x-m) L) (x-m) L with L = log2(e), and rescales s and t when m grows; joining two such triples is the same
// step, so that threads, wavefronts and workgroups of a row join theirs in a fixed order.  With the total
//     lse = m + ln s,   logprob = (x_label - m) - ln s,   entropy = ln s - ln 2 * t / s.
// The sums are fp32: 512 terms in a thread at 131072 classes, then a tree.  Which terms a thread has follows from where the row
// begins in memory (skew_of) and from the number of rows, classes and top classes (shape_of): the same row in another batch
// can differ in its last bits.
//
// Top classes.  Classes are ordered by one 64-bit key: the value's bits made monotonic, above the complement of the class
// number, so that no two are equal.  Every thread of a row knows the largest value of its own vectors; the top_k-th largest
// of these (to 16 bits, by bisection: count the threads at or above a bit pattern) bounds the top_k-th largest class from
// below.  The few classes at or above the bound are listed -- from the group of vectors that holds a thread's largest, which
// it has kept in registers, or by reading the thread's vectors again where a second group reaches the bound -- and each takes
// the place that the number of larger keys in the list says.  The list does not hold them where more than 256 classes reach the
// bound: many equal ones or, in fp32, many whose values share their upper 16 bits with it (near 10 a band of 1/16).  Then, and
// for rows with a NaN, each wavefront takes its largest keys one by one and the lists are merged.  (fp32 rows of distinct values
// within 0.02, against rows of deviation 3: 8192 x 4200 with 5 top classes 182 and 29 us, 4096 x 50021 with 8 810 and 146,
// 1 x 65537 with 20 37 and 16.)
#include <algorithm>

#include "kernels.h"
#include "quads.h"

namespace rvn {

namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.69314718055994531f;
constexpr float kLowest = -3.402823466e38f;

typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef u4 u4_any __attribute__((aligned(2)));

template <typename T>
struct Vec;  // 16 bytes of a row as fp32 values, and back
template <>
struct Vec<float> {
    static constexpr int E = 4, FLY = 4;  // FLY: vectors a thread requests before it uses the first
    static __device__ __forceinline__ float one(const void *p, int64_t i) { return static_cast<const float *>(p)[i]; }
    static __device__ __forceinline__ void widen(u4 w, float (&v)[E]) {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = __uint_as_float(w[e]);
    }
    static __device__ __forceinline__ u4 narrow(const float (&v)[E]) {
        return u4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    }
    static __device__ __forceinline__ void put(void *p, int64_t i, float v) { static_cast<float *>(p)[i] = v; }
};
struct Bf16 {
    uint16_t bits;
};
template <>
struct Vec<Bf16> {
    static constexpr int E = 8, FLY = 2;
    static __device__ __forceinline__ float one(const void *p, int64_t i) {
        return __uint_as_float((uint32_t)static_cast<const uint16_t *>(p)[i] << 16);
    }
    static __device__ __forceinline__ void widen(u4 w, float (&v)[E]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[2 * e] = __uint_as_float(w[e] << 16);
            v[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ uint32_t pair(float lo, float hi) {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        typedef float f2 __attribute__((ext_vector_type(2)));
        const f2 v = {lo, hi};
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));  // nearest even
    }
    static __device__ __forceinline__ u4 narrow(const float (&v)[E]) {
        return u4{pair(v[0], v[1]), pair(v[2], v[3]), pair(v[4], v[5]), pair(v[6], v[7])};
    }
    static __device__ __forceinline__ void put(void *p, int64_t i, float v) {
        static_cast<uint16_t *>(p)[i] = (uint16_t)pair(v, 0.f);
    }
};

// The vector that starts at class `at` (which may lie before the row's first) of `classes` of a row; what lies outside
// these reads as -infinity.  Memory at classes lo .. hi - 1 of the row belongs to the matrix: a vector in there is read at
// once and its outsiders dropped.
template <typename T>
__device__ __forceinline__ void load_vec(const T *row, int at, int classes, int lo, int hi, float (&v)[Vec<T>::E]) {
    constexpr int E = Vec<T>::E;
    if (at + E <= 0 || at >= classes) {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = -INFINITY;
    } else if (at >= lo && at + E <= hi) {
        Vec<T>::widen(*reinterpret_cast<const u4_any *>(row + at), v);
        if (at < 0 || at + E > classes) {
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = at + e >= 0 && at + e < classes ? v[e] : -INFINITY;
        }
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = at + e >= 0 && at + e < classes ? Vec<T>::one(row, at + e) : -INFINITY;
    }
}
// How far a matrix reaches before the first and behind the last class of row `at`, up to a cache line.
__device__ __forceinline__ int reach(int64_t rows_away, int64_t ld) { return rows_away == 0 ? 0 : ld < 64 ? (int)ld : 64; }

// Elements from the last border to p: the vectors of a row start that much before it, so that their accesses are aligned
// wherever the row begins; from 64 vectors on to whole cache lines, so that neighbouring workgroups write no line together.
// (Rows of an odd number of bf16 logits: 4096 x 50021 in 98.6 us with vectors from the row's start, 86 on 16-byte borders.)
template <typename T>
__device__ __forceinline__ int skew_of(const T *p, int classes) {
    const uintptr_t border = classes >= 64 * Vec<T>::E ? 128 : 16;
    return (int)((reinterpret_cast<uintptr_t>(p) & (border - 1)) / sizeof(T));
}

// Bits that order as the values do, -0 as 0, NaN above all; never 0, and never 0xffffffff, which is above every key.
constexpr uint32_t kNanOrder = 0xff800001u, kLowestOrder = 0x007fffffu;  // (of -infinity)
__device__ __forceinline__ uint32_t order_bits(float x) {
    if (x != x) return kNanOrder;
    const uint32_t b = __float_as_uint(x + 0.f);
    return b ^ ((int32_t)b < 0 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t order) {
    if (order == kNanOrder) return __uint_as_float(0x7fc00000u);
    return __uint_as_float(order ^ ((int32_t)order < 0 ? 0x80000000u : 0xffffffffu));
}

__device__ __forceinline__ uint32_t wave_most(uint32_t v) {  // over the 64 lanes, all of them active
#define RVN_STEP(ctrl, rows) v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, rows, 0xf, false))
    RVN_STEP(0x111, 0xf);  // row_shr 1, 2, 4, 8: the last lane of each row of 16 has the row's
    RVN_STEP(0x112, 0xf);
    RVN_STEP(0x114, 0xf);
    RVN_STEP(0x118, 0xf);
    RVN_STEP(0x142, 0xa);  // row_bcast 15 and 31: lane 63 has all
    RVN_STEP(0x143, 0xc);
#undef RVN_STEP
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

struct alignas(8) Key {
    uint32_t hi, lo;  // order bits; complement of the class number.  {0, 0}: none
};
__device__ __forceinline__ bool less(Key a, Key b) { return ((uint64_t)a.hi << 32 | a.lo) < ((uint64_t)b.hi << 32 | b.lo); }
__device__ __forceinline__ Key wave_most(Key k) {
    const uint32_t hi = wave_most(k.hi);
    return Key{hi, wave_most(k.hi == hi ? k.lo : 0u)};
}

// Largest of the lanes' values, none of them NaN.
__device__ __forceinline__ float wave_largest(float v) {
    const uint32_t most = wave_most(order_bits(v));
    return value_of(most);
}

struct Sums {
    float m, s, t;
};
__device__ __forceinline__ Sums join(Sums a, Sums b) {
    const float m = fmaxf(a.m, b.m);
    const float da = (a.m - m) * kLog2e, db = (b.m - m) * kLog2e;
    const float fa = __builtin_amdgcn_exp2f(da), fb = __builtin_amdgcn_exp2f(db);
    // (differences below -200 have a factor of 0: clamped, so that 0 * -infinity cannot arise)
    return Sums{m, a.s * fa + b.s * fb, fa * (a.t + a.s * fmaxf(da, -200.f)) + fb * (b.t + b.s * fmaxf(db, -200.f))};
}
// The join of the 64 lanes' sums, in every lane: to the largest m of all first, then three plain sums' worth of lane moves.
__device__ __forceinline__ Sums wave_join(Sums v) {
    const float m = wave_largest(v.m), down = (v.m - m) * kLog2e, f = __builtin_amdgcn_exp2f(down);
    return Sums{m, wave_total(v.s * f), wave_total(f * (v.t + v.s * fmaxf(down, -200.f)))};
}

// A team of NT threads on `length` classes of a row from class `first`: vector v of that part, its classes
// v * E - skew .. + E - 1, belongs to thread v % NT.
template <typename T>
struct Part {
    const T *row;  // at class `first`
    int first, length, lo, hi, skew, vecs, NT;
    // classes f .. f + l - 1 of row `at` of a matrix
    __device__ __forceinline__ Part(const T *x, int64_t at, int64_t rows, int64_t ld, int classes, int f, int l, int nt)
        : row(x + at * ld + f), first(f), length(l), lo(-f - reach(at, ld)), hi(classes - f + reach(rows - 1 - at, ld)),
          skew(skew_of(row, l)), vecs((l + skew + Vec<T>::E - 1) / Vec<T>::E), NT(nt) {}
    __device__ __forceinline__ int at(int v) const { return v * Vec<T>::E - skew; }
    __device__ __forceinline__ void load(int v, float (&x)[Vec<T>::E]) const { load_vec(row, at(v), length, lo, hi, x); }
};

template <typename T>
__device__ __forceinline__ void add_values(Sums &a, const float (&x)[Vec<T>::FLY][Vec<T>::E], float most) {
    constexpr int E = Vec<T>::E;
    const float m = fmaxf(a.m, most);
    const float down = (a.m - m) * kLog2e, f = __builtin_amdgcn_exp2f(down);
    a.t = f * (a.t + a.s * fmaxf(down, -200.f));
    a.s *= f;
    a.m = m;
#pragma unroll
    for (int u = 0; u < Vec<T>::FLY; ++u)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float d = (x[u][e] - m) * kLog2e, w = __builtin_amdgcn_exp2f(d);
            a.s += w;
            a.t = fmaf(w, fmaxf(d, -200.f), a.t);  // (a NaN stays one in w)
        }
}

// The largest value of a thread's vectors, the first group of vectors that holds it and what it holds, and the largest
// value of the others.
template <int FLY>
struct Top {
    float value, second;
    int group;
    u4 kept[FLY];
};

// TOP: fills `top` (else it is not looked at).
template <bool TOP, typename T>
__device__ __forceinline__ Sums stream(const Part<T> &p, int thread, Top<Vec<T>::FLY> &top) {
    constexpr int E = Vec<T>::E;
    Sums a{kLowest, 0.f, 0.f};
    if constexpr (TOP) {
        top.value = top.second = -INFINITY;
        top.group = 0;
#pragma unroll
        for (int u = 0; u < Vec<T>::FLY; ++u) top.kept[u] = u4{0u, 0u, 0u, 0u};
    }
    for (int g = 0; thread + g * Vec<T>::FLY * p.NT < p.vecs; ++g) {
        float x[Vec<T>::FLY][E];
        u4 raw[Vec<T>::FLY];
        const int v0 = thread + g * Vec<T>::FLY * p.NT;
        if (p.at(v0) >= 0 && p.at(v0 + (Vec<T>::FLY - 1) * p.NT) + E <= p.length) {
#pragma unroll
            for (int u = 0; u < Vec<T>::FLY; ++u) raw[u] = *reinterpret_cast<const u4_any *>(p.row + p.at(v0 + u * p.NT));
        } else {
#pragma unroll
            for (int u = 0; u < Vec<T>::FLY; ++u) {
                if (v0 + u * p.NT < p.vecs) {
                    p.load(v0 + u * p.NT, x[u]);
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e) x[u][e] = -INFINITY;
                }
                raw[u] = Vec<T>::narrow(x[u]);  // (exact: these were the type's own values)
            }
        }
#pragma unroll
        for (int u = 0; u < Vec<T>::FLY; ++u) Vec<T>::widen(raw[u], x[u]);
        float most = x[0][0];
#pragma unroll
        for (int u = 0; u < Vec<T>::FLY; ++u)
#pragma unroll
            for (int e = 0; e < E; ++e) most = fmaxf(most, x[u][e]);
        if constexpr (TOP) {
            const bool up = g == 0 || most > top.value;
            if (g > 0) top.second = fmaxf(top.second, up ? top.value : most);
            top.value = up ? most : top.value;
            top.group = up ? g : top.group;
#pragma unroll
            for (int u = 0; u < Vec<T>::FLY; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) top.kept[u][i] = up ? raw[u][i] : top.kept[u][i];
        }
        add_values<T>(a, x, most);
    }
    return a;
}

// ---- the top classes of a part, by a bound -------------------------------------------------------------------------

constexpr int kListed = 256;  // keys that a team's list holds

template <int NW>
struct TeamLds {
    Key list[kListed];
    uint32_t tops[NW * 64];
    int listed;
};

template <int NW>
__device__ __forceinline__ void team_barrier() {
    if constexpr (NW == 1) wave_exchange();
    else __syncthreads();
}

// Lists the classes of vector v, which holds x, whose values reach `least`.
template <typename T>
__device__ __forceinline__ void list_values(const Part<T> &p, int v, const float (&x)[Vec<T>::E], float least, Key *list, int *listed) {
#pragma unroll
    for (int e = 0; e < Vec<T>::E; ++e) {
        if (!(x[e] >= least)) continue;
        const int i = p.at(v) + e;
        if (i < 0 || i >= p.length) continue;
        const int slot = atomicAdd(listed, 1);
        if (slot < kListed) list[slot] = Key{order_bits(x[e]), 0xffffffffu - (uint32_t)(p.first + i)};
    }
}

// Fills lds.list with lds.listed keys among which are the part's top_k largest (or all that it has).  More than kListed:
// the list is not complete.  The part holds no NaN.  All threads of the team call it; the last barrier is the caller's.
template <typename T, int NW>
__device__ __forceinline__ void list_top(const Part<T> &p, int thread, const Top<Vec<T>::FLY> &top, int top_k, TeamLds<NW> &lds) {
    const bool has = thread < p.vecs;
    const uint32_t mine = has ? order_bits(top.value) : 0u;
    uint32_t seen[NW];
    if (thread == 0) lds.listed = 0;
    if constexpr (NW == 1) {
        seen[0] = mine;
    } else {
        lds.tops[thread] = mine;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < NW; ++w) seen[w] = lds.tops[w * 64 + (thread & 63)];
    }
    team_barrier<NW>();
    uint32_t bound = 0;
    for (int bit = 31; bit >= 16; --bit) {
        if (bit == 31 && min(p.vecs, p.NT) <= top_k) break;  // no more threads than that have a vector: all is listed
        const uint32_t next = bound | 1u << bit;
        int count = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) count += __popcll(__ballot(seen[w] >= next));
        if (count >= top_k) bound = next;
        if (count == top_k) break;  // (uniform) exactly these
    }
    const float least = bound <= kLowestOrder ? -INFINITY : value_of(bound);  // order bits reach `bound`: the value reaches this
    // A thread whose largest reaches the bound lists what it kept; where its second group reaches it too, the wavefront reads
    // all vectors of that thread, one a lane.
    const bool reaches = has && mine >= bound, all = reaches && order_bits(top.second) >= bound && p.vecs > Vec<T>::FLY * p.NT;
    if (reaches && !all) {
#pragma unroll
        for (int u = 0; u < Vec<T>::FLY; ++u) {
            const int v = thread + (top.group * Vec<T>::FLY + u) * p.NT;
            float x[Vec<T>::E];
            Vec<T>::widen(top.kept[u], x);
            if (v < p.vecs) list_values(p, v, x, least, lds.list, &lds.listed);
        }
    }
    const int lane = thread & 63;
    for (unsigned long long left = __ballot(all); left; left &= left - 1) {
        const int owner = thread - lane + __ffsll(left) - 1;
        for (int v = owner + lane * p.NT; v < p.vecs; v += 64 * p.NT) {
            float x[Vec<T>::E];
            p.load(v, x);
            list_values(p, v, x, least, lds.list, &lds.listed);
        }
    }
}

// place(r, key) for the top_k largest of `count` <= kListed keys, each by one thread: r keys are larger.  A thread counts for
// two keys at a time, so that what it reads of the list serves both (8192 rows of 100 bf16 classes, 32 of them: 25.1 -> 17.4 us).
template <typename Place>
__device__ __forceinline__ void place_top(const Key *list, int count, int top_k, int thread, int threads, Place place) {
    for (int i = thread; i < count; i += 2 * threads) {
        const bool two = i + threads < count;
        const Key k = list[i], l = list[two ? i + threads : i];
        int above_k = 0, above_l = 0;
        for (int j = 0; j < count; ++j) {
            const Key other = list[j];
            above_k += less(k, other) ? 1 : 0;
            above_l += less(l, other) ? 1 : 0;
        }
        if (above_k < top_k) place(above_k, k);
        if (two && above_l < top_k) place(above_l, l);
    }
}

// ---- the same one by one: ties beyond the list, NaN ----------------------------------------------------------------

template <typename T>
__device__ __forceinline__ Key best_below(const Part<T> &p, int v, Key below, Key best) {
    constexpr int E = Vec<T>::E;
    float x[E];
    p.load(v, x);
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int i = p.at(v) + e;
        const Key k{order_bits(x[e]), 0xffffffffu - (uint32_t)(p.first + i)};
        if (i >= 0 && i < p.length && less(k, below) && less(best, k)) best = k;
    }
    return best;
}

// list[0 .. top_k) = the largest keys of the vectors of one wavefront's threads in falling order, then {0, 0}.  Every
// lane of the wavefront is active.
template <typename T>
__device__ __forceinline__ void wave_top(const Part<T> &p, int thread, int top_k, Key *list) {
    const int lane = thread & 63;
    const Key above{0xffffffffu, 0xffffffffu};
    Key mine{0u, 0u};
    for (int v = thread; v < p.vecs; v += p.NT) mine = best_below(p, v, above, mine);
    for (int r = 0; r < top_k; ++r) {
        const Key most = wave_most(mine);
        if (lane == 0) list[r] = most;
        if (most.hi == 0u) {  // (uniform) nothing left
            if (lane > r && lane < top_k) list[lane] = Key{0u, 0u};
            return;
        }
        if (r + 1 == top_k) return;
        // the one thread that gave it looks for its next: the wavefront reads that thread's vectors
        const int winner = __ffsll((unsigned long long)__ballot(mine.hi == most.hi && mine.lo == most.lo)) - 1;
        Key next{0u, 0u};
        for (int v = (thread - lane) + winner + lane * p.NT; v < p.vecs; v += 64 * p.NT) next = best_below(p, v, most, next);
        next = wave_most(next);
        if (lane == winner) mine = next;
    }
}

// Merges `lists` <= 64 falling lists of top_k keys; `emit(r, key)` is called by lane 0 for the r-th largest.
template <typename Emit>
__device__ __forceinline__ void merge_lists(const Key *keys, int lists, int top_k, int lane, Emit emit) {
    int at = 0;
    Key mine = lane < lists ? keys[lane * top_k] : Key{0u, 0u};
    for (int r = 0; r < top_k; ++r) {
        const Key most = wave_most(mine);
        if (lane == 0) emit(r, most);
        if (mine.hi == most.hi && mine.lo == most.lo && most.hi != 0u) {
            ++at;
            mine = at < top_k ? keys[lane * top_k + at] : Key{0u, 0u};
        }
    }
}

// place(r, key) for the r-th largest class of the part, r < top_k ({0, 0} where the part has fewer).  nan: the part holds
// one.  All threads of the team call it, with the same nan.
template <typename T, int NW, typename Place>
__device__ __forceinline__ void team_top(const Part<T> &p, int thread, const Top<Vec<T>::FLY> &top, bool nan, int top_k, TeamLds<NW> &lds, Place place) {
    if (!nan) {
        list_top(p, thread, top, top_k, lds);
        team_barrier<NW>();
        const int count = lds.listed;
        if (count <= kListed) {
            for (int r = count + thread; r < top_k; r += NW * 64) place(r, Key{0u, 0u});
            place_top(lds.list, count, top_k, thread, NW * 64, place);
            return;
        }
        team_barrier<NW>();  // (every thread has read the count)
    }
    static_assert(NW * RVN_MAX_TOP_K <= kListed, "a list for every wavefront");
    wave_top(p, thread, top_k, lds.list + (thread >> 6) * top_k);
    team_barrier<NW>();
    if (thread < 64) merge_lists(lds.list, NW, top_k, thread, place);
}

// One lane writes a row's results.
struct Row {
    float m, log_s;
    bool nan, empty;
};
__device__ __forceinline__ Row row_of(Sums a) { return Row{a.m, logf(a.s), !(a.s >= 0.f), a.s == 0.f}; }

__device__ __forceinline__ float log_probability(const Row &r, float x) {
    return r.nan ? __uint_as_float(0x7fc00000u) : r.empty ? -INFINITY : (x - r.m) - r.log_s;
}

// A row's label and its logit, requested before the row is read: neither depends on it.
struct Given {
    int64_t label;
    float logit;
};
template <typename T>
__device__ __forceinline__ Given given_of(const T *row, int classes, int64_t at, const int64_t *labels) {
    Given g{RVN_NO_LABEL, 0.f};
    if (labels) g.label = labels[at];
    if (g.label >= 0 && g.label < classes) g.logit = Vec<T>::one(row, g.label);
    return g;
}

__device__ __forceinline__ void put_row(int classes, int64_t at, Sums a, const Given &given, const LogprobOut &out) {
    const Row r = row_of(a);
    if (out.logprob) {
        float v = __uint_as_float(0x7fc00000u);
        if (given.label == RVN_NO_LABEL) v = 0.f;
        else if (given.label >= 0 && given.label < classes) v = log_probability(r, given.logit);
        out.logprob[at] = v;
    }
    if (out.entropy) out.entropy[at] = r.empty ? 0.f : r.log_s - kLn2 * (a.t / a.s);
    if (out.lse) out.lse[at] = r.nan ? __uint_as_float(0x7fc00000u) : a.m + r.log_s;
}

__device__ __forceinline__ void put_top(const LogprobOut &out, int64_t at, int r, Key k, const Row &row) {
    out.top_ids[at * out.top_k + r] = (int64_t)(0xffffffffu - k.lo);
    if (out.top_logprob) out.top_logprob[at * out.top_k + r] = log_probability(row, value_of(k.hi));
}

// One wavefront per row, for short rows; four rows to a workgroup.  (8192 x 4095 fp32: 134 MB in 24.7 us, 5.4 TB/s, with 5 top classes
// 27.8; 8192 x 1000 bf16 8.8 and 13.8, where the search costs as much as the reads; 128 x 10 5.9.)
template <typename T, bool TOP>
__global__ __launch_bounds__(kThreads) void logprob_wave_k(const T *x, int64_t rows, int64_t ld, int classes, const int64_t *labels,
                                                           const LogprobOut out) {
    __shared__ TeamLds<1> lds[kThreads / 64];
    const int wave = (int)threadIdx.x >> 6, lane = (int)threadIdx.x & 63;
    const int64_t at = (int64_t)blockIdx.x * (kThreads / 64) + wave;
    if (at >= rows) return;
    const Part<T> p(x, at, rows, ld, classes, 0, classes, 64);
    const Given given = given_of(p.row, classes, at, labels);
    Top<Vec<T>::FLY> top;
    const Sums a = wave_join(stream<TOP>(p, lane, top));
    if (lane == 0) put_row(classes, at, a, given, out);
    if constexpr (TOP) {
        const Row row = row_of(a);
        team_top<T, 1>(p, lane, top, row.nan, out.top_k, lds[wave], [&](int i, Key k) { put_top(out, at, i, k, row); });
    }
}

// A workgroup of NW wavefronts per part of a row.  splits == 1: the whole row, results written here.  Otherwise the
// part's sums and list go to `sums` and `keys` ([row][split]) for logprob_join_k.  (4096 x 50021 with 8 top classes: bf16, 410 MB, 94 us
// in the median of a trace, 4.4 TB/s, 85 a call in a row of calls; fp32, 820 MB, 146 us, 5.6 TB/s.)
template <typename T, int NW, bool TOP>
__global__ __launch_bounds__(NW * 64) void logprob_block_k(const T *x, int64_t rows, int64_t ld, int classes, int splits, int share,
                                                           const int64_t *labels, const LogprobOut out, float4 *sums, Key *keys) {
    __shared__ TeamLds<NW> lds;
    __shared__ Sums parts[NW];
    const int thread = (int)threadIdx.x, wave = thread >> 6, lane = thread & 63;
    const int64_t at = splits == 1 ? (int64_t)blockIdx.x : (int64_t)(blockIdx.x / (unsigned)splits);
    const int split = splits == 1 ? 0 : (int)(blockIdx.x - (unsigned)at * (unsigned)splits);
    const int first = split * share;
    const Part<T> p(x, at, rows, ld, classes, first, min(share, classes - first), NW * 64);
    Given given{RVN_NO_LABEL, 0.f};
    if (splits == 1) given = given_of(p.row, classes, at, labels);
    Top<Vec<T>::FLY> top;
    const Sums mine = wave_join(stream<TOP>(p, thread, top));
    if (lane == 0) parts[wave] = mine;
    __syncthreads();
    Sums a = parts[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) a = join(a, parts[w]);
    const int64_t slot = at * splits + split;
    if (thread == 0) {
        if (splits == 1) put_row(classes, at, a, given, out);
        else sums[slot] = make_float4(a.m, a.s, a.t, 0.f);
    }
    if constexpr (TOP) {
        const Row r = row_of(a);
        team_top<T, NW>(p, thread, top, r.nan, out.top_k, lds, [&](int i, Key k) {
            if (splits == 1) put_top(out, at, i, k, r);
            else keys[slot * out.top_k + i] = k;
        });
    }
}

// Joins the parts (at most 64) of a row.  A part's last key bounds the row's top_k-th from below; what reaches the largest
// of these bounds is listed and placed as above.  (One row of 9 parts with 20 top classes: 5.3 us, a chain of latencies.)
template <typename T>
__global__ __launch_bounds__(kThreads) void logprob_join_k(const T *x, int64_t ld, int classes, int splits, const int64_t *labels,
                                                           const LogprobOut out, const float4 *sums, const Key *keys) {
    __shared__ Key list[kListed];
    __shared__ int listed;
    const int thread = (int)threadIdx.x, lane = thread & 63, top_k = out.top_k;
    const int64_t at = blockIdx.x;
    const Key *row_keys = keys + at * splits * top_k;
    const Given given = given_of(x + at * ld, classes, at, labels);
    Sums a{kLowest, 0.f, 0.f};
    Key last{0u, 0u};
    if (lane < splits) {
        const float4 v = sums[at * splits + lane];
        a = Sums{v.x, v.y, v.z};
        if (top_k > 0) last = row_keys[lane * top_k + top_k - 1];
    }
    a = wave_join(a);
    if (thread == 0) put_row(classes, at, a, given, out), listed = 0;
    if (top_k == 0) return;
    const Row r = row_of(a);
    const Key bound = wave_most(last);
    __syncthreads();
    for (int i = thread; i < splits * top_k; i += kThreads) {
        const Key k = row_keys[i];
        if (k.hi == 0u || less(k, bound)) continue;
        const int slot = atomicAdd(&listed, 1);
        if (slot < kListed) list[slot] = k;
    }
    __syncthreads();
    if (listed <= kListed) place_top(list, listed, top_k, thread, kThreads, [&](int i, Key k) { put_top(out, at, i, k, r); });
    else if (thread < 64) merge_lists(row_keys, splits, top_k, lane, [&](int i, Key k) { put_top(out, at, i, k, r); });
}

// ---- gradient ------------------------------------------------------------------------------------------------

// 2^tshift neighbouring threads share a row; blockIdx.x counts pieces of FLY vectors a thread, blockIdx.y groups of rows.
// (4096 x 50021 bf16: 820 MB in 139 us, 5.9 TB/s; fp32, 1.64 GB, 293 us, 5.6 TB/s; a library's copies of these take 152
// and 314 us.)
template <typename T, bool ENTROPY>
__global__ __launch_bounds__(kThreads) void logprob_bwd_k(const T *x, int64_t rows, int64_t ld, int classes, int tshift,
                                                          const int64_t *labels, const float *lse, const float *entropy,
                                                          const float *d_logprob, const float *d_entropy, float scale, T *out,
                                                          int64_t out_ld) {
    constexpr int E = Vec<T>::E;
    const int team = 1 << tshift, per_block = kThreads >> tshift;
    const int v0 = (int)blockIdx.x * team * Vec<T>::FLY + ((int)threadIdx.x & (team - 1));
    for (int64_t at = (int64_t)blockIdx.y * per_block + ((int)threadIdx.x >> tshift); at < rows; at += (int64_t)gridDim.y * per_block) {
        const T *row = x + at * ld;
        T *to = out + at * out_ld;
        const int skew = skew_of(to, classes), vecs = (classes + skew + E - 1) / E;
        const int64_t label = labels ? labels[at] : RVN_NO_LABEL;
        // a row of no weight is not read where that shows before its other scalars have come
        const bool idle = !ENTROPY && label == RVN_NO_LABEL;
        float g[Vec<T>::FLY][E];
#pragma unroll
        for (int u = 0; u < Vec<T>::FLY; ++u)
            load_vec(row, (v0 + u * team) * E - skew, idle ? 0 : classes, -reach(at, ld), classes + reach(rows - 1 - at, ld), g[u]);
        const float norm = lse[at];
        float given = 0.f, spread = 0.f, h = 0.f;
        if (label != RVN_NO_LABEL) given = label >= 0 && label < classes ? scale * (d_logprob ? d_logprob[at] : 1.f) : __uint_as_float(0x7fc00000u);
        if (ENTROPY) spread = scale * d_entropy[at], h = entropy[at];
        // a term whose weight is 0 is absent, whatever the row holds; so is every term of a row that has no class
        const bool none = (given == 0.f && spread == 0.f) || norm == -INFINITY;
#pragma unroll
        for (int u = 0; u < Vec<T>::FLY; ++u) {
            const int first = (v0 + u * team) * E - skew;
            if (none) {
#pragma unroll
                for (int e = 0; e < E; ++e) g[u][e] = 0.f;
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float logp = g[u][e] - norm, p = __builtin_amdgcn_exp2f(logp * kLog2e);
                    g[u][e] = -given * p;
                    if (ENTROPY) g[u][e] -= spread * (p * (fmaxf(logp, -200.f) + h));  // (p is 0 there)
                }
                if (label >= first && label < first + E) {
#pragma unroll
                    for (int e = 0; e < E; ++e) g[u][e] += label == first + e ? given : 0.f;
                }
            }
            if (first >= 0 && first + E <= classes) {
                *reinterpret_cast<u4 *>(to + first) = Vec<T>::narrow(g[u]);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (first + e >= 0 && first + e < classes) Vec<T>::put(to, first + e, g[u][e]);
            }
        }
    }
}

constexpr int kFewTop = 12;

struct Shape {
    bool wave;           // a wavefront a row
    int splits, share;   // else workgroups a row, and the classes of each
};

// Rows up to 8 KB go to one wavefront each, and up to 32 KB where they are so many that each SIMD has two: a wavefront needs
// no barrier, where a workgroup waits for its slowest at every join.  (5 top classes, by workgroups and by wavefronts: 8192 x 1000
// bf16 28.3 and 14.1 us, 32 x 2000 5.7 and 6.5; 8192 x 4200 bf16 35.1 and 24.1, fp32 37.3 and 28.7; 2048 x 15000 bf16 20.3 and
// 18.4; 3000 x 32003 bf16 47.4 both, without top classes 42.1 and 44.9.)  The more top classes, the more of a wavefront's 64
// threads have to read their vectors again, which a workgroup spreads over 256: 16 of 2048 x 15000 cost 21.9 and 22.4, 32 of them
// 24.2 and 31.8.
// Else a row goes to a workgroup, or to several, joined by a second launch, where the workgroups are few.  A second launch pays from
// 56 KB a row on (5 top classes of 8 bf16 rows: 25000 classes 8.5 us in one launch, 9.6 in two; 40000 9.7 and 9.1).  The parts are
// of 8 KB at least (1 x 40000 5.0 us, with 16 KB 5.3), with many top classes, of which each part lists so many, of 16 (1 x 65537 with
// 20: 13.1 us, with 8 KB 14.2), as from 64 rows on (100 x 50000, 5 top classes: 12.2, with 8 KB 13.1), from
// 192 on, where rows alone nearly fill the chip, of 64 (300 x 131072: 18.6 us, 25.8 unsplit; 256 x 50021 with 5 top classes: 15.0
// unsplit, 16.3 split).
Shape shape_of(int64_t rows, int classes, int size, int top_k) {
    const int64_t bytes = (int64_t)classes * size;
    if (bytes <= 8192 || (rows >= 2048 && bytes <= 32768 && top_k <= kFewTop)) return Shape{true, 1, classes};
    const int64_t part = rows < 64 && top_k <= kFewTop ? 8192 : rows < 192 ? 16384 : 65536;
    const int64_t most = bytes <= 57344 ? 1 : rows < 192 ? (bytes + part - 1) / part : bytes / part;
    const int64_t splits = std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(most, 64), 1200 / rows));
    if (splits == 1) return Shape{false, 1, classes};
    const int step = 16 / size;
    const int share = (int)(((classes + splits - 1) / splits + step - 1) / step * step);
    return Shape{false, (classes + share - 1) / share, share};
}

// A launch counts its threads in 32 bits: rows beyond these, at 256 threads each, take another.
constexpr int64_t kRowsAtOnce = 1 << 23;

template <typename T>
void forward(Ctx &cx, const Logits &x, const Shape &s, const int64_t *labels, const LogprobOut &out, void *scratch) {
    const T *p = static_cast<const T *>(x.p);
    const double bytes = (double)x.rows * ((double)x.classes * sizeof(T) + 20.0 + 12.0 * out.top_k);
    if (!cx.launch(K_LOGPROB, bytes, 5.0 * (double)x.rows * x.classes)) return;
    if (s.wave) {
        const int per = kThreads / 64;
        cx.run(out.top_k ? logprob_wave_k<T, true> : logprob_wave_k<T, false>, dim3((unsigned)((x.rows + per - 1) / per)), dim3(kThreads), 0, p,
               x.rows, x.ld, x.classes, labels, out);
        return;
    }
    float4 *sums = static_cast<float4 *>(scratch);
    Key *keys = reinterpret_cast<Key *>(sums + (s.splits > 1 ? x.rows * s.splits : 0));
    cx.run(out.top_k ? logprob_block_k<T, 4, true> : logprob_block_k<T, 4, false>, dim3((unsigned)(x.rows * s.splits)), dim3(256), 0, p, x.rows, x.ld,
           x.classes, s.splits, s.share, labels, out, sums, keys);
    if (s.splits == 1) return;
    if (!cx.launch(K_LOGPROB, 0.0)) return;
    cx.run(logprob_join_k<T>, dim3((unsigned)x.rows), dim3(kThreads), 0, p, x.ld, x.classes, s.splits, labels, out, sums, keys);
}

template <typename T>
void backward(Ctx &cx, const Logits &x, const int64_t *labels, const float *lse, const float *entropy, const float *d_logprob,
              const float *d_entropy, float scale, T *out, int64_t out_ld) {
    if (!cx.launch(K_LOGPROB, (double)x.rows * (2.0 * x.classes * sizeof(T) + 16.0), 8.0 * (double)x.rows * x.classes)) return;
    // vectors of a row that starts anywhere between two borders (see skew_of)
    const int border = (x.classes >= 64 * Vec<T>::E ? 128 : 16) / (int)sizeof(T), vecs = (x.classes + border - 1 + Vec<T>::E - 1) / Vec<T>::E;
    int tshift = 0;
    while (tshift < 8 && (Vec<T>::FLY << tshift) < vecs) ++tshift;
    // Fewer threads a row, down to a wavefront, where a last piece leaves over an eighth of the threads without a vector and
    // shorter pieces fewer (8192 x 4200: 33.4 us with pieces of 256 threads, 23.5 with 64 in bf16, 57.7 and 43.4 in fp32;
    // 8192 x 1000, where two pieces of 64 idle as much as one of 128: 10.3 and 12.1, 12.8 and 16.0).
    auto idle = [&](int shift) {
        const int piece = Vec<T>::FLY << shift, last = vecs % piece;
        return last ? piece - last : 0;
    };
    for (int shift = tshift - 1; shift >= 6 && 8 * idle(tshift) > vecs; --shift)
        if (idle(shift) < idle(tshift)) tshift = shift;
    const int64_t groups = (x.rows + (kThreads >> tshift) - 1) / (kThreads >> tshift);
    const dim3 grid((unsigned)((vecs + (Vec<T>::FLY << tshift) - 1) / (Vec<T>::FLY << tshift)), (unsigned)(groups < 65535 ? groups : 65535));
    cx.run(d_entropy ? logprob_bwd_k<T, true> : logprob_bwd_k<T, false>, grid, dim3(kThreads), 0, static_cast<const T *>(x.p), x.rows, x.ld, x.classes, tshift, labels, lse, entropy,
           d_logprob, d_entropy, scale, out, out_ld);
}

}  // namespace

size_t logprob_scratch_bytes(int64_t rows, int classes, int top_k) {
    size_t most = 0;  // of the two types' shapes
    for (int size = 2; size <= 4; size += 2) {
        for (int k : {top_k, std::min(top_k, kFewTop)}) {  // (enough for every smaller number of top classes, too)
            const Shape s = shape_of(rows, classes, size, k);
            const size_t need = s.splits > 1 ? (size_t)rows * s.splits * (sizeof(float4) + (size_t)k * sizeof(Key)) : 0;
            most = most > need ? most : need;
        }
    }
    return most;
}

void logprob_fwd(Ctx &cx, const Logits &x, const int64_t *labels, const LogprobOut &out, void *scratch) {
    const int size = x.bf16 ? 2 : 4;
    const Shape s = shape_of(x.rows, x.classes, size, out.top_k);
    for (int64_t at = 0; at < x.rows; at += kRowsAtOnce) {
        const int64_t k = at * out.top_k;
        const Logits part{static_cast<const char *>(x.p) + at * x.ld * size, x.bf16, std::min(x.rows - at, kRowsAtOnce), x.ld, x.classes};
        const LogprobOut to{out.logprob ? out.logprob + at : nullptr, out.entropy ? out.entropy + at : nullptr, out.lse ? out.lse + at : nullptr,
                            out.top_ids ? out.top_ids + k : nullptr, out.top_logprob ? out.top_logprob + k : nullptr, out.top_k};
        const int64_t *const given = labels ? labels + at : nullptr;
        if (x.bf16) forward<Bf16>(cx, part, s, given, to, scratch);
        else forward<float>(cx, part, s, given, to, scratch);
    }
}

void logprob_bwd(Ctx &cx, const Logits &x, const int64_t *labels, const float *lse, const float *entropy, const float *d_logprob,
                 const float *d_entropy, float scale, void *out, int64_t out_ld) {
    if (x.bf16) backward(cx, x, labels, lse, entropy, d_logprob, d_entropy, scale, static_cast<Bf16 *>(out), out_ld);
    else backward(cx, x, labels, lse, entropy, d_logprob, d_entropy, scale, static_cast<float *>(out), out_ld);
}

}  // namespace rvn
