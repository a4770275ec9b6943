// Routing from logits (pgmoe_route) and its gradient (pgmoe_route_backward).
//
// A token belongs to 16 lanes, four tokens to a wavefront; lane l of them holds the experts l * PER .. l * PER + PER - 1
// in registers (PER = experts / 16, rounded up to a power of two).  So a search for the largest value costs PER steps in
// every lane and four exchanges, for four tokens at once, and the lowest lane that holds it has the lowest index.
//
// Selection.  Every expert's value becomes an integer key that orders as the value does, with places below all values for
// an expert that is unavailable, outside the kept groups, or taken.  The last four bits of a key are the expert's place in its lane
// (15 the first), so that a lane's largest key names its expert, the first of equal ones.  What is compared are so 32-bit results
// without their last four bits; hence the chosen neighbours (and the two groups at the border) are looked at once more, and a token where two of them
// lie close by the measure at CLOSE is decided in 64 bits.  Values that are equal because logit and bias are equal are no such case: either
// way the lowest index wins.  16-bit logits without a bias have those bits to spare.
//
// What bounds it is not bytes but the chain of dependent instructions of the searches: 16384 tokens of 256 experts, 8 of them, sigmoid,
// bfloat16, take 7.6 us (1.2 TB/s), 12.4 with a bias and 16.5 with groups too; softmax of as many without and with a bias 10.4 and 18.4 (131
// registers, three wavefronts a SIMD where the sigmoid has four); softmax of 128 experts, 2 of them, 5.4 and 8.5; one token 3.1.
// The gradient of 16384 x 128 float32 with that of the scores 7.8 us (3.2 TB/s), of 8191 x 256 bfloat16 6.1.
#include <algorithm>
#include <climits>
#include <cmath>

#include "ffn_common.h"

namespace pgmoe {

struct RouteArgs {
    const void *logits;
    size_t stride;
    const float *bias;
    int T, E, k, n_groups, keep;
    int renorm;
    float scale;
    int32_t *idx;
    float *weight, *scores;
    int size, shift;  // experts of a group, lanes of one as a power of two
    int straddle;     // groups that are not whole lanes
    int capacity;
    int lds;       // bytes of a token
};

constexpr int ROUTE_LANES = 16;                                // of one token
constexpr int ROUTE_THREADS = 256, ROUTE_TOKENS = ROUTE_THREADS / ROUTE_LANES;
// Selection values closer than this, relative to what they are made of, are compared in 64 bits.  A score is off by some thirty half-steps of
// 2^-24 (exp, a sum of 16 + 4 terms and their exp, an inverse), 1.8e-6 of itself, and by a third of a half-step of the largest score for exp's
// argument: the two that are compared by 3.7e-6.  A key leaves out 2^-19 of the value, 1.9e-6, and the sum with the bias a half-step.
// With a bias the value may be far smaller than the score in it, so the measure is the larger of the value and the token's largest score,
// the same for all its experts: one further down with a larger score cannot pass by.  Two groups are compared by four scores, 8e-6 of the
// largest, and four values and two sums of half a step each, 2.4e-7 of the largest sum of magnitudes.  Without a bias nothing
// cancels, and a group's measure is its value.  No measure is below 2^-24.
constexpr float CLOSE = 6e-6f;

// Keys of values, which are not NaN: integers in the order of the values, -0 as 0.
template <typename V>
struct Keys;
template <>
struct Keys<float> {
    typedef int32_t T;
    __device__ static T of(float v) {
        const int32_t b = __float_as_int(v + 0.f);
        return b ^ ((b >> 31) & INT_MAX);
    }
    __device__ static float value(T k) { return __int_as_float(k ^ ((k >> 31) & INT_MAX)); }
    static constexpr T lowest = INT_MIN;
};
template <>
struct Keys<double> {
    typedef int64_t T;
    __device__ static T of(double v) {
        const int64_t b = __double_as_longlong(v + 0.0);
        return b ^ ((b >> 63) & LLONG_MAX);
    }
    static constexpr T lowest = LLONG_MIN;
};
// below every value, in rising order; the last two with the place in the lane added
constexpr int32_t KEY_TAKEN = INT_MIN, KEY_OUTSIDE = INT_MIN + 16, KEY_UNAVAILABLE = INT_MIN + 32, KEY_VALUES = INT_MIN + 48;

// Reductions over the 16 lanes of a token (a row of the wavefront): rotations by 8, 4, 2 and 1 inside the row, which the vector unit
// does on the way (a shuffle through LDS takes some hundred clocks, and a selection is a chain of them).
template <int CTRL>
__device__ inline int row_moved(int v) {
    return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, false);
}
template <int CTRL>
__device__ inline float row_moved(float v) {
    return __int_as_float(row_moved<CTRL>(__float_as_int(v)));
}
template <int CTRL>
__device__ inline int64_t row_moved(int64_t v) {
    return (int64_t)((uint64_t)(uint32_t)row_moved<CTRL>((int)v) | (uint64_t)(uint32_t)row_moved<CTRL>((int)(v >> 32)) << 32);
}
template <int CTRL>
__device__ inline double row_moved(double v) {
    return __longlong_as_double(row_moved<CTRL>((int64_t)__double_as_longlong(v)));
}
template <typename V, typename F>
__device__ inline V lanes_reduce(V v, F f) {
    v = f(v, row_moved<0x128>(v));  // row_ror:8
    v = f(v, row_moved<0x124>(v));
    v = f(v, row_moved<0x122>(v));
    return f(v, row_moved<0x121>(v));
}
template <typename V>
__device__ inline V lanes_sum(V v) {
    return lanes_reduce(v, [](V a, V b) { return a + b; });
}
template <typename V>
__device__ inline V lanes_max(V v) {
    return lanes_reduce(v, [](V a, V b) { return b > a ? b : a; });
}
template <typename V>
__device__ inline V lanes_min(V v) {
    return lanes_reduce(v, [](V a, V b) { return b < a ? b : a; });
}

// What the lanes of a wavefront wrote to LDS is there for its other lanes behind this (they run in lockstep and LDS
// operations complete in order: nothing but the compiler has to be held back).
__device__ inline void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

__device__ inline bool available(float z) { return z > -INFINITY; }  // false for NaN too

// exp(x): 2^t with the rest of the product by log2 e put back, three half-steps of 2^-24 from exact. Results below 2^-126 may be 0.
// Nothing is put back where 2^t is infinite (from t = 128 on: infinity less a rest of it is NaN) or below 2^-128.
__device__ inline float exp_of(float x) {
    const float t = x * 1.44269502f, rest = fmaf(x, 1.92596303e-8f, fmaf(x, 1.44269502f, -t));
    const float e = __builtin_amdgcn_exp2f(t);
    return fabsf(t) < 128.f ? fmaf(e, rest * 0.693147182f, e) : e;
}
__device__ inline float inverse_of(float x) { return __builtin_amdgcn_rcpf(x); }  // one step of 2^-24
__device__ inline double exp_of(double x) { return exp(x); }
__device__ inline double inverse_of(double x) { return 1.0 / x; }
// exp(z - m), 1 at the largest of infinite logits and 0 for an unavailable one.  (Values first, choices afterwards: no branches.)
template <typename V>
__device__ inline V exp_below(float z, float m) {
    const V e = exp_of(V(z) - V(m));
    const V one_at_m = z == m ? V(1) : e;
    return available(z) ? one_at_m : V(0);
}
// 0 for an unavailable logit, which is -infinity here
template <typename V>
__device__ inline V sigmoid(float z) {
    return inverse_of(V(1) + exp_of(-V(z)));
}

template <typename L>
__device__ inline float logit_at(const RouteArgs &a, size_t t, int e) {
    const float z = (float)reinterpret_cast<const L *>(a.logits)[t * a.stride + e];
    return available(z) ? z : -INFINITY;
}

// This lane's logits of token t; unavailable (-infinity) past the last expert.  VEC: all PER exist, at an address that their bytes (or 16) divide.
template <bool VEC, typename L, int PER>
__device__ inline void load_logits(const L *row, int E, int first, float (&z)[PER]) {
    if (VEC) {
        constexpr int N = PER * sizeof(L) > 16 ? 16 / sizeof(L) : PER;
        typedef L Lx __attribute__((ext_vector_type(N)));
#pragma unroll
        for (int i = 0; i < PER; i += N) {
            const Lx v = *reinterpret_cast<const Lx *>(row + (first < E ? first : 0) + i);
#pragma unroll
            for (int j = 0; j < N; ++j) z[i + j] = (float)v[j];
        }
    } else {
#pragma unroll
        for (int i = 0; i < PER; ++i) z[i] = (float)row[min(first + i, E - 1)];
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) z[i] = first + i < E && available(z[i]) ? z[i] : -INFINITY;
}

template <bool VEC, int PER>
__device__ inline void load_floats(const float *row, int E, int first, float (&v)[PER]) {
    if (VEC && PER % 4 == 0) {
#pragma unroll
        for (int i = 0; i < PER; i += 4) {
            const floatx4 x = *reinterpret_cast<const floatx4 *>(row + (first < E ? first : 0) + i);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i + j] = x[j];
        }
    } else {
#pragma unroll
        for (int i = 0; i < PER; ++i) v[i] = row[min(first + i, E - 1)];
    }
}

// This lane's results into a row.
template <bool VEC, typename L, int PER>
__device__ inline void store_row(L *row, int E, int first, const float (&v)[PER]) {
    constexpr int N = PER * sizeof(L) > 16 ? 16 / sizeof(L) : PER;
    typedef L Lx __attribute__((ext_vector_type(N)));
    if (VEC) {
        if (first < E) {
#pragma unroll
            for (int i = 0; i < PER; i += N) {
                Lx x;
#pragma unroll
                for (int j = 0; j < N; ++j) x[j] = (L)v[i + j];
                *reinterpret_cast<Lx *>(row + first + i) = x;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (first + i < E) row[first + i] = (L)v[i];
    }
}

// Scores of this lane's experts from its logits; m: the token's largest logit.  Returns the token's largest score.
template <bool SIGMOID, int PER>
__device__ inline float scores_of(const float (&z)[PER], float m, float (&s)[PER]) {
    if (SIGMOID) {
#pragma unroll
        for (int i = 0; i < PER; ++i) s[i] = sigmoid<float>(z[i]);
        return sigmoid<float>(m);
    } else {
        float sum = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            s[i] = exp_below<float>(z[i], m);
            sum += s[i];
        }
        sum = lanes_sum(sum);
        const float inv = sum > 0.f ? inverse_of(sum) : 0.f;
#pragma unroll
        for (int i = 0; i < PER; ++i) s[i] *= inv;
        return inv;  // the largest term is 1
    }
}

// A token's places in LDS: what a selection leaves (experts and their keys, and, where 32 bits do not decide, 64-bit values), and
// the experts' values where groups straddle lanes.
struct RoutePlaces {
    int32_t *chosen, *keys;  // [capacity]
    double *exact;           // [capacity]
    float *values;           // [n_experts]
    int capacity;
};
constexpr int ROUTE_MORE = 32;  // candidates beyond the k that are looked at before all experts are

// The two largest of what it is shown.
template <typename V>
struct TwoLargest {
    V one = -(V)INFINITY, two = -(V)INFINITY;
    __device__ void take(V x) {
        const V low_one = x > one ? one : x;
        one = x > one ? x : one;
        two = low_one > two ? low_one : two;
    }
    template <int CTRL>
    __device__ void join() {  // with another lane's
        const V o = row_moved<CTRL>(one), t = row_moved<CTRL>(two);
        take(o);
        take(t);
    }
};

// Which groups are kept, as a bit for each in the first of its `part` lanes, from what each of these has seen of the group.  part = 2^shift.  Returns
// whether 32 bits may not have decided it (V = float only; most: the token's largest score).
template <typename V>
__device__ bool keep_groups(const RouteArgs &a, TwoLargest<V> best, int lane, int shift, float most, unsigned *mask) {
    typedef typename Keys<V>::T Key;
    constexpr Key low = Keys<V>::lowest;
    const int mine = lane >> shift;
    if (shift > 0) best.template join<0xB1>();   // quad_perm 1 0 3 2
    if (shift > 1) best.template join<0x4E>();   // quad_perm 2 3 0 1
    if (shift > 2) best.template join<0x141>();  // row_half_mirror: quads are of one mind
    if (shift > 3) best.template join<0x140>();  // row_mirror
    Key worth = low;
    V value = -(V)INFINITY;
    if (mine < a.n_groups) {
        value = best.two > -(V)INFINITY ? best.one + best.two : best.one;
        worth = value > -(V)INFINITY ? Keys<V>::of(value) : low;
    }
    // kept: fewer than `keep` groups are worthier, or as worthy and lower.  All lanes of a group say the same, so each group counts `part` times.
    int above = 0;
    static_for<ROUTE_LANES - 1>([&](auto r_) {
        constexpr int R = decltype(r_)::value + 1;
        const Key o = row_moved<0x120 + R>(worth);
        const int theirs = ((lane - R) & (ROUTE_LANES - 1)) >> shift;  // row_ror:R brings what is R lanes below
        above += theirs < a.n_groups && (o > worth || (o == worth && theirs < mine)) ? 1 : 0;
    });
    const bool kept = mine < a.n_groups && above < a.keep << shift;
    *mask = (unsigned)(__ballot(kept) >> (threadIdx.x & 48)) & 0xffffu;
    if (sizeof(V) == 8 || a.keep == a.n_groups) return false;
    // the worst kept against the best other
    const float inside = -lanes_max(kept ? -(float)value : -INFINITY);
    const float outside = lanes_max(mine < a.n_groups && !kept && worth > low ? (float)value : -INFINITY);
    float terms = fabsf(inside);
    if (a.bias) {
        const float one = fabsf((float)best.one), two = fabsf((float)best.two);
        terms = 4.f / 3 * most + 0.04f * lanes_max(worth > low ? (best.two > -(V)INFINITY ? one + two : one) : 0.f);
    }
    return outside > -INFINITY && !(inside - outside > CLOSE * fmaxf(terms, 6e-8f));
}

// Takes the expert of the largest key: the lowest of those that have it.
template <int PER>
__device__ inline int take_largest(int32_t (&key)[PER], int first, int32_t *top) {
    int32_t best = key[0];
#pragma unroll
    for (int i = 1; i < PER; ++i) best = key[i] > best ? key[i] : best;
    *top = lanes_max(best & ~15);
    const int candidate = (best & ~15) == *top ? first + 15 - (best & 15) : INT_MAX, won = lanes_min(candidate);
    const int32_t mine = candidate == won ? best : KEY_TAKEN;
#pragma unroll
    for (int i = 0; i < PER; ++i) key[i] = key[i] == mine ? KEY_TAKEN : key[i];
    return won;
}

// Selects the k experts of one token; returns where they are: at.chosen or at.keys.  logit(e): a logit of this token.  FULL: logits have 32 bits.
template <bool SIGMOID, bool FULL, int PER, typename F>
__device__ const int32_t *select_experts(const RouteArgs &a, const float (&z)[PER], const float (&b)[PER], int first, int lane, float m, const RoutePlaces &at, F logit) {
    int32_t key[PER];
    unsigned gone = 0;  // of this lane's experts: outside the kept groups, later also taken
    // In 64 bits, one expert at a time: there are few such tokens, and what they run is short code rather than fast.
    double sum = 0.0;
    auto exact_sum = [&]() {
        if (SIGMOID || sum > 0.0) return;
#pragma unroll 1
        for (int e = lane; e < a.E; e += ROUTE_LANES) sum += exp_below<double>(logit(e), m);
        sum = lanes_sum(sum);
    };
    auto exact_value = [&](int e) {
        const float ze = logit(e), be = a.bias ? a.bias[e] : 0.f;
        const double v = (SIGMOID ? sigmoid<double>(ze) : exp_below<double>(ze, m) / sum) + (double)be;
        return available(ze) && be > -INFINITY ? v : -(double)INFINITY;
    };
    float most = 0.f;  // the largest score and at least 2^-24, where scores are compared
    {
        float v[PER];
        if (a.bias || a.n_groups > 1) {
            most = fmaxf(scores_of<SIGMOID, PER>(z, m, v), 6e-8f);
#pragma unroll
            for (int i = 0; i < PER; ++i) v[i] += b[i];
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            // without a bias by the logit: scores rise with it, and it is exact
            const int32_t of = Keys<float>::of(a.bias ? v[i] : z[i]) & ~15, there = available(z[i]) ? of : KEY_UNAVAILABLE;
            key[i] = first + i >= a.E ? KEY_TAKEN : there | (15 - i);
        }
        if (a.n_groups > 1) {
            // 2^shift lanes a group, as many as there are, look for the two largest of a part of it each
            const int shift = a.shift, size = a.size, mine = lane >> shift, in_part = lane - (mine << shift);
            const int from = size * in_part >> shift, to = mine < a.n_groups ? size * (in_part + 1) >> shift : from;
            TwoLargest<float> best;
            if (!a.straddle) {  // these are the lane's own
#pragma unroll
                for (int i = 0; i < PER; ++i) best.take(available(z[i]) ? v[i] : -INFINITY);
            } else {
#pragma unroll
                for (int i = 0; i < PER; ++i)
                    if (first + i < a.E) at.values[first + i] = available(z[i]) ? v[i] : -INFINITY;
                wave_sync();
                for (int j = from; j < to; ++j) best.take(at.values[mine * size + j]);
            }
            unsigned mask;
            if (keep_groups(a, best, lane, shift, most, &mask)) {
                exact_sum();
                TwoLargest<double> exact;
#pragma unroll 1
                for (int j = from; j < to; ++j) exact.take(exact_value(mine * size + j));
                keep_groups(a, exact, lane, shift, most, &mask);
            }
            if (!a.straddle) {
                const bool out = !((mask >> (mine << shift)) & 1) && mine < a.n_groups;
                gone = out ? ~0u : 0u;
#pragma unroll
                for (int i = 0; i < PER; ++i) key[i] = out ? KEY_OUTSIDE | (15 - i) : key[i];
            } else {
                int g = first / size, in_group = first - g * size;
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    const bool out = !((mask >> (g << shift)) & 1);
                    gone |= out ? 1u << i : 0u;
                    key[i] = out && first + i < a.E ? KEY_OUTSIDE | (15 - i) : key[i];
                    const bool next = ++in_group == size;
                    in_group = next ? 0 : in_group;
                    g += next ? 1 : 0;
                }
            }
        }
    }
    // where keys do not decide, one further than asked for: to compare the last chosen with the first that is not
    const bool look = a.bias || FULL;
    int n = look ? min(a.k + 1, a.E) : a.k;
    int32_t top = 0;
    for (int j = 0; j < n; ++j) {
        const int won = take_largest(key, first, &top);
        if (lane == 0) {
            at.chosen[j] = won;
            if (look) at.keys[j] = top;
        }
    }
    if (!look) return at.chosen;
    wave_sync();
    auto near = [&](int32_t upper, int32_t lower) {  // might the order be another in 64 bits?
        const float hi = Keys<float>::value(upper), lo = Keys<float>::value(lower);
        const bool unsure = a.bias ? lo > -INFINITY && !(hi - lo > CLOSE * fmaxf(fabsf(hi), most)) : upper == lower;
        return lower >= KEY_VALUES && unsure;
    };
    bool close = false;
    for (int j = lane; j + 1 < n; j += ROUTE_LANES)
        if (near(at.keys[j], at.keys[j + 1])) {
            const int e = at.chosen[j], f = at.chosen[j + 1];
            // (behind the last chosen there may be more: beside an equal one also a larger one)
            close |= j + 1 == a.k || logit(e) != logit(f) || (a.bias && !(a.bias[e] == a.bias[f]));
        }
    if (!lanes_max(close ? 1 : 0)) return at.chosen;

    // all that may belong to the k: as many more as lie close to each other
    int32_t last = at.keys[n - 1], before = n > 1 ? at.keys[n - 2] : last;
    bool all = false;
    while (n > a.k && n < a.E && near(before, last)) {
        if (n == at.capacity) {
            all = true;
            break;
        }
        before = last;
        const int won = take_largest(key, first, &last);
        if (lane == 0) at.chosen[n] = won;
        ++n;
    }
    // The first that lies apart is none of them.  (It may be of a group that is not kept, whatever its value.)
    if (n > a.k && !near(before, last)) --n;
    wave_sync();
    if (a.bias) exact_sum();
    auto rank_value = [&](int e) { return a.bias ? exact_value(e) : (double)logit(e); };
    if (all) {  // too many: all experts again, in 64 bits
        for (int j = 0; j < a.k; ++j) {
            int64_t top = LLONG_MIN;
            int won = INT_MAX;
#pragma unroll 1
            for (int i = 0; i < PER; ++i) {
                const int e = first + i;
                if (e >= a.E || (gone >> i) & 1) continue;
                const int64_t k = available(logit(e)) ? Keys<double>::of(rank_value(e)) : Keys<double>::lowest + 1;
                won = k > top ? e : won;
                top = k > top ? k : top;
            }
            const int64_t best = lanes_max(top);
            won = lanes_min(top == best ? won : INT_MAX);
            if (won >= first && won < first + PER) gone |= 1u << (won - first);
            if (lane == 0) at.chosen[j] = won;
        }
        return at.chosen;
    }
    for (int j = lane; j < n; j += ROUTE_LANES) at.exact[j] = rank_value(at.chosen[j]);
    wave_sync();
    for (int j = lane; j < n; j += ROUTE_LANES) {
        const double x = at.exact[j];
        const int e = at.chosen[j];
        int rank = 0;
        for (int i = 0; i < n; ++i) {
            const double y = at.exact[i];
            // equal ones by index; of those at -infinity the order found holds
            rank += y > x || (y == x && (x > -(double)INFINITY ? at.chosen[i] < e : i < j)) ? 1 : 0;
        }
        at.keys[rank] = e;  // (the keys have been read)
    }
    wave_sync();
    return at.keys;
}

template <typename L, bool SIGMOID, int PER, bool VEC>
__global__ __launch_bounds__(ROUTE_THREADS) void route_logits_kernel(const RouteArgs a) {
    extern __shared__ char lds[];
    const int lane = threadIdx.x & (ROUTE_LANES - 1), token = threadIdx.x / ROUTE_LANES;
    const size_t t = (size_t)blockIdx.x * (blockDim.x / ROUTE_LANES) + token;
    if (t >= (size_t)a.T) return;  // whole rows of 16 lanes; no workgroup barrier below
    const bool look = a.bias || sizeof(L) == 4;
    // per token: where keys do not decide `capacity` experts, keys and values, without k experts; n_experts values where groups straddle lanes
    RoutePlaces at;
    at.exact = reinterpret_cast<double *>(lds + (size_t)token * a.lds);
    at.chosen = reinterpret_cast<int32_t *>(at.exact + (look ? a.capacity : 0));
    at.keys = at.chosen + (look ? a.capacity : a.k);
    at.values = reinterpret_cast<float *>(at.keys + (look ? a.capacity : 0));
    at.capacity = a.capacity;
    const int first = lane * PER;
    float z[PER], b[PER];
    if (a.bias) load_floats<VEC>(a.bias, a.E, first, b);
    load_logits<VEC>(reinterpret_cast<const L *>(a.logits) + t * a.stride, a.E, first, z);
#pragma unroll
    for (int i = 0; i < PER; ++i) b[i] = !a.bias ? 0.f : b[i] == b[i] ? b[i] : -INFINITY;
    float m = z[0];
#pragma unroll
    for (int i = 1; i < PER; ++i) m = fmaxf(m, z[i]);
    m = lanes_max(m);

    const int32_t *chosen = select_experts<SIGMOID, sizeof(L) == 4>(a, z, b, first, lane, m, at, [&](int e) { return logit_at<L>(a, t, e); });
    wave_sync();

    float s[PER], sum = 0.f;  // scores, softmax before the division; of exp(z - m) over all experts
    if (a.scores || (!SIGMOID && !a.renorm)) {
        if (!SIGMOID) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                s[i] = exp_below<float>(z[i], m);
                sum += s[i];
            }
            sum = lanes_sum(sum);
        } else {
#pragma unroll
            for (int i = 0; i < PER; ++i) s[i] = sigmoid<float>(z[i]);
        }
    }
    // Weights, lane j the j-th (and 16 + j-th ..).  Renormalised ones are taken relative to the largest selected logit, so that neither
    // sum nor quotient underflows where all of them are small: sigmoid(z) = exp(min(z, 0)) / (1 + exp(-|z|)).
    auto chosen_logit = [&](int j) { return j < a.k ? logit_at<L>(a, t, chosen[j]) : -INFINITY; };
    const float z0 = chosen_logit(lane);
    float top = SIGMOID ? fminf(z0, 0.f) : z0, total = 0.f;
    auto part = [&](float zj) {
        if (SIGMOID) return exp_below<float>(fminf(zj, 0.f), top) * inverse_of(1.f + exp_of(-fabsf(zj)));
        return exp_below<float>(zj, top);
    };
    if (a.renorm) {
        for (int j = lane + ROUTE_LANES; j < a.k; j += ROUTE_LANES) top = fmaxf(top, SIGMOID ? fminf(chosen_logit(j), 0.f) : chosen_logit(j));
        top = lanes_max(top);
        total = part(z0);
        for (int j = lane + ROUTE_LANES; j < a.k; j += ROUTE_LANES) total += part(chosen_logit(j));
        total = lanes_sum(total);
    }
    for (int j = lane; j < a.k; j += ROUTE_LANES) {
        const float zj = j == lane ? z0 : chosen_logit(j);
        const float w = a.renorm ? part(zj) / total : SIGMOID ? sigmoid<float>(zj) : exp_below<float>(zj, m) / sum;
        a.idx[t * a.k + j] = chosen[j];
        a.weight[t * a.k + j] = available(zj) ? a.scale * w : 0.f;
    }
    if (a.scores) {  // last: they may take the logits' place
        if (!SIGMOID) {
            const float inv = sum > 0.f ? 1.f / sum : 0.f;
#pragma unroll
            for (int i = 0; i < PER; ++i) s[i] *= inv;
        }
        store_row<VEC>(a.scores + t * a.E, a.E, first, s);
    }
}

struct RouteBackwardArgs {
    const void *logits;
    size_t stride;
    const int32_t *idx;
    const float *d_weight, *d_scores;
    void *d_logits;
    size_t d_stride;
    int T, E, k, renorm;
    float scale;
};

// The selected experts' part of the gradient goes through LDS, one float an expert: what lane j works out for the j-th
// belongs to the lane that holds that expert.  Renormalised, with r_j = s_j / total,
//   s_j d_s[j] = c r_j (d_w[j] - sum_i d_w[i] r_i),
// whose sum over j is 0: softmax's common term has nothing of it, and r is taken as in the forward kernel.
template <typename L, bool SIGMOID, int PER, bool VEC>
__global__ __launch_bounds__(ROUTE_THREADS) void route_logits_backward_kernel(const RouteBackwardArgs a) {
    extern __shared__ float parts[];
    const int lane = threadIdx.x & (ROUTE_LANES - 1), token = threadIdx.x / ROUTE_LANES;
    const size_t t = (size_t)blockIdx.x * ROUTE_TOKENS + token;
    if (t >= (size_t)a.T) return;  // whole rows of 16 lanes; no workgroup barrier below
    float *part = parts + token * ROUTE_LANES * PER;
    const int first = lane * PER;
    const L *row = reinterpret_cast<const L *>(a.logits) + t * a.stride;
    const bool every = a.d_scores || (!SIGMOID && !a.renorm);  // the gradient of every expert needs its score
    float z[PER], s[PER], m = -INFINITY, sum = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        part[first + i] = 0.f;
        s[i] = 0.f;
    }
    if (every) {
        load_logits<VEC>(row, a.E, first, z);
        if (!SIGMOID) {
#pragma unroll
            for (int i = 0; i < PER; ++i) m = fmaxf(m, z[i]);
            m = lanes_max(m);
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            s[i] = SIGMOID ? sigmoid<float>(z[i]) : exp_below<float>(z[i], m);
            sum += s[i];
        }
        if (!SIGMOID) {
            sum = lanes_sum(sum);
            const float inv = sum > 0.f ? 1.f / sum : 0.f;
#pragma unroll
            for (int i = 0; i < PER; ++i) s[i] *= inv;
        }
    }
    // the selected ones: lane j the j-th
    float top = -INFINITY, total = 0.f, dot = 0.f;
    auto logit_of = [&](int j, int &e) {
        e = a.idx[t * a.k + j];
        const float zj = e >= 0 && e < a.E ? (float)row[e] : -INFINITY;
        return available(zj) ? zj : -INFINITY;
    };
    auto ratio = [&](float zj) {  // s_j, up to a factor common to the token's
        if (SIGMOID) return exp_below<float>(fminf(zj, 0.f), top) * inverse_of(1.f + exp_of(-fabsf(zj)));
        return exp_below<float>(zj, top);
    };
    int e;
    if (a.renorm) {
        for (int j = lane; j < a.k; j += ROUTE_LANES) {
            const float zj = logit_of(j, e);
            top = fmaxf(top, SIGMOID ? fminf(zj, 0.f) : zj);
        }
        top = lanes_max(top);
        for (int j = lane; j < a.k; j += ROUTE_LANES) {
            const float r = ratio(logit_of(j, e));
            total += r;
            dot += r == 0.f ? 0.f : r * a.d_weight[t * a.k + j];
        }
        total = lanes_sum(total);
        dot = lanes_sum(dot) / total;
    }
    float common = 0.f;  // softmax: sum of s d_s
    wave_sync();
    for (int j = lane; j < a.k; j += ROUTE_LANES) {
        const float zj = logit_of(j, e);
        if (!available(zj)) continue;
        const float g = a.d_weight[t * a.k + j];
        float d;  // s_j times the part of d_s[j] that comes through the weights
        if (a.renorm) d = ratio(zj) / total * (g - dot);
        else d = (SIGMOID ? sigmoid<float>(zj) : exp_below<float>(zj, m) / sum) * g;
        d *= a.scale;
        if (SIGMOID) d *= sigmoid<float>(-zj);
        else if (!a.renorm) common += d;
        atomicAdd(&part[e], d);
    }
    float ds[PER];
    if (a.d_scores) load_floats<VEC>(a.d_scores + t * a.E, a.E, first, ds);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        ds[i] = a.d_scores && s[i] > 0.f ? ds[i] : 0.f;
        if (!SIGMOID) common += s[i] * ds[i];
    }
    if (!SIGMOID && every) common = lanes_sum(common);
    wave_sync();
    float d[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        d[i] = part[first + i];
        const float more = SIGMOID ? s[i] * sigmoid<float>(-z[i]) * ds[i] : s[i] * (ds[i] - common);
        d[i] = every && s[i] > 0.f ? d[i] + more : d[i];
    }
    store_row<VEC>(reinterpret_cast<L *>(a.d_logits) + t * a.d_stride, a.E, first, d);
}

static int check_router(const pgmoe_router *r, const char *fn) {
    if (!r) return fail(nullptr, PGMOE_EINVAL, "%s: router is NULL", fn);
    if (r->n_experts < 1 || r->n_experts > PGMOE_MAX_EXPERTS)
        return fail(nullptr, PGMOE_EINVAL, "%s: n_experts=%d outside 1..%d", fn, r->n_experts, PGMOE_MAX_EXPERTS);
    const int groups = r->n_groups ? r->n_groups : 1, keep = r->topk_groups ? r->topk_groups : groups;
    if (groups < 1 || groups > PGMOE_MAX_GROUPS || r->n_experts % groups)
        return fail(nullptr, PGMOE_EINVAL, "%s: n_groups=%d is no divisor of n_experts=%d in 1..%d", fn, groups, r->n_experts, PGMOE_MAX_GROUPS);
    if (keep < 1 || keep > groups) return fail(nullptr, PGMOE_EINVAL, "%s: topk_groups=%d outside 1..n_groups=%d", fn, keep, groups);
    if (r->top_k < 1 || r->top_k > r->n_experts / groups * keep)
        return fail(nullptr, PGMOE_EINVAL, "%s: top_k=%d outside 1..%d, the experts of the kept groups", fn, r->top_k, r->n_experts / groups * keep);
    if (r->score != PGMOE_SCORE_SOFTMAX && r->score != PGMOE_SCORE_SIGMOID) return fail(nullptr, PGMOE_EINVAL, "%s: score=%d unknown", fn, r->score);
    if (r->renormalize != 0 && r->renormalize != 1) return fail(nullptr, PGMOE_EINVAL, "%s: renormalize=%d is neither 0 nor 1", fn, r->renormalize);
    if (!std::isfinite(r->scale)) return fail(nullptr, PGMOE_EINVAL, "%s: scale is not finite", fn);
    if (r->logits_dtype != PGMOE_F32 && r->logits_dtype != PGMOE_BF16 && r->logits_dtype != PGMOE_F16)
        return fail(nullptr, PGMOE_EINVAL, "%s: logits_dtype=%d is neither f32 nor bf16 nor f16", fn, r->logits_dtype);
    return PGMOE_OK;
}

constexpr int ROUTE_TOKENS_MAX = (1 << 28) - ROUTE_TOKENS;  // whole workgroups of 16 lanes a token
static_assert((int64_t)ROUTE_TOKENS_MAX * ROUTE_LANES <= GRID_THREADS_MAX && ROUTE_TOKENS_MAX % ROUTE_TOKENS == 0, "one launch");
static int check_tokens(int T, const char *fn) {
    if (T < 0) return fail(nullptr, PGMOE_EINVAL, "%s: T=%d is negative", fn, T);
    if (T > ROUTE_TOKENS_MAX) return fail(nullptr, PGMOE_EINVAL, "%s: T=%d tokens are more than one launch holds, %d", fn, T, ROUTE_TOKENS_MAX);
    return PGMOE_OK;
}

// Experts a lane holds.
static int route_per(int E) {
    int per = 1;
    while (per * ROUTE_LANES < E) per *= 2;
    return per;
}
// Do all lanes that hold experts hold PER of them, at addresses of whole loads?
static bool route_vec(const pgmoe_router *r, const void *rows, int64_t stride) {
    const int per = route_per(r->n_experts);
    const size_t bytes = std::min<size_t>(16, per * dtype_bytes(r->logits_dtype));
    return r->n_experts % per == 0 && aligned(rows, bytes) && stride * dtype_bytes(r->logits_dtype) % bytes == 0;
}

// Do two matrices of n rows of `bytes` bytes, at rows so many bytes apart, share any?  Rows as far apart as the others' may lie between them.
static bool rows_overlap(const void *a, int64_t a_apart, const void *b, int64_t b_apart, int64_t bytes, int64_t n) {
    const int64_t d = (const char *)b - (const char *)a;
    if (d >= (n - 1) * a_apart + bytes || -d >= (n - 1) * b_apart + bytes) return false;
    if (a_apart != b_apart) return true;
    const int64_t phase = (d % a_apart + a_apart) % a_apart;
    return phase < bytes || a_apart - phase < bytes;
}

// The instantiation for a type of logits, a score, a number of experts and the form of the loads: KERNEL<L, SIGMOID, PER, VEC>.
#define ROUTE_LAUNCH_PER(KERNEL, L, SIG, PER, vec, ...)                                      \
    do {                                                                                     \
        if (vec) hipLaunchKernelGGL((KERNEL<L, SIG, PER, true>), __VA_ARGS__);               \
        else hipLaunchKernelGGL((KERNEL<L, SIG, PER, false>), __VA_ARGS__);                  \
    } while (0)
#define ROUTE_LAUNCH_E(KERNEL, L, SIG, E, ...)                                               \
    do {                                                                                     \
        switch (route_per(E)) {                                                              \
        case 1: ROUTE_LAUNCH_PER(KERNEL, L, SIG, 1, __VA_ARGS__); break;                     \
        case 2: ROUTE_LAUNCH_PER(KERNEL, L, SIG, 2, __VA_ARGS__); break;                     \
        case 4: ROUTE_LAUNCH_PER(KERNEL, L, SIG, 4, __VA_ARGS__); break;                     \
        case 8: ROUTE_LAUNCH_PER(KERNEL, L, SIG, 8, __VA_ARGS__); break;                     \
        default: ROUTE_LAUNCH_PER(KERNEL, L, SIG, 16, __VA_ARGS__);                          \
        }                                                                                    \
    } while (0)
#define ROUTE_LAUNCH(KERNEL, r, ...)                                                                     \
    do {                                                                                                 \
        const bool sig_ = (r)->score == PGMOE_SCORE_SIGMOID;                                             \
        if ((r)->logits_dtype == PGMOE_F32) {                                                            \
            if (sig_) ROUTE_LAUNCH_E(KERNEL, float, true, (r)->n_experts, __VA_ARGS__);                  \
            else ROUTE_LAUNCH_E(KERNEL, float, false, (r)->n_experts, __VA_ARGS__);                      \
        } else if ((r)->logits_dtype == PGMOE_BF16) {                                                    \
            if (sig_) ROUTE_LAUNCH_E(KERNEL, __bf16, true, (r)->n_experts, __VA_ARGS__);                 \
            else ROUTE_LAUNCH_E(KERNEL, __bf16, false, (r)->n_experts, __VA_ARGS__);                     \
        } else {                                                                                         \
            if (sig_) ROUTE_LAUNCH_E(KERNEL, _Float16, true, (r)->n_experts, __VA_ARGS__);               \
            else ROUTE_LAUNCH_E(KERNEL, _Float16, false, (r)->n_experts, __VA_ARGS__);                   \
        }                                                                                                \
    } while (0)

}  // namespace pgmoe

using namespace pgmoe;

extern "C" {

int pgmoe_route(const pgmoe_router *router, const void *logits, int64_t logits_stride, const float *bias, int T,
                int32_t *topk_idx, float *topk_weight, float *scores_out, void *stream) {
    const char *fn = "pgmoe_route";
    const int rc = check_router(router, fn);
    if (rc) return rc;
    if (const int bad = check_tokens(T, fn)) return bad;
    if (logits_stride < router->n_experts) return fail(nullptr, PGMOE_EINVAL, "%s: logits_stride=%lld is less than n_experts=%d", fn, (long long)logits_stride, router->n_experts);
    if (T == 0) return PGMOE_OK;
    const size_t elem = dtype_bytes(router->logits_dtype);
    NEED_PTR(nullptr, fn, logits, elem);
    OPT_PTR(nullptr, fn, bias, 4);
    NEED_PTR(nullptr, fn, topk_idx, 4);
    NEED_PTR(nullptr, fn, topk_weight, 4);
    OPT_PTR(nullptr, fn, scores_out, 4);
    const int groups = router->n_groups ? router->n_groups : 1, keep = router->topk_groups ? router->topk_groups : groups;
    RouteArgs a = {logits, (size_t)logits_stride, bias, T, router->n_experts, router->top_k, groups, keep, router->renormalize,
                   router->scale, topk_idx, topk_weight, scores_out, router->n_experts / groups, 0, 0, 0, 0};
    while (groups << (a.shift + 1) <= ROUTE_LANES) ++a.shift;
    a.straddle = groups > 1 && a.size != route_per(a.E) << a.shift;
    a.capacity = std::min(a.E, a.k + ROUTE_MORE);
    a.lds = ((bias || router->logits_dtype == PGMOE_F32 ? 16 * a.capacity : 4 * a.k) + (a.straddle ? 4 * a.E : 0) + 15) & ~15;
    // sixteen tokens a workgroup, four where that would take more than 40 KiB of LDS: four workgroups a CU either way
    const int threads = ROUTE_TOKENS * a.lds > 40 * 1024 ? 64 : ROUTE_THREADS, tokens = threads / ROUTE_LANES;
    const size_t lds = (size_t)tokens * a.lds;
    const bool vec = route_vec(router, logits, logits_stride) && aligned(bias, 16) && aligned(scores_out, 16);
    const dim3 grid((T + tokens - 1) / tokens), block(threads);
    ROUTE_LAUNCH(route_logits_kernel, router, vec, grid, block, lds, (hipStream_t)stream, a);
    return launched(fn);
}

int pgmoe_route_backward(const pgmoe_router *router, const void *logits, int64_t logits_stride, const int32_t *topk_idx,
                         const float *d_weight, const float *d_scores, int T, void *d_logits, int64_t d_logits_stride, void *stream) {
    const char *fn = "pgmoe_route_backward";
    const int rc = check_router(router, fn);
    if (rc) return rc;
    if (const int bad = check_tokens(T, fn)) return bad;
    if (logits_stride < router->n_experts || d_logits_stride < router->n_experts)
        return fail(nullptr, PGMOE_EINVAL, "%s: a stride (%lld, %lld) is less than n_experts=%d", fn, (long long)logits_stride, (long long)d_logits_stride, router->n_experts);
    if (T == 0) return PGMOE_OK;
    const size_t elem = dtype_bytes(router->logits_dtype);
    NEED_PTR(nullptr, fn, logits, elem);
    NEED_PTR(nullptr, fn, topk_idx, 4);
    NEED_PTR(nullptr, fn, d_weight, 4);
    OPT_PTR(nullptr, fn, d_scores, 4);
    NEED_PTR(nullptr, fn, d_logits, elem);
    if (rows_overlap(logits, logits_stride * elem, d_logits, d_logits_stride * elem, router->n_experts * elem, T)) return fail(nullptr, PGMOE_EINVAL, "%s: d_logits overlaps logits", fn);
    const RouteBackwardArgs a = {logits, (size_t)logits_stride, topk_idx, d_weight, d_scores, d_logits, (size_t)d_logits_stride,
                                 T, router->n_experts, router->top_k, router->renormalize, router->scale};
    const size_t lds = (size_t)ROUTE_THREADS * route_per(a.E) * 4;  // at most 16 KiB
    const dim3 grid((T + ROUTE_TOKENS - 1) / ROUTE_TOKENS), block(ROUTE_THREADS);
    const bool vec = route_vec(router, logits, logits_stride) && route_vec(router, d_logits, d_logits_stride) && aligned(d_scores, 16);
    ROUTE_LAUNCH(route_logits_backward_kernel, router, vec, grid, block, lds, (hipStream_t)stream, a);
    return launched(fn);
}

}  // extern "C"
