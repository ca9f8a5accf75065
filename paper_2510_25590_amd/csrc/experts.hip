// What surrounds products over groups of rows (regione_linear_grouped) where a router forms the groups: the choice of experts, the sort of the chosen (token, expert) pairs
// by expert, and the weighted sum of the experts' rows back at their tokens.
#include "common.h"
#include <math.h>
#include <type_traits>

namespace {

constexpr int kThreads = 256;
constexpr int kMostExperts = 1024, kMostChosen = 32, kMostGroups = 64;
constexpr int64_t kMostPairs = int64_t{1} << 24;             // rows that a grouped product takes
// Tokens from which on four share a wave, without and with scores to look at beside the logits (bias, groups).  us, a wave to a token / to four: 64 experts, float32, 6 chosen, 1024 tokens 3.6 / 3.4, 4608
// 4.8 / 3.8, 65536 29.6 / 11.0; 256 experts, bf16, 8 chosen, 1024 tokens 4.7 / 4.8, 2048 5.1 / 4.8, 65536 49 / 21; 256 experts in 8 groups with a bias, 8 chosen, 1024 tokens 6.9 / 8.8, 4608 10.4 / 10.7,
// 8192 13.9 / 12.1, 65536 85 / 52
constexpr int64_t kRouteShared = 2048, kRouteSharedScored = 8192;

typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;

// ---- choice of experts

struct RouteCall {
    const void* logits; const float* bias; const uint8_t* mask; int32_t* expert; float* weight;
    int64_t n_tokens; int n_experts, n_groups, top_groups, group_best, top_k, per, group_shift;   // experts per group; a group's lanes are 1 << group_shift
    int sigmoid, renormalise, whole; float scale;            // whole: every lane's experts exist and lie at a multiple of their own size
};

// Reductions over LPT lanes (16: a DPP row; 64: the wave) that leave the result in all of them.  Step X combines a lane with one of the other half of its 2 X lanes, whose X lanes agree by
// then: which of them does not matter, so that mirrors serve where DPP has no exchange.  Nothing goes through the LDS crossbar, whose latency is ten times as long.
template <int X> __device__ __forceinline__ int lane_across(int v) {
    if constexpr (X == 1) return __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xf, 0xf, true);              // quad_perm 1 0 3 2
    else if constexpr (X == 2) return __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xf, 0xf, true);         // quad_perm 2 3 0 1
    else if constexpr (X == 4) return __builtin_amdgcn_update_dpp(0, v, 0x141, 0xf, 0xf, true);        // row_half_mirror
    else if constexpr (X == 8) return __builtin_amdgcn_update_dpp(0, v, 0x140, 0xf, 0xf, true);        // row_mirror
    else {
        // the instruction exchanges the odd rows (the upper half) of one register with the even rows (the lower half) of the other
        const auto both = X == 16 ? __builtin_amdgcn_permlane16_swap(v, v, false, false) : __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return static_cast<int>(threadIdx.x & X ? both[0] : both[1]);
    }
}
template <int X> __device__ __forceinline__ unsigned lane_across(unsigned v) { return static_cast<unsigned>(lane_across<X>(static_cast<int>(v))); }
template <int X> __device__ __forceinline__ float lane_across(float v) { return __int_as_float(lane_across<X>(__float_as_int(v))); }
template <int X> __device__ __forceinline__ double lane_across(double v) { return __hiloint2double(lane_across<X>(__double2hiint(v)), lane_across<X>(__double2loint(v))); }
// both halves' values, in an order that is the same in all lanes
template <int X> __device__ __forceinline__ void lane_halves(int v, int& a, int& b) {
    const auto both = X == 16 ? __builtin_amdgcn_permlane16_swap(v, v, false, false) : __builtin_amdgcn_permlane32_swap(v, v, false, false);
    a = static_cast<int>(both[0]);
    b = static_cast<int>(both[1]);
}
template <int X> __device__ __forceinline__ void lane_halves(unsigned v, unsigned& a, unsigned& b) { lane_halves<X>(static_cast<int>(v), reinterpret_cast<int&>(a), reinterpret_cast<int&>(b)); }
template <int X> __device__ __forceinline__ void lane_halves(float v, float& a, float& b) {
    int x, y;
    lane_halves<X>(__float_as_int(v), x, y);
    a = __int_as_float(x);
    b = __int_as_float(y);
}
template <int X> __device__ __forceinline__ void lane_halves(double v, double& a, double& b) {
    int ah, al, bh, bl;
    lane_halves<X>(__double2hiint(v), ah, bh);
    lane_halves<X>(__double2loint(v), al, bl);
    a = __hiloint2double(ah, al);
    b = __hiloint2double(bh, bl);
}
template <int X, int LPT, typename V, typename F> __device__ __forceinline__ V over_lanes(V v, F f) {
    if constexpr (X >= LPT) {
        return v;
    } else if constexpr (X < 16) {
        return over_lanes<2 * X, LPT>(f(v, lane_across<X>(v)), f);
    } else {
        V a, b;
        lane_halves<X>(v, a, b);
        return over_lanes<2 * X, LPT>(f(a, b), f);
    }
}
__device__ __forceinline__ float bigger(float a, float b) { return __builtin_fmaxf(a, b); }
__device__ __forceinline__ double bigger(double a, double b) { return __builtin_fmax(a, b); }
__device__ __forceinline__ unsigned bigger(unsigned a, unsigned b) { return a > b ? a : b; }
__device__ __forceinline__ float smaller(float a, float b) { return __builtin_fminf(a, b); }
__device__ __forceinline__ double smaller(double a, double b) { return __builtin_fmin(a, b); }
__device__ __forceinline__ unsigned smaller(unsigned a, unsigned b) { return a < b ? a : b; }
template <int LPT, typename V> __device__ __forceinline__ V lanes_max(V v) { return over_lanes<1, LPT>(v, [](V a, V b) { return bigger(a, b); }); }
template <int LPT, typename V> __device__ __forceinline__ V lanes_min(V v) { return over_lanes<1, LPT>(v, [](V a, V b) { return smaller(a, b); }); }
template <int LPT, typename V> __device__ __forceinline__ V lanes_sum(V v) { return over_lanes<1, LPT>(v, [](V a, V b) { return a + b; }); }
// of lane `from`, the same number for all lanes of the token
template <int LPT> __device__ __forceinline__ int lane_value(int v, int from) {
    if constexpr (LPT == 64) return __builtin_amdgcn_readlane(v, from);
    else return __builtin_amdgcn_ds_bpermute(from * 4, v);
}
template <int LPT> __device__ __forceinline__ float lane_value(float v, int from) { return __int_as_float(lane_value<LPT>(__float_as_int(v), from)); }
template <int LPT> __device__ __forceinline__ double lane_value(double v, int from) { return __hiloint2double(lane_value<LPT>(__double2hiint(v), from), lane_value<LPT>(__double2loint(v), from)); }

// Two largest values of the lanes of a group (1 to LPT lanes).
template <int X, int LPT, typename V> __device__ __forceinline__ void best_two(V& a, V& b, int lanes) {
    if constexpr (X < LPT) {
        if (X >= lanes) return;
        const V oa = lane_across<X>(a), ob = lane_across<X>(b);
        b = bigger(smaller(a, oa), bigger(b, ob));
        a = bigger(a, oa);
        best_two<2 * X, LPT>(a, b, lanes);
    }
}

template <typename T> __device__ __forceinline__ float as_float(T v);
template <> __device__ __forceinline__ float as_float<float>(float v) { return v; }
template <> __device__ __forceinline__ float as_float<bf16_t>(bf16_t v) { return bf16_to_f32(v); }

// A value and its expert as one number, larger for larger values and, among equal ones, for lower experts: a maximum finds both at once.  Float32 values are put into the upper bits of
// a double, whose lowest ten hold the expert; bf16 values into the upper half of a word.  A value of -infinity is no expert.
struct WideKey {
    typedef double type;
    static constexpr double NONE = -INFINITY;
    static constexpr int PAST = 0x7fe00000;                                // of 2^1023, past all float32 values, in the place of +infinity, which cannot hold an expert: with other bits set it is NaN
    static __device__ __forceinline__ double make(float v, int expert) {
        v += 0.0f;                                                         // (-0 is as large as 0)
        const double d = static_cast<double>(v);
        const int low = (1023 - expert) ^ ((__float_as_int(v) >> 31) & 1023);
        const int high = __double2hiint(d) < PAST ? __double2hiint(d) : PAST;
        return __hiloint2double(high, v > -INFINITY ? __double2loint(d) | low : 0);
    }
    static __device__ __forceinline__ int expert(double k) { return 1023 - ((__double2loint(k) & 1023) ^ ((__double2hiint(k) >> 31) & 1023)); }
    static __device__ __forceinline__ float value(double k) { return static_cast<float>(__hiloint2double(__double2hiint(k), __double2loint(k) & ~1023)); }
};
struct NarrowKey {
    typedef unsigned type;
    static constexpr unsigned NONE = 0;
    static __device__ __forceinline__ unsigned make(float v, int expert) {
        unsigned bits = __float_as_uint(v);
        bits = bits == 0x80000000u ? 0u : bits;                            // (-0 is as large as 0)
        const unsigned ordered = bits ^ (static_cast<unsigned>(static_cast<int>(bits) >> 31) | 0x80000000u);
        return v > -INFINITY ? (ordered & 0xffff0000u) | static_cast<unsigned>(1023 - expert) : NONE;
    }
    static __device__ __forceinline__ int expert(unsigned k) { return 1023 - static_cast<int>(k & 1023u); }
    static __device__ __forceinline__ float value(unsigned k) {
        const unsigned bits = k >> 16;
        return __uint_as_float((bits & 0x8000u ? bits & 0x7fffu : ~bits & 0xffffu) << 16);
    }
};

// Falling order by Batcher's odd-even merge sort.
template <int N, typename K> __device__ __forceinline__ void sort_falling(K (&v)[N]) {
#pragma unroll
    for (int p = 1; p < N; p *= 2)
#pragma unroll
        for (int k = p; k >= 1; k /= 2)
#pragma unroll
            for (int j = k % p; j + k < N; j += 2 * k)
#pragma unroll
                for (int i = 0; i < k; ++i)
                    if (i + j + k < N && (i + j) / (2 * p) == (i + j + k) / (2 * p)) {
                        const K a = v[i + j], b = v[i + j + k];
                        v[i + j] = bigger(a, b);
                        v[i + j + k] = smaller(a, b);
                    }
}
// b where the mask is set, a elsewhere: written as a selection, array elements i and i + 1 become one element of a computed number.
__device__ __forceinline__ unsigned merge(unsigned a, unsigned b, unsigned mask) { return (b & mask) | (a & ~mask); }
__device__ __forceinline__ double merge(double a, double b, unsigned mask) {
    return __hiloint2double(static_cast<int>(merge(static_cast<unsigned>(__double2hiint(a)), static_cast<unsigned>(__double2hiint(b)), mask)),
                            static_cast<int>(merge(static_cast<unsigned>(__double2loint(a)), static_cast<unsigned>(__double2loint(b)), mask)));
}
// Lane j < top_k of the token's ends up with its choice j as a key.
template <typename KEY, int LPT, int EPL>
__device__ __forceinline__ typename KEY::type choose(typename KEY::type (&v)[EPL], int l, int top_k) {
    typedef typename KEY::type K;
    constexpr bool SORTED = EPL <= 16;
    if constexpr (SORTED) sort_falling(v);
    K chosen = KEY::NONE;
    for (int j = 0; j < top_k; ++j) {
        K best = v[0];
        if constexpr (!SORTED) {
#pragma unroll
            for (int i = 1; i < EPL; ++i) best = bigger(best, v[i]);
        }
        const K most = lanes_max<LPT>(best);
        if constexpr (SORTED) {
            const unsigned mine = v[0] == most ? ~0u : 0u;
#pragma unroll
            for (int i = 0; i + 1 < EPL; ++i) v[i] = merge(v[i], v[i + 1], mine);
            v[EPL - 1] = merge(v[EPL - 1], KEY::NONE, mine);
        } else {
#pragma unroll
            for (int i = 0; i < EPL; ++i) v[i] = v[i] == most ? KEY::NONE : v[i];
        }
        chosen = l == j ? most : chosen;
    }
    return chosen;
}

// Where the whole wave chooses for one token, which lane and which of its places hold a maximum is a matter of scalar instructions, and the keys need not hold the expert: float32 values in the
// order of words, 0 for no expert.  Lane j < top_k ends up with its choice j (others are left as they were).
__device__ __forceinline__ unsigned ordered(float v) {
    const unsigned bits = __float_as_uint(v + 0.0f);                       // (-0 is as large as 0)
    return v > -INFINITY ? bits ^ (static_cast<unsigned>(static_cast<int>(bits) >> 31) | 0x80000000u) : 0u;
}
__device__ __forceinline__ float from_ordered(unsigned k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
template <int EPL>
__device__ __forceinline__ void choose_wave(unsigned (&v)[EPL], int top_k, int shift, int per, int& chosen, unsigned& its) {
    for (int j = 0; j < top_k; ++j) {
        unsigned best = v[0];
#pragma unroll
        for (int i = 1; i < EPL; ++i) best = bigger(best, v[i]);
        const unsigned most = static_cast<unsigned>(__builtin_amdgcn_readfirstlane(static_cast<int>(lanes_max<64>(best))));
        if (most == 0) break;
        uint64_t held[EPL], any = 0;
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
            held[i] = __ballot(v[i] == most);
            any |= held[i];
        }
        const int owner = __builtin_ctzll(any);
        const uint64_t bit = uint64_t{1} << owner;
        int place = 0;
        bool open = true;
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
            const bool here = open && (held[i] & bit) != 0;
            place = here ? i : place;
            open = open && !here;
            const bool gone = here && static_cast<int>(threadIdx.x & 63) == owner;
            v[i] = gone ? 0u : v[i];
        }
        const bool mine = static_cast<int>(threadIdx.x & 63) == j;
        chosen = mine ? (owner >> shift) * per + (owner & ((1 << shift) - 1)) * EPL + place : chosen;
        its = mine ? most : its;
    }
}

// The groups that stay: a group's place is the number of groups that come before it, those with more and those with as much and a lower number.  sum: of the lane's group.
template <int LPT, typename V> __device__ __forceinline__ bool group_stays(const RouteCall& c, V sum, int lane, int group) {
    int before = 0;
    if constexpr (std::is_same<V, float>::value) {
        const unsigned mine = ordered(sum);
#pragma unroll 4
        for (int h = 0; h < c.n_groups; ++h) {
            const unsigned other = static_cast<unsigned>(lane_value<LPT>(static_cast<int>(mine), LPT == 64 ? h << c.group_shift : (lane & ~(LPT - 1)) + (h << c.group_shift)));
            before += (h < group ? other >= mine : other > mine) ? 1 : 0;
        }
        return before < c.top_groups;
    }
#pragma unroll 4
    for (int h = 0; h < c.n_groups; ++h) {
        const V other = lane_value<LPT>(sum, LPT == 64 ? h << c.group_shift : (lane & ~(LPT - 1)) + (h << c.group_shift));
        before += other > sum || (other == sum && h < group) ? 1 : 0;
    }
    return before < c.top_groups;
}
template <int LPT, int EPL, typename V> __device__ __forceinline__ V group_sum(const RouteCall& c, const V (&value)[EPL]) {
    V a = -INFINITY, b = -INFINITY;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
        b = bigger(b, smaller(a, value[i]));
        a = bigger(a, value[i]);
    }
    best_two<1, LPT>(a, b, 1 << c.group_shift);
    return c.group_best == 2 && b > static_cast<V>(-INFINITY) ? a + b : a;
}

// exp(x) to 2^-46 (2^-44 for x of hundreds), in 64 bits so that nothing but the last rounding counts in float32: 2^n times the exponential's series up to the eleventh power of |r| <= ln(2) / 2 (the twelfth is 2^-47).
__device__ __forceinline__ double exp64(double x) {
    x = __builtin_fmin(__builtin_fmax(x, -800.0), 800.0);
    const double n = __builtin_rint(x * 1.4426950408889634), r = __builtin_fma(n, -0.6931471805599453, x);
    double p = 1.0 / 39916800.0;
    p = __builtin_fma(p, r, 1.0 / 3628800.0);
    p = __builtin_fma(p, r, 1.0 / 362880.0);
    p = __builtin_fma(p, r, 1.0 / 40320.0);
    p = __builtin_fma(p, r, 1.0 / 5040.0);
    p = __builtin_fma(p, r, 1.0 / 720.0);
    p = __builtin_fma(p, r, 1.0 / 120.0);
    p = __builtin_fma(p, r, 1.0 / 24.0);
    p = __builtin_fma(p, r, 1.0 / 6.0);
    p = __builtin_fma(p, r, 0.5);
    p = __builtin_fma(p, r, 1.0);
    p = __builtin_fma(p, r, 1.0);
    return __builtin_ldexp(p, static_cast<int>(n));
}
// 1 / x for x of 2^-1023 to 2^1023, to about 2^-45: the reciprocal instruction and one step of Newton's; 0 for infinity
__device__ __forceinline__ double over64(double x) {
    const double r = __builtin_amdgcn_rcp(x);
    return x < INFINITY ? __builtin_fma(r, __builtin_fma(-x, r, 1.0), r) : 0.0;
}

// The choice in 64 bits.  Returns the expert and sets its logit in lane j.
template <int LPT, int EPL>
__device__ __forceinline__ int choose_exactly(const RouteCall& c, const float (&logit)[EPL], float top, int l, int lane, int group, int expert0, int mine, float& chosen_logit) {
    constexpr double NONE = -INFINITY;
    double value[EPL], all = 0.0;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
        value[i] = logit[i] == -INFINITY ? 0.0 : exp(c.sigmoid ? -static_cast<double>(logit[i]) : static_cast<double>(logit[i]) - static_cast<double>(top));
        all += value[i];
    }
    if (!c.sigmoid) all = lanes_sum<LPT>(all);
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
        double v = c.sigmoid ? 1.0 / (1.0 + value[i]) : value[i] / all;
        if (c.bias && i < mine) v += static_cast<double>(c.bias[expert0 + i]);
        value[i] = logit[i] > -INFINITY && v > NONE ? v : NONE;            // (a bias of NaN or -infinity takes its expert out)
    }
    if (c.n_groups > 1) {
        const bool stays = group_stays<LPT>(c, group_sum<LPT, EPL>(c, value), lane, group);
#pragma unroll
        for (int i = 0; i < EPL; ++i) value[i] = !stays ? NONE : c.bias ? value[i] : static_cast<double>(logit[i]);
    }
    int chosen = -1;
    chosen_logit = 0.f;
    for (int j = 0; j < c.top_k; ++j) {
        double best = value[0];
#pragma unroll
        for (int i = 1; i < EPL; ++i) best = bigger(best, value[i]);
        const double most = lanes_max<LPT>(best);
        const uint64_t held = __ballot(best == most && most > NONE);
        const unsigned seg = LPT == 64 ? 0 : static_cast<unsigned>(lane & ~(LPT - 1));
        const uint64_t here = LPT == 64 ? held : (held >> seg) & ((uint64_t{1} << (LPT & 63)) - 1);
        if (held == 0) break;
        const int owner = here ? __builtin_ctzll(here) : 0;
        int place = 0;
        float its = 0.f;
        bool found = !(here && l == owner);
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
            const bool hit = !found && value[i] == most;
            place = hit ? i : place;
            its = hit ? logit[i] : its;
            value[i] = hit ? NONE : value[i];
            found = found || hit;
        }
        const int from = static_cast<int>(seg + owner) * 4;
        const int e = __builtin_amdgcn_ds_bpermute(from, expert0 + place);
        const float x = __int_as_float(__builtin_amdgcn_ds_bpermute(from, __float_as_int(its)));
        if (l == j && here) { chosen = e; chosen_logit = x; }
    }
    return chosen;
}

// The first `looked` lanes' experts, with their logits, in the order of their values in 64 bits.
template <int LPT, int EPL>
__device__ __forceinline__ void put_in_order(const RouteCall& c, const float (&logit)[EPL], float top, int l, int lane, int looked, float bias, int& chosen, float& chosen_logit) {
    const double x = static_cast<double>(chosen_logit);
    double v = exp(c.sigmoid ? -x : x - static_cast<double>(top));
    if (c.sigmoid) {
        v = 1.0 / (1.0 + v);
    } else {
        double all = 0.0;
#pragma unroll 1
        for (int i = 0; i < EPL; ++i) {
            float at = logit[0];
#pragma unroll
            for (int q = 1; q < EPL; ++q) at = i == q ? logit[q] : at;
            all += at == -INFINITY ? 0.0 : exp(static_cast<double>(at) - static_cast<double>(top));
        }
        v /= lanes_sum<LPT>(all);
    }
    v = chosen < 0 ? -INFINITY : v + static_cast<double>(bias);
    const int e = chosen < 0 ? 1024 + l : chosen;
    int rank = 0;
#pragma unroll 1
    for (int j = 0; j < looked; ++j) {
        const int from = LPT == 64 ? j : (lane & ~(LPT - 1)) + j;
        const double other = lane_value<LPT>(v, from);
        rank += other > v || (other == v && lane_value<LPT>(e, from) < e) ? 1 : 0;
    }
    const int to = ((lane & ~(LPT - 1)) + (l < looked ? rank : l)) * 4;
    chosen = __builtin_amdgcn_ds_permute(to, chosen);
    chosen_logit = __int_as_float(__builtin_amdgcn_ds_permute(to, __float_as_int(chosen_logit)));
}

// LPT lanes choose the experts of a token.  A group has LPT / (n_groups rounded up to a power of two) lanes of EPL experts each, in order, so that the lowest lane and then its lowest
// place hold the lowest expert.
// Without bias and groups the scores lie in the order of the logits (SCORED false).  With them the choice is that of values in 64 bits: in 32 bits the rounding of the exponential would decide
// between experts that differ by less, and another order of the same operations would choose others.  It is made in 32 bits all the same, and made again in 64 where that cannot be sure: where
// two values that follow each other in the choice, or the last group that stays and the first that does not, are closer than the errors of both.  (Equal values of equal logits and biases are.)
// What bounds it: instructions, and for few tokens the chain of maxima.  Kernel trace, us: one token of 64 experts 2.3; 65536 tokens of 128 experts, bf16, 8 chosen, 11.3 to 12.7 (1.7 TB/s; 390 vector instructions per
// wave of four tokens); 4608 tokens of 256 experts, float32, in 8 groups with a bias, 10 to 11 (790 per wave and token).
template <typename T, int LPT, int EPL, bool SCORED>
__global__ void __launch_bounds__(kThreads)
route_kernel(RouteCall c) {
    typedef typename std::conditional<!SCORED && sizeof(T) == 2, NarrowKey, WideKey>::type Key;
    const int lane = threadIdx.x & 63, l = lane & (LPT - 1);
    const int64_t token = (static_cast<int64_t>(blockIdx.x) * (kThreads / 64) + (threadIdx.x >> 6)) * (64 / LPT) + lane / LPT;
    if (token - lane / LPT >= c.n_tokens) return;                          // (the whole wave)
    const bool there = token < c.n_tokens, routed = there && (!c.mask || c.mask[token] != 0);
    const int group_lanes = SCORED ? 1 << c.group_shift : LPT, group = SCORED ? l >> c.group_shift : 0, per = SCORED ? c.per : c.n_experts;
    const int first = (l & (group_lanes - 1)) * EPL, expert0 = group * per + first;      // of this lane
    int mine = group < c.n_groups ? per - first : 0;                       // its experts
    mine = mine < 0 ? 0 : (mine < EPL ? mine : EPL);

    float logit[EPL];
    const T* row = static_cast<const T*>(c.logits) + (routed ? token : 0) * c.n_experts;
    if (c.whole) {
        typedef T piece __attribute__((ext_vector_type(EPL * sizeof(T) > 16 ? 16 / sizeof(T) : EPL)));
        constexpr int PE = sizeof(piece) / sizeof(T);
        piece p[EPL / PE];
        const bool any = group < c.n_groups;
#pragma unroll
        for (int i = 0; i < EPL / PE; ++i) p[i] = reinterpret_cast<const piece*>(row + (any ? expert0 : 0))[i];
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
            T v;
            if constexpr (PE == 1) v = reinterpret_cast<const T*>(p)[i]; else v = p[i / PE][i % PE];
            logit[i] = any ? as_float<T>(v) : -INFINITY;
        }
    } else {
#pragma unroll
        for (int i = 0; i < EPL; ++i) logit[i] = i < mine ? as_float<T>(row[expert0 + i]) : -INFINITY;
    }
    float bias[SCORED ? EPL : 1];                                          // (requested with the logits)
    if constexpr (SCORED) {
        if (c.bias && c.whole) {
            typedef float piece __attribute__((ext_vector_type(EPL > 4 ? 4 : EPL)));
            constexpr int PE = sizeof(piece) / sizeof(float);
#pragma unroll
            for (int i = 0; i < EPL; i += PE) {
                const piece p = *reinterpret_cast<const piece*>(c.bias + (group < c.n_groups ? expert0 : 0) + i);
#pragma unroll
                for (int e = 0; e < PE; ++e) bias[i + e] = reinterpret_cast<const float*>(&p)[e];
            }
        } else {
#pragma unroll
            for (int i = 0; i < EPL; ++i) bias[i] = c.bias && i < mine ? c.bias[expert0 + i] : 0.f;
        }
    }
    // NaN is no score at all; what overflows counts as the largest value there is (NarrowKey: in its place, infinity)
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
        if constexpr (std::is_same<Key, WideKey>::value) logit[i] = logit[i] < 3.402823466e38f ? logit[i] : logit[i] > 0.f ? 3.402823466e38f : -INFINITY;
        else logit[i] = logit[i] > -INFINITY ? logit[i] : -INFINITY;
    }

    float top = 0.f;
    double all = 0.0;                                                      // sum of the softmax's exponentials
    if (!c.sigmoid && (SCORED || !c.renormalise)) {
        top = logit[0];
#pragma unroll
        for (int i = 1; i < EPL; ++i) top = bigger(top, logit[i]);
        top = lanes_max<LPT>(top);
        top = __builtin_fminf(top, 3.402823466e38f);
    }
    typedef typename std::conditional<LPT == 64, unsigned, typename Key::type>::type K;
    K key[EPL];
    auto make_key = [](float v, int expert) { if constexpr (LPT == 64) return ordered(v); else return Key::make(v, expert); };
    float value[EPL];
    float thin = INFINITY;                                                 // the gap between the groups that stay and the others, less what it has to be at least
    if constexpr (SCORED) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
            value[i] = logit[i] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((c.sigmoid ? -logit[i] : logit[i] - top) * 1.4426950408889634f);
            sum += value[i];
        }
        if (!c.sigmoid) sum = lanes_sum<LPT>(sum);
        const float over = c.sigmoid ? 1.f : __builtin_amdgcn_rcpf(sum);
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
            float v = c.sigmoid ? __builtin_amdgcn_rcpf(1.f + value[i]) : value[i] * over;
            if (c.bias) v += bias[i];
            value[i] = logit[i] > -INFINITY && v > -INFINITY ? v : -INFINITY;
        }
        bool stays = true;
        if (c.n_groups > 1) {
            const float s = group_sum<LPT, EPL>(c, value);
            stays = group_stays<LPT>(c, s, lane, group);
            if (c.top_groups < c.n_groups) {
                const bool real = group < c.n_groups;
                const float in = lanes_min<LPT>(real && stays ? s : INFINITY), out = lanes_max<LPT>(real && !stays ? s : -INFINITY);
                // in = out = -infinity (groups without experts) is sure; so are infinite gaps
                thin = in == -INFINITY || in - out == INFINITY ? INFINITY : in - out - 0x1p-20f * ((c.sigmoid ? 1.25f : 16.f) + 0.5f * (__builtin_fabsf(in) + __builtin_fabsf(out)));
                thin = thin == thin ? thin : -1.f;
            }
        }
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
            value[i] = stays ? value[i] : -INFINITY;
            key[i] = make_key(!stays ? -INFINITY : c.bias ? value[i] : logit[i], expert0 + i);
        }
    } else {
        if (!c.sigmoid && !c.renormalise) {
            // (in 64 bits, as with bias or groups: in float32 a weight of 128 experts is off by up to three half steps.  65536 tokens, bf16, float32 / this
            // 14.9 / 19.1 us)
#pragma unroll
            for (int i = 0; i < EPL; ++i) all += logit[i] == -INFINITY ? 0.0 : exp64(static_cast<double>(__builtin_fminf(logit[i], 3.402823466e38f)) - static_cast<double>(top));
            all = lanes_sum<LPT>(all);
        }
#pragma unroll
        for (int i = 0; i < EPL; ++i) key[i] = make_key(logit[i], expert0 + i);
    }

    // lane j of the token's ends up with its choice j; where the choice has to be sure, the first two that are not chosen are looked at, too
    const bool check = SCORED && c.bias != nullptr;
    const int looked = check ? c.top_k + 2 : c.top_k;
    int chosen = -1;
    float chosen_logit = 0.f;
    if constexpr (LPT == 64) {
        unsigned its = 0;
        choose_wave<EPL>(key, looked, SCORED ? c.group_shift : 6, per, chosen, its);
        if (chosen >= 0) chosen_logit = from_ordered(its);
    } else {
        const K took = choose<Key, LPT, EPL>(key, l, looked);
        if (took != Key::NONE) { chosen = Key::expert(took); chosen_logit = Key::value(took); }
    }
    if constexpr (SCORED) {
        bool sure = thin > 0.f;
        if (check) {
            const float v = chosen < 0 ? -INFINITY : chosen_logit, b = chosen < 0 ? 0.f : c.bias[chosen];
            chosen_logit = chosen < 0 ? 0.f : __builtin_fminf(as_float<T>(row[chosen]), 3.402823466e38f);      // (as in `logit`: from +infinity every difference is infinite)
            const float next_v = __shfl_down(v, 1, LPT), next_b = __shfl_down(b, 1, LPT), next_x = __shfl_down(chosen_logit, 1, LPT), last_v = __shfl_down(v, 2, LPT);
            // What two values may be off together, in 2^-24.  Softmax, times the score: 2 each for its exponential and the reciprocal, 1 for their product, 37 for the additions of the sum (32 in a lane, over
            // 64 of them), 2 + 2.5 ln(1024) for the sum's exponentials, at most 60 in all, and 2.5 |x - top| for the score's exponent, which with the score is at most 0.92.  Sigmoid: 3.5.  For the bias 1
            // times each value.  `least`: this value and the next; `wide`: this one and any, as two scores add up to 1 at most (`least` there does not know of the other's score).
            const float least = (c.sigmoid ? 0x1p-21f : 0x1p-20f) * (1.f + __builtin_fabsf(v)) + (c.sigmoid ? 0.f : 0x1p-17f * (__builtin_fabsf(v - b) + __builtin_fabsf(next_v - next_b)));
            const float wide = (c.sigmoid ? 0x1p-21f : 0x1p-18f) * (1.f + __builtin_fabsf(v));
            const bool near = l < c.top_k && next_v > -INFINITY && !(v - next_v > least) && !(next_x == chosen_logit && next_b == b);
            // the last choice and the second one behind it too near: there may be more of them (infinities of one sign: as near as can be)
            const bool crowded = l == c.top_k - 1 && last_v > -INFINITY && !(v - last_v > wide);
            if (__ballot(crowded && routed)) {
                const int from = LPT == 64 ? c.top_k - 1 : (lane & ~(LPT - 1)) + c.top_k - 1;
                const float edge_v = lane_value<LPT>(v, from), edge_b = lane_value<LPT>(b, from), edge_x = lane_value<LPT>(chosen_logit, from), edge = lane_value<LPT>(wide, from);
                const bool look = lane_value<LPT>(crowded ? 1 : 0, from) != 0;
#pragma unroll
                for (int i = 0; i < EPL; ++i)
                    if (look && i < mine && !(__builtin_fabsf(value[i] - edge_v) > edge) && value[i] > -INFINITY) sure = sure && logit[i] == edge_x && c.bias[expert0 + i] == edge_b;
            }
            if (__ballot(near && routed)) put_in_order<LPT, EPL>(c, logit, top, l, lane, looked, b, chosen, chosen_logit);
            if (l >= c.top_k) chosen = -1;
        }
        chosen_logit = __builtin_fminf(chosen_logit, 3.402823466e38f);
        // once for all tokens of the wave
        if (__ballot(!sure && routed)) {
            chosen = choose_exactly<LPT, EPL>(c, logit, top, l, lane, group, expert0, mine, chosen_logit);
        }
        if (!c.sigmoid && !c.renormalise) {
            all = 0.0;
#pragma unroll
            for (int i = 0; i < EPL; ++i) all += logit[i] == -INFINITY ? 0.0 : exp(static_cast<double>(logit[i]) - static_cast<double>(top));
            all = lanes_sum<LPT>(all);
        }
    }
    // Weights, in 64 bits: once per wave.  Renormalised softmax weights do not depend on the other experts, nor on how far below them the chosen ones lie.
    chosen_logit = __builtin_fminf(chosen_logit, 3.402823466e38f);
    const bool has = routed && chosen >= 0;
    double w = 0.0;
    if (c.sigmoid) {
        w = has && chosen_logit > -709.f ? over64(1.0 + exp64(-static_cast<double>(chosen_logit))) : 0.0;       // (e^709 is 2^1022.9)
    } else {
        const float from = c.renormalise ? lanes_max<LPT>(has ? chosen_logit : -INFINITY) : top;
        w = has ? exp64(static_cast<double>(chosen_logit) - static_cast<double>(from)) : 0.0;
    }
    if (c.renormalise) all = lanes_sum<LPT>(w);
    if (c.renormalise || !c.sigmoid) w = all > 0.0 ? w * over64(all) : 0.0;
    if (there && l < c.top_k) {
        c.expert[token * c.top_k + l] = has ? chosen : -1;
        c.weight[token * c.top_k + l] = has ? static_cast<float>(w * static_cast<double>(c.scale)) : 0.f;
    }
}

// experts of a lane where LPT lanes share a token
int experts_per_lane(RouteCall& c, int lpt) {
    c.per = c.n_experts / c.n_groups;
    c.group_shift = lpt == 16 ? 4 : 6;
    for (int g = 1; g < c.n_groups; g *= 2) --c.group_shift;
    return (c.per + (1 << c.group_shift) - 1) >> c.group_shift;
}
template <typename T, int LPT, int EPL>
int launch_route(regione_ctx* ctx, RouteCall& c, bool scored) {
    c.whole = c.per == EPL << c.group_shift && rg_aligned16(c.bias);
    const int64_t tokens_per = (kThreads / 64) * (64 / LPT), blocks = (c.n_tokens + tokens_per - 1) / tokens_per;
    if (scored) hipLaunchKernelGGL((route_kernel<T, LPT, EPL, true>), dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, ctx->stream, c);
    else hipLaunchKernelGGL((route_kernel<T, LPT, EPL, false>), dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, ctx->stream, c);
    RG_LAUNCH_CHECK();
    return REGIONE_OK;
}
template <typename T>
int launch_route(regione_ctx* ctx, RouteCall& c, bool scored) {
    // (two lanes more than choices)
    if (c.n_tokens >= (scored ? kRouteSharedScored : kRouteShared) && c.top_k <= 14 && c.n_groups <= 16) {
        const int need = experts_per_lane(c, 16);
        if (need <= 4) return launch_route<T, 16, 4>(ctx, c, scored);
        if (need <= 8) return launch_route<T, 16, 8>(ctx, c, scored);
        if (need <= 16) return launch_route<T, 16, 16>(ctx, c, scored);
    }
    const int need = experts_per_lane(c, 64);
    if (need <= 1) return launch_route<T, 64, 1>(ctx, c, scored);
    if (need <= 2) return launch_route<T, 64, 2>(ctx, c, scored);
    if (need <= 4) return launch_route<T, 64, 4>(ctx, c, scored);
    if (need <= 8) return launch_route<T, 64, 8>(ctx, c, scored);
    if (need <= 16) return launch_route<T, 64, 16>(ctx, c, scored);
    return launch_route<T, 64, 32>(ctx, c, scored);
}

// ---- the sort by expert

// A stable counting sort.  The pairs are cut into chunks of whole parts of 1024 * AHEAD; every workgroup counts its chunk, and a second launch places it behind the chunks before: a wave owns
// 64 * AHEAD consecutive pairs of a part, which stay in its registers between their counting and their placing, so that a pair's place is its expert's first row + the expert's pairs of
// earlier chunks, of earlier parts, of earlier waves, and of earlier pairs of its wave.
// Latency throughout: a few trips to memory, and a chain of LDS accesses per 64 pairs of a wave.  us, AHEAD 2 / 4 / 8 (one launch where a part holds all pairs, else two): 72 pairs of 16
// experts 3.7 / 4.3 / 5.8, 4096 of 128 7.8 / 6.3 / 7.9, 8192 of 128 7.9 / 9.5 / 9.2, 65536 of 128 9.0 / 10.2 / 14.0, 524288 of 128 11.1 / 11.6 / 15.0, of 256 13.3 / 12.5 / 15.3.
// The token of a pair by a multiplication and the ranks in 32-bit halves: 4096 pairs 6.6 -> 6.2, 524288 12.6 -> 12.4 (with AHEAD 4, another card).
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64, kMostChunks = 256;

// pair number q of a lane: the wave's pairs 64 q + lane
template <int AHEAD>
__device__ __forceinline__ void load_pairs(const int32_t* expert, int64_t wave0, int64_t end, int n_experts, int (&id)[AHEAD]) {
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) {
        const int64_t at = wave0 + 64 * q + (threadIdx.x & 63);
        id[q] = at < end ? expert[at] : -1;
    }
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) id[q] = id[q] >= 0 && id[q] < n_experts ? id[q] : -1;
}
template <int AHEAD>
__global__ void __launch_bounds__(kSortThreads)
count_pairs_kernel(const int32_t* __restrict__ expert, int64_t n, int64_t per_chunk, int n_experts, int32_t* __restrict__ counts) {
    __shared__ int32_t count[kMostExperts];
    for (int e = threadIdx.x; e < n_experts; e += kSortThreads) count[e] = 0;
    __syncthreads();
    const int64_t begin = static_cast<int64_t>(blockIdx.x) * per_chunk, end = begin + per_chunk < n ? begin + per_chunk : n;
    for (int64_t part = begin; part < end; part += kSortThreads * AHEAD) {
        int id[AHEAD];
        load_pairs(expert, part + (threadIdx.x >> 6) * (64 * AHEAD), end, n_experts, id);
#pragma unroll
        for (int q = 0; q < AHEAD; ++q)
            if (id[q] >= 0) atomicAdd(&count[id[q]], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < n_experts; e += kSortThreads) counts[static_cast<int64_t>(blockIdx.x) * n_experts + e] = count[e];
}
// counts: [chunks][n_experts], or null where there is one chunk.  A thread per expert adds things up; the sums over the chunks are shared by all threads.
template <int AHEAD>
__global__ void __launch_bounds__(kSortThreads)
place_pairs_kernel(const int32_t* __restrict__ expert, int64_t n, int64_t per_chunk, int n_experts, int bits, unsigned inverse, const int32_t* __restrict__ counts,
                   int32_t* __restrict__ offsets, int32_t* __restrict__ row_token, int32_t* __restrict__ slot) {
    extern __shared__ int32_t lds[];                                       // [kSortWaves][n_experts], then [kSortWaves]; before that the threads' sums over the chunks
    int32_t* const sums = lds + kSortWaves * n_experts;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e = threadIdx.x;
    const int64_t begin = static_cast<int64_t>(blockIdx.x) * per_chunk, end = begin + per_chunk < n ? begin + per_chunk : n;
    int id[AHEAD];
    load_pairs(expert, begin + wave * (64 * AHEAD), end, n_experts, id);

    int before = 0, all = 0;                                               // this thread's expert's pairs: of the chunks before, and all
    if (counts) {
        const int shares = kSortThreads / n_experts, mine = e / n_experts, chunks = static_cast<int>(gridDim.x);
        if (mine < shares) {
            const int32_t* const at = counts + (e - mine * n_experts);
#pragma unroll 8
            for (int c = mine; c < chunks; c += shares) {
                const int v = at[static_cast<int64_t>(c) * n_experts];
                before += c < static_cast<int>(blockIdx.x) ? v : 0;
                all += v;
            }
            lds[e] = before;
            lds[kSortThreads + e] = all;
        }
        __syncthreads();
        before = all = 0;
        if (e < n_experts)
            for (int t = e; t < shares * n_experts; t += n_experts) {
                before += lds[t];
                all += lds[kSortThreads + t];
            }
        __syncthreads();
    }
    int next = 0;                                                          // where this thread's expert's next pair goes
    for (int64_t part = begin; part < end || part == begin; part += kSortThreads * AHEAD) {
        if (part != begin) load_pairs(expert, part + wave * (64 * AHEAD), end, n_experts, id);
        for (int i = threadIdx.x; i < kSortWaves * n_experts; i += kSortThreads) lds[i] = 0;
        __syncthreads();
#pragma unroll
        for (int q = 0; q < AHEAD; ++q)
            if (id[q] >= 0) atomicAdd(&lds[wave * n_experts + id[q]], 1);
        __syncthreads();
        if (part == begin) {
            if (!counts && e < n_experts) for (int w = 0; w < kSortWaves; ++w) all += lds[w * n_experts + e];
            int upto = all;                                                // inclusive sums over the experts
            for (int d = 1; d < 64; d *= 2) {
                const int v = __shfl_up(upto, d);
                upto += lane >= d ? v : 0;
            }
            if (lane == 63) sums[wave] = upto;
            __syncthreads();
            for (int w = 0; w < wave; ++w) upto += sums[w];
            next = upto - all + before;
            if (blockIdx.x == 0 && e < n_experts) {
                offsets[e + 1] = upto;
                if (e == 0) offsets[0] = 0;
            }
        }
        if (e < n_experts)
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) {
                const int v = lds[w * n_experts + e];
                lds[w * n_experts + e] = next;
                next += v;
            }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < AHEAD; ++q) {
            const unsigned i = static_cast<unsigned>(part) + wave * (64 * AHEAD) + 64 * q + lane;
            const uint64_t there = __ballot(id[q] >= 0);
            unsigned low = static_cast<unsigned>(there), high = static_cast<unsigned>(there >> 32);      // lanes with this lane's expert
            for (int b = 0; b < bits; ++b) {
                const unsigned other = ((id[q] >> b) & 1) - 1u;            // all ones where the bit is not set
                const uint64_t with = __ballot(other == 0u);
                low &= static_cast<unsigned>(with) ^ other;
                high &= static_cast<unsigned>(with >> 32) ^ other;
            }
            const uint64_t same = static_cast<uint64_t>(high) << 32 | low;
            const int rank = __builtin_amdgcn_mbcnt_hi(static_cast<unsigned>(same >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<unsigned>(same), 0));
            if (id[q] >= 0) {
                volatile int32_t* const to = &lds[wave * n_experts + id[q]];      // (the other lanes change it)
                const int place = *to + rank;
                __builtin_amdgcn_wave_barrier();
                if (rank == 0) *to = place + __builtin_popcountll(same);
                slot[i] = place;
                row_token[place] = static_cast<int32_t>(inverse ? __umulhi(i, inverse) : i);
            } else if (i < end) {
                slot[i] = -1;
            }
            __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();
    }
}

// ---- the weighted sum

// out[t] = base[t] + sum over j of weight[t, j] * rows[slot[t, j]], in the order of j, float32 in registers, one rounding.  A wave owns 64 * N columns of a token: whole lines of every row, each read
// once, past the caches.  HBM bounds it: 16384 tokens of four rows of 4096 columns and a base, bf16, 805 MB, 136 us, 5.9 TB/s.
// Where widths or addresses are no whole pieces of 16 bytes, a column to a lane: loads of two or four bytes bound it then.  The same with 4095 columns 481 us (1.7 TB/s), in float32 344 against 274.
template <typename T> struct Loaded;
template <> struct Loaded<bf16_t> { typedef u32x4 type; static constexpr int N = 8; };
template <> struct Loaded<float> { typedef f32x4 type; static constexpr int N = 4; };

template <typename T, int N> __device__ __forceinline__ void load_values(const T* p, float (&v)[N]) {
    if constexpr (N == 1) {
        v[0] = as_float<T>(*p);
    } else if constexpr (sizeof(T) == 2) {
        const u32x4 r = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __uint_as_float((e & 1) ? r[e / 2] & 0xffff0000u : r[e / 2] << 16);
    } else {
#pragma unroll
        for (int q = 0; q < N / 4; ++q) {
            const f32x4 r = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p) + q);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * q + e] = r[e];
        }
    }
}
template <typename T, int N> __device__ __forceinline__ void store_values(T* p, const float (&v)[N]) {
    if constexpr (N == 1) {
        if constexpr (sizeof(T) == 2) *p = f32_to_bf16(v[0]); else *p = v[0];
    } else if constexpr (sizeof(T) == 2) {
        u32x4 r;
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = static_cast<unsigned>(f32_to_bf16(v[2 * e])) | static_cast<unsigned>(f32_to_bf16(v[2 * e + 1])) << 16;
        __builtin_nontemporal_store(r, reinterpret_cast<u32x4*>(p));
    } else {
#pragma unroll
        for (int q = 0; q < N / 4; ++q) __builtin_nontemporal_store(f32x4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]}, reinterpret_cast<f32x4*>(p) + q);
    }
}
constexpr int kSumAhead = 4;                                               // rows whose loads are in flight together
template <typename TR, typename TO, int N>
__global__ void __launch_bounds__(kThreads)
combine_kernel(const TR* __restrict__ rows, int64_t n_rows, const int32_t* __restrict__ slot, const float* __restrict__ weight, const TO* base, int64_t n_tokens, int top_k, int cols, int parts,
               TO* out) {
    const int64_t units = n_tokens * parts, stride = static_cast<int64_t>(gridDim.x) * (kThreads / 64);
    for (int64_t unit = static_cast<int64_t>(blockIdx.x) * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); unit < units; unit += stride) {
        const int64_t token = unit / parts;
        const int col = (static_cast<int>(unit - token * parts) * 64 + static_cast<int>(threadIdx.x & 63)) * N;
        if (col >= cols) continue;
        float sum[N];
        if (base) load_values<TO, N>(base + token * cols + col, sum);
        else
#pragma unroll
            for (int e = 0; e < N; ++e) sum[e] = 0.f;
        for (int j0 = 0; j0 < top_k; j0 += kSumAhead) {
            float v[kSumAhead][N];
            int64_t at[kSumAhead];
            float w[kSumAhead];
#pragma unroll
            for (int j = 0; j < kSumAhead; ++j) {
                at[j] = j0 + j < top_k ? slot[token * top_k + j0 + j] : -1;
                w[j] = !weight ? 1.f : j0 + j < top_k ? weight[token * top_k + j0 + j] : 0.f;
                if (at[j] >= n_rows) at[j] = -1;
            }
#pragma unroll
            for (int j = 0; j < kSumAhead; ++j) if (at[j] >= 0) load_values<TR, N>(rows + at[j] * cols + col, v[j]);
#pragma unroll
            for (int j = 0; j < kSumAhead; ++j)
                if (at[j] >= 0)
#pragma unroll
                    for (int e = 0; e < N; ++e) sum[e] = __builtin_fmaf(w[j], v[j][e], sum[e]);
        }
        store_values<TO, N>(out + token * cols + col, sum);
    }
}

template <typename TR, typename TO, int N>
int launch_combine(regione_ctx* ctx, const void* rows, int64_t n_rows, const int32_t* slot, const float* weight, const void* base, int64_t n_tokens, int top_k, int cols, void* out) {
    const int parts = (cols + 64 * N - 1) / (64 * N);
    int64_t blocks = (n_tokens * parts + kThreads / 64 - 1) / (kThreads / 64);
    if (blocks > (1 << 20)) blocks = 1 << 20;
    hipLaunchKernelGGL((combine_kernel<TR, TO, N>), dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, ctx->stream, static_cast<const TR*>(rows), n_rows, slot, weight,
                       static_cast<const TO*>(base), n_tokens, top_k, cols, parts, static_cast<TO*>(out));
    RG_LAUNCH_CHECK();
    return REGIONE_OK;
}
template <typename TR, typename TO>
int launch_combine(regione_ctx* ctx, const void* rows, int64_t n_rows, const int32_t* slot, const float* weight, const void* base, int64_t n_tokens, int top_k, int cols, void* out) {
    constexpr int N = sizeof(TR) == 2 || sizeof(TO) == 2 ? 8 : 4;          // 16 bytes of the narrower type
    if (cols % N == 0 && rg_aligned16(rows) && rg_aligned16(base) && rg_aligned16(out)) return launch_combine<TR, TO, N>(ctx, rows, n_rows, slot, weight, base, n_tokens, top_k, cols, out);
    return launch_combine<TR, TO, 1>(ctx, rows, n_rows, slot, weight, base, n_tokens, top_k, cols, out);
}

template <int AHEAD>
int launch_sort(regione_ctx* ctx, const int32_t* expert, int64_t n, int n_experts, int top_k, int32_t* offsets, int32_t* row_token, int32_t* slot) {
    constexpr int64_t PART = kSortThreads * AHEAD;
    const int64_t parts = (n + PART - 1) / PART, per_chunk = (parts + kMostChunks - 1) / kMostChunks * PART, chunks = n > PART ? (n + per_chunk - 1) / per_chunk : 1;
    if (chunks > 1 && static_cast<size_t>(chunks) * n_experts * sizeof(int32_t) > ctx->gemm_part_bytes)
        RG_FAIL(REGIONE_ERR_WORKSPACE, "expert_slots: %lld pairs need more workspace than the context has", (long long)n);
    int bits = 0;
    while ((1 << bits) < n_experts) ++bits;
    // i / top_k = i * inverse / 2^32 rounded down, as i (below 2^24) times what the inverse is too large by (less than top_k, 2^-32) stays below 1 / top_k
    const unsigned inverse = top_k == 1 ? 0u : static_cast<unsigned>((0x100000000ull + top_k - 1) / top_k);
    int32_t* counts = chunks > 1 ? reinterpret_cast<int32_t*>(ctx->gemm_part) : nullptr;
    if (counts) {
        hipLaunchKernelGGL((count_pairs_kernel<AHEAD>), dim3(static_cast<unsigned>(chunks)), dim3(kSortThreads), 0, ctx->stream, expert, n, per_chunk, n_experts, counts);
        RG_LAUNCH_CHECK();
    }
    size_t lds = (static_cast<size_t>(kSortWaves) * n_experts + kSortWaves) * sizeof(int32_t);
    if (counts && lds < 2 * kSortThreads * sizeof(int32_t)) lds = 2 * kSortThreads * sizeof(int32_t);
    static std::atomic<uint64_t> granted{0};
    if (lds > 65536)
        if (int rc = rg_grant_lds(ctx, reinterpret_cast<const void*>(place_pairs_kernel<AHEAD>), granted, (static_cast<size_t>(kSortWaves) * kMostExperts + kSortWaves) * sizeof(int32_t))) return rc;
    hipLaunchKernelGGL((place_pairs_kernel<AHEAD>), dim3(static_cast<unsigned>(chunks)), dim3(kSortThreads), lds, ctx->stream, expert, n, per_chunk, n_experts, bits, inverse, counts, offsets, row_token, slot);
    RG_LAUNCH_CHECK();
    return REGIONE_OK;
}

}  // namespace

extern "C" int regione_expert_route(regione_ctx* ctx, const void* logits, int32_t dtype, const float* bias_opt, const uint8_t* mask_opt, int64_t n_tokens, int32_t n_experts, int32_t score,
                                    int32_t n_groups, int32_t top_groups, int32_t group_best, int32_t top_k, int32_t renormalise, float scale, int32_t* expert, float* weight) {
    if (!ctx) RG_FAIL(REGIONE_ERR_INVALID_ARG, "expert_route: null context");
    if (dtype != REGIONE_BF16 && dtype != REGIONE_FP32) RG_FAIL(REGIONE_ERR_INVALID_ARG, "expert_route: bad dtype %d", dtype);
    if (score != REGIONE_SCORE_SOFTMAX && score != REGIONE_SCORE_SIGMOID) RG_FAIL(REGIONE_ERR_INVALID_ARG, "expert_route: bad score %d", score);
    if (n_tokens < 0 || n_experts <= 0 || top_k <= 0 || n_groups <= 0) RG_FAIL(REGIONE_ERR_INVALID_ARG, "expert_route: n_tokens=%lld n_experts=%d top_k=%d n_groups=%d", (long long)n_tokens, n_experts, top_k, n_groups);
    if (group_best != 1 && group_best != 2) RG_FAIL(REGIONE_ERR_INVALID_ARG, "expert_route: group_best=%d (1 or 2)", group_best);
    if (!isfinite(scale)) RG_FAIL(REGIONE_ERR_INVALID_ARG, "expert_route: scale is not finite");
    if (n_experts > kMostExperts || top_k > kMostChosen || n_groups > kMostGroups || n_tokens * top_k > kMostPairs || n_tokens > kMostPairs)
        RG_FAIL(REGIONE_ERR_UNSUPPORTED, "expert_route: %lld tokens, %d experts (at most %d), top_k=%d (%d), %d groups (%d); at most 2^24 choices", (long long)n_tokens, n_experts, kMostExperts, top_k, kMostChosen, n_groups, kMostGroups);
    if (n_experts % n_groups || top_groups < 1 || top_groups > n_groups || top_k > top_groups * (n_experts / n_groups))
        RG_FAIL(REGIONE_ERR_BAD_SHAPE, "expert_route: %d of %d experts in %d of %d groups", top_k, n_experts, top_groups, n_groups);
    if (n_tokens == 0) return REGIONE_OK;
    if (!logits || !expert || !weight) RG_FAIL(REGIONE_ERR_INVALID_ARG, "expert_route: null tensor");
    if (!rg_aligned16(logits)) RG_FAIL(REGIONE_ERR_INVALID_ARG, "expert_route: logits must be 16-byte aligned");
    RouteCall c = {logits, bias_opt, mask_opt, expert, weight, n_tokens, n_experts, n_groups, top_groups, group_best, top_k, 0, 0, score == REGIONE_SCORE_SIGMOID, renormalise != 0, 0, scale};
    const bool scored = bias_opt || n_groups > 1;
    ProfScope prof(ctx, REGIONE_PROF_ROWS);
    return dtype == REGIONE_FP32 ? launch_route<float>(ctx, c, scored) : launch_route<bf16_t>(ctx, c, scored);
}

extern "C" int regione_expert_slots(regione_ctx* ctx, const int32_t* expert, int64_t n_tokens, int32_t top_k, int32_t n_experts, int32_t* group_offsets, int32_t* row_token, int32_t* slot) {
    if (!ctx) RG_FAIL(REGIONE_ERR_INVALID_ARG, "expert_slots: null context");
    if (n_tokens < 0 || top_k <= 0 || n_experts <= 0) RG_FAIL(REGIONE_ERR_INVALID_ARG, "expert_slots: n_tokens=%lld top_k=%d n_experts=%d", (long long)n_tokens, top_k, n_experts);
    if (n_experts > kMostExperts || top_k > kMostChosen || n_tokens > kMostPairs || n_tokens * top_k > kMostPairs)
        RG_FAIL(REGIONE_ERR_UNSUPPORTED, "expert_slots: %lld x %d pairs (at most 2^24, %d per token), %d experts (at most %d)", (long long)n_tokens, top_k, kMostChosen, n_experts, kMostExperts);
    if (!group_offsets || (n_tokens > 0 && (!expert || !row_token || !slot))) RG_FAIL(REGIONE_ERR_INVALID_ARG, "expert_slots: null tensor");
    const int64_t n = n_tokens * top_k;
    ProfScope prof(ctx, REGIONE_PROF_ROWS);
    if (n <= 2048 || (n > 4096 && n <= 262144)) return launch_sort<2>(ctx, expert, n, n_experts, top_k, group_offsets, row_token, slot);
    return launch_sort<4>(ctx, expert, n, n_experts, top_k, group_offsets, row_token, slot);
}

extern "C" int regione_expert_combine(regione_ctx* ctx, const void* rows, int32_t rows_dtype, int64_t n_rows, const int32_t* slot, const float* weight_opt, const void* base_opt,
                                      int64_t n_tokens, int32_t top_k, int32_t cols, int32_t out_dtype, void* out) {
    if (!ctx) RG_FAIL(REGIONE_ERR_INVALID_ARG, "expert_combine: null context");
    if ((rows_dtype != REGIONE_BF16 && rows_dtype != REGIONE_FP32) || (out_dtype != REGIONE_BF16 && out_dtype != REGIONE_FP32))
        RG_FAIL(REGIONE_ERR_INVALID_ARG, "expert_combine: bad dtype %d or %d", rows_dtype, out_dtype);
    if (n_tokens < 0 || n_rows < 0 || top_k <= 0 || cols <= 0) RG_FAIL(REGIONE_ERR_INVALID_ARG, "expert_combine: n_tokens=%lld n_rows=%lld top_k=%d cols=%d", (long long)n_tokens, (long long)n_rows, top_k, cols);
    if (top_k > kMostChosen || n_tokens > kMostPairs || n_tokens * top_k > kMostPairs || cols > (1 << 24))
        RG_FAIL(REGIONE_ERR_UNSUPPORTED, "expert_combine: %lld x %d pairs (at most 2^24, %d per token) of %d columns (at most 2^24)", (long long)n_tokens, top_k, kMostChosen, cols);
    if (n_tokens == 0) return REGIONE_OK;
    if (!slot || !out || (n_rows > 0 && !rows)) RG_FAIL(REGIONE_ERR_INVALID_ARG, "expert_combine: null tensor");
    ProfScope prof(ctx, REGIONE_PROF_ROWS);
    if (rows_dtype == REGIONE_FP32)
        return out_dtype == REGIONE_FP32 ? launch_combine<float, float>(ctx, rows, n_rows, slot, weight_opt, base_opt, n_tokens, top_k, cols, out)
                                         : launch_combine<float, bf16_t>(ctx, rows, n_rows, slot, weight_opt, base_opt, n_tokens, top_k, cols, out);
    return out_dtype == REGIONE_FP32 ? launch_combine<bf16_t, float>(ctx, rows, n_rows, slot, weight_opt, base_opt, n_tokens, top_k, cols, out)
                                     : launch_combine<bf16_t, bf16_t>(ctx, rows, n_rows, slot, weight_opt, base_opt, n_tokens, top_k, cols, out);
}
