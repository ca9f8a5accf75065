// What surrounds products over groups of rows (regione_linear_grouped) where a router forms the groups: the choice of experts, the sort of the chosen (token, expert) pairs
// by expert, and the weighted sum of the experts' rows back at their tokens.
#include "common.h"
#include <math.h>
#include <type_traits>

namespace {

constexpr int kThreads = 256;
constexpr int kMostExperts = 1024, kMostChosen = 32, kMostGroups = 64;
constexpr int64_t kMostPairs = int64_t{1} << 24;             // rows that a grouped product takes

typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;

// ---- choice of experts

struct RouteCall {
    const void* logits; const float* bias; const uint8_t* mask; int32_t* expert; float* weight;
    int64_t n_tokens; int n_experts, n_groups, top_groups, group_best, top_k, group_lanes;
    int sigmoid, renormalise, whole; float scale;            // whole: every lane's experts exist and lie at a multiple of their own size
};

// Lane exchange within LPT lanes (16: a DPP row; 64: the wave): v of the lane XOR 1, 2, 4, 8 by DPP, further ones through the LDS crossbar.
template <int X> __device__ __forceinline__ int lane_xor(int v) {
    if constexpr (X == 1) return __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xf, 0xf, true);              // quad_perm 1 0 3 2
    else if constexpr (X == 2) return __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xf, 0xf, true);         // quad_perm 2 3 0 1
    else if constexpr (X == 4) return __builtin_amdgcn_ds_swizzle(v, 0x101f);
    else if constexpr (X == 8) return __builtin_amdgcn_update_dpp(0, v, 0x128, 0xf, 0xf, true);        // row_ror:8
    else if constexpr (X == 16) return __builtin_amdgcn_ds_swizzle(v, 0x401f);
    else return __builtin_amdgcn_ds_bpermute(((threadIdx.x & 63) ^ 32) * 4, v);
}
template <int X> __device__ __forceinline__ float lane_xor(float v) { return __int_as_float(lane_xor<X>(__float_as_int(v))); }
template <int X> __device__ __forceinline__ double lane_xor(double v) { return __hiloint2double(lane_xor<X>(__double2hiint(v)), lane_xor<X>(__double2loint(v))); }
template <int X, int LPT, typename V, typename F> __device__ __forceinline__ V over_lanes(V v, F f) {
    if constexpr (X < LPT) return over_lanes<2 * X, LPT>(f(v, lane_xor<X>(v)), f);
    else return v;
}
__device__ __forceinline__ float bigger(float a, float b) { return __builtin_fmaxf(a, b); }
__device__ __forceinline__ double bigger(double a, double b) { return __builtin_fmax(a, b); }
template <int LPT, typename V> __device__ __forceinline__ V lanes_max(V v) { return over_lanes<1, LPT>(v, [](V a, V b) { return bigger(a, b); }); }
template <int LPT, typename V> __device__ __forceinline__ V lanes_sum(V v) { return over_lanes<1, LPT>(v, [](V a, V b) { return a + b; }); }

// Two largest values of the lanes of a group (1 to LPT lanes).
template <int X, int LPT> __device__ __forceinline__ void best_two(double& a, double& b, int lanes) {
    if constexpr (X < LPT) {
        const double oa = lane_xor<X>(a), ob = lane_xor<X>(b);
        if (X < lanes) {
            b = bigger(__builtin_fmin(a, oa), bigger(b, ob));
            a = bigger(a, oa);
        }
        best_two<2 * X, LPT>(a, b, lanes);
    }
}

template <typename T> __device__ __forceinline__ float as_float(T v);
template <> __device__ __forceinline__ float as_float<float>(float v) { return v; }
template <> __device__ __forceinline__ float as_float<bf16_t>(bf16_t v) { return bf16_to_f32(v); }

// LPT lanes choose the experts of a token.  A group has LPT / (n_groups rounded up to a power of two) lanes of EPL experts each, in order, so that among equal values the lowest lane and
// then its lowest place hold the lowest expert.
// Which expert is chosen is decided in 64 bits wherever a score takes part (EXACT: with a bias, or sums of two scores over a group): in 32 bits the rounding of the exponential would
// decide between experts that differ by less, and another order of the same operations would choose others.  Without either the scores lie in the order of the logits.
template <typename T, int LPT, int EPL, bool EXACT>
__global__ void __launch_bounds__(kThreads)
route_kernel(RouteCall c) {
    typedef typename std::conditional<EXACT, double, float>::type V;
    constexpr V NONE = static_cast<V>(-INFINITY);
    const int lane = threadIdx.x & 63, l = lane & (LPT - 1);
    const int64_t token = (static_cast<int64_t>(blockIdx.x) * (kThreads / 64) + (threadIdx.x >> 6)) * (64 / LPT) + lane / LPT;
    if (token - lane / LPT >= c.n_tokens) return;                          // (the whole wave)
    const bool there = token < c.n_tokens, routed = there && (!c.mask || c.mask[token] != 0);
    const int group_lanes = c.group_lanes, group = l / group_lanes, per = c.n_experts / c.n_groups, first = (l & (group_lanes - 1)) * EPL;
    const int expert0 = group * per + first;                               // of this lane
    int mine = group < c.n_groups ? per - first : 0;                       // its experts
    mine = mine < 0 ? 0 : (mine < EPL ? mine : EPL);

    float logit[EPL];
    V value[EPL];
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
    // NaN is no score at all; what overflows counts as the largest value there is
#pragma unroll
    for (int i = 0; i < EPL; ++i) logit[i] = logit[i] > -INFINITY ? __builtin_fminf(logit[i], 3.402823466e38f) : -INFINITY;

    float top = logit[0];
#pragma unroll
    for (int i = 1; i < EPL; ++i) top = bigger(top, logit[i]);
    top = lanes_max<LPT>(top);
    double all = 0.0;                                                      // sum of the softmax's exponentials
    if constexpr (EXACT) {
        double e[EPL];
#pragma unroll
        for (int i = 0; i < EPL; ++i) e[i] = logit[i] == -INFINITY ? 0.0 : exp(c.sigmoid ? -static_cast<double>(logit[i]) : static_cast<double>(logit[i]) - static_cast<double>(top));
        if (!c.sigmoid) {
#pragma unroll
            for (int i = 0; i < EPL; ++i) all += e[i];
            all = lanes_sum<LPT>(all);
        }
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
            double v = c.sigmoid ? 1.0 / (1.0 + e[i]) : e[i] / all;
            if (c.bias && i < mine) v += static_cast<double>(c.bias[expert0 + i]);
            value[i] = logit[i] > -INFINITY && v > NONE ? v : NONE;        // (a bias of NaN or -infinity takes its expert out)
        }
    } else {
#pragma unroll
        for (int i = 0; i < EPL; ++i) value[i] = logit[i];
        if (!c.sigmoid && !c.renormalise) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < EPL; ++i) sum += logit[i] == -INFINITY ? 0.f : expf(logit[i] - top);
            all = lanes_sum<LPT>(sum);
        }
    }

    if (EXACT && c.n_groups > 1) {
        // A group's place is the number of groups that come before it: those with more, and those with as much and a lower number.
        double a = NONE, b = NONE;
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
            const double v = static_cast<double>(value[i]);
            b = bigger(b, __builtin_fmin(a, v));
            a = bigger(a, v);
        }
        best_two<1, LPT>(a, b, group_lanes);
        const double sum = c.group_best == 2 && b > NONE ? a + b : a;
        int before = 0;
        for (int h = 0; h < c.n_groups; ++h) {
            const int from = ((lane & ~(LPT - 1)) + h * group_lanes) * 4;
            const double other = __hiloint2double(__builtin_amdgcn_ds_bpermute(from, __double2hiint(sum)), __builtin_amdgcn_ds_bpermute(from, __double2loint(sum)));
            before += other > sum || (other == sum && h < group) ? 1 : 0;
        }
        if (before >= c.top_groups)
#pragma unroll
            for (int i = 0; i < EPL; ++i) value[i] = NONE;
        else if (!c.bias)
#pragma unroll
            for (int i = 0; i < EPL; ++i) value[i] = static_cast<V>(logit[i]);
    }

    // lane j of the token's ends up with its choice j
    int chosen = -1;
    float chosen_logit = 0.f;
    for (int j = 0; j < c.top_k; ++j) {
        V best = value[0];
#pragma unroll
        for (int i = 1; i < EPL; ++i) best = bigger(best, value[i]);
        const V most = lanes_max<LPT>(best);
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
    // Weights, in 64 bits: once per wave.  Renormalised softmax weights do not depend on the other experts, nor on how far below them the chosen ones lie.
    const bool has = routed && chosen >= 0;
    double w = 0.0;
    if (c.sigmoid) {
        if (has) w = 1.0 / (1.0 + exp(-static_cast<double>(chosen_logit)));
    } else {
        const float from = c.renormalise ? lanes_max<LPT>(has ? chosen_logit : -INFINITY) : top;
        if (has) w = exp(static_cast<double>(chosen_logit) - static_cast<double>(from));
        if (has && !c.renormalise) w /= all;
    }
    if (c.renormalise) {
        const double sum = lanes_sum<LPT>(w);
        w = sum > 0.0 ? w / sum : 0.0;
    }
    if (there && l < c.top_k) {
        c.expert[token * c.top_k + l] = has ? chosen : -1;
        c.weight[token * c.top_k + l] = has ? static_cast<float>(w * static_cast<double>(c.scale)) : 0.f;
    }
}

template <typename T, int LPT, int EPL>
int launch_route(regione_ctx* ctx, RouteCall& c, bool exact) {
    c.group_lanes = LPT;
    for (int g = 1; g < c.n_groups; g *= 2) c.group_lanes /= 2;
    c.whole = c.n_experts / c.n_groups == c.group_lanes * EPL;
    const int64_t tokens_per = (kThreads / 64) * (64 / LPT), blocks = (c.n_tokens + tokens_per - 1) / tokens_per;
    if (exact) hipLaunchKernelGGL((route_kernel<T, LPT, EPL, true>), dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, ctx->stream, c);
    else hipLaunchKernelGGL((route_kernel<T, LPT, EPL, false>), dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, ctx->stream, c);
    RG_LAUNCH_CHECK();
    return REGIONE_OK;
}
template <typename T>
int launch_route(regione_ctx* ctx, RouteCall& c, bool exact) {
    int lanes = 64;
    for (int g = 1; g < c.n_groups; g *= 2) lanes /= 2;
    const int need = (c.n_experts / c.n_groups + lanes - 1) / lanes;
    if (need <= 1) return launch_route<T, 64, 1>(ctx, c, exact);
    if (need <= 2) return launch_route<T, 64, 2>(ctx, c, exact);
    if (need <= 4) return launch_route<T, 64, 4>(ctx, c, exact);
    if (need <= 8) return launch_route<T, 64, 8>(ctx, c, exact);
    if (need <= 16) return launch_route<T, 64, 16>(ctx, c, exact);
    return launch_route<T, 64, 32>(ctx, c, exact);
}

// ---- the sort by expert

// A stable counting sort.  The pairs are cut into chunks of whole rounds of kRound; every workgroup counts its chunk, and a second launch places it behind the chunks before: the waves of
// a workgroup own consecutive parts of the chunk, so that a pair's place is its expert's first row + the expert's pairs of earlier chunks, of earlier waves, and of earlier pairs of its wave.
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64, kMostChunks = 256, kSortLeast = 512;      // kSortLeast: pairs per wave of a chunk at least, where there are several

__device__ __forceinline__ int pair_expert(const int32_t* expert, int64_t at, int64_t end, int n_experts) {
    if (at >= end) return -1;
    const int e = expert[at];
    return e >= 0 && e < n_experts ? e : -1;
}
__global__ void __launch_bounds__(kSortThreads)
count_pairs_kernel(const int32_t* __restrict__ expert, int64_t n, int64_t per_chunk, int n_experts, int32_t* __restrict__ counts) {
    __shared__ int32_t count[kMostExperts];
    for (int e = threadIdx.x; e < n_experts; e += kSortThreads) count[e] = 0;
    __syncthreads();
    const int64_t begin = static_cast<int64_t>(blockIdx.x) * per_chunk, end = begin + per_chunk < n ? begin + per_chunk : n;
    for (int64_t i = begin + threadIdx.x; i < end; i += kSortThreads) {
        const int e = pair_expert(expert, i, end, n_experts);
        if (e >= 0) atomicAdd(&count[e], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < n_experts; e += kSortThreads) counts[static_cast<int64_t>(blockIdx.x) * n_experts + e] = count[e];
}
// counts: [chunks][n_experts], or null where there is one chunk
__global__ void __launch_bounds__(kSortThreads)
place_pairs_kernel(const int32_t* __restrict__ expert, int64_t n, int64_t per_chunk, int n_experts, int bits, int top_k, const int32_t* __restrict__ counts,
                   int32_t* __restrict__ offsets, int32_t* __restrict__ row_token, int32_t* __restrict__ slot) {
    extern __shared__ int32_t lds[];                                       // [kSortWaves][n_experts], then [kSortWaves]
    int32_t* const sums = lds + kSortWaves * n_experts;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t begin = static_cast<int64_t>(blockIdx.x) * per_chunk, end = begin + per_chunk < n ? begin + per_chunk : n;
    const int64_t per_wave = (per_chunk / kSortWaves + 63) / 64 * 64;
    const int64_t w0 = begin + wave * per_wave, w1 = w0 + per_wave < end ? w0 + per_wave : end;
    for (int i = threadIdx.x; i < kSortWaves * n_experts; i += kSortThreads) lds[i] = 0;
    __syncthreads();
    for (int64_t i = w0 + lane; i < w1; i += 64) {
        const int e = pair_expert(expert, i, w1, n_experts);
        if (e >= 0) atomicAdd(&lds[wave * n_experts + e], 1);
    }
    // this thread's expert: pairs of the chunks before, and all
    const int e = threadIdx.x;
    int before = 0, all = 0;
    if (counts && e < n_experts)
        for (unsigned c = 0; c < gridDim.x; ++c) {
            const int v = counts[static_cast<int64_t>(c) * n_experts + e];
            before += c < blockIdx.x ? v : 0;
            all += v;
        }
    __syncthreads();
    if (!counts && e < n_experts) for (int w = 0; w < kSortWaves; ++w) all += lds[w * n_experts + e];
    int upto = all;                                                        // inclusive sums over the experts
    for (int d = 1; d < 64; d *= 2) {
        const int v = __shfl_up(upto, d);
        upto += lane >= d ? v : 0;
    }
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    for (int w = 0; w < wave; ++w) upto += sums[w];
    if (e < n_experts) {
        if (blockIdx.x == 0) {
            offsets[e + 1] = upto;
            if (e == 0) offsets[0] = 0;
        }
        int at = upto - all + before;
        for (int w = 0; w < kSortWaves; ++w) {
            const int v = lds[w * n_experts + e];
            lds[w * n_experts + e] = at;
            at += v;
        }
    }
    __syncthreads();
    for (int64_t i0 = w0; i0 < w1; i0 += 64) {
        const int64_t i = i0 + lane;
        const int id = pair_expert(expert, i, w1, n_experts);
        uint64_t same = __ballot(id >= 0);                                 // lanes with this lane's expert
        for (int b = 0; b < bits; ++b) {
            const bool set = (id >> b) & 1;
            const uint64_t with = __ballot(set);
            same &= set ? with : ~with;
        }
        const int rank = __builtin_popcountll(same & ((uint64_t{1} << lane) - 1));
        if (id >= 0) {
            volatile int32_t* const next = &lds[wave * n_experts + id];           // (the other lanes' doing)
            const int place = *next + rank;
            __builtin_amdgcn_wave_barrier();
            if (rank == 0) *next = place + __builtin_popcountll(same);
            slot[i] = place;
            row_token[place] = static_cast<int32_t>(i / top_k);
        } else if (i < w1) {
            slot[i] = -1;
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// ---- the weighted sum

// out[t] = base[t] + sum over j of weight[t, j] * rows[slot[t, j]], in the order of j, float32 in registers, one rounding.  A wave owns WIDE * 64 columns of a token.
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
    RouteCall c = {logits, bias_opt, mask_opt, expert, weight, n_tokens, n_experts, n_groups, top_groups, group_best, top_k, 0, score == REGIONE_SCORE_SIGMOID, renormalise != 0, 0, scale};
    const bool exact = bias_opt || n_groups > 1;
    ProfScope prof(ctx, REGIONE_PROF_ROWS);
    return dtype == REGIONE_FP32 ? launch_route<float>(ctx, c, exact) : launch_route<bf16_t>(ctx, c, exact);
}

extern "C" int regione_expert_slots(regione_ctx* ctx, const int32_t* expert, int64_t n_tokens, int32_t top_k, int32_t n_experts, int32_t* group_offsets, int32_t* row_token, int32_t* slot) {
    if (!ctx) RG_FAIL(REGIONE_ERR_INVALID_ARG, "expert_slots: null context");
    if (n_tokens < 0 || top_k <= 0 || n_experts <= 0) RG_FAIL(REGIONE_ERR_INVALID_ARG, "expert_slots: n_tokens=%lld top_k=%d n_experts=%d", (long long)n_tokens, top_k, n_experts);
    if (n_experts > kMostExperts || top_k > kMostChosen || n_tokens > kMostPairs || n_tokens * top_k > kMostPairs)
        RG_FAIL(REGIONE_ERR_UNSUPPORTED, "expert_slots: %lld x %d pairs (at most 2^24, %d per token), %d experts (at most %d)", (long long)n_tokens, top_k, kMostChosen, n_experts, kMostExperts);
    if (!group_offsets || (n_tokens > 0 && (!expert || !row_token || !slot))) RG_FAIL(REGIONE_ERR_INVALID_ARG, "expert_slots: null tensor");
    const int64_t n = n_tokens * top_k;
    int64_t chunks = (n + kSortWaves * kSortLeast - 1) / (kSortWaves * kSortLeast);
    chunks = chunks < 1 ? 1 : (chunks < kMostChunks ? chunks : kMostChunks);
    const int64_t round = kSortThreads, per_chunk = ((n + chunks - 1) / chunks + round - 1) / round * round;
    chunks = n > 0 ? (n + per_chunk - 1) / per_chunk : 1;
    if (chunks > 1 && static_cast<size_t>(chunks) * n_experts * sizeof(int32_t) > ctx->gemm_part_bytes)
        RG_FAIL(REGIONE_ERR_WORKSPACE, "expert_slots: %lld pairs need more workspace than the context has", (long long)n);
    int bits = 0;
    while ((1 << bits) < n_experts) ++bits;
    ProfScope prof(ctx, REGIONE_PROF_ROWS);
    int32_t* counts = chunks > 1 ? reinterpret_cast<int32_t*>(ctx->gemm_part) : nullptr;
    if (counts) {
        hipLaunchKernelGGL(count_pairs_kernel, dim3(static_cast<unsigned>(chunks)), dim3(kSortThreads), 0, ctx->stream, expert, n, per_chunk, n_experts, counts);
        RG_LAUNCH_CHECK();
    }
    const size_t lds = (static_cast<size_t>(kSortWaves) * n_experts + kSortWaves) * sizeof(int32_t);
    static std::atomic<uint64_t> granted{0};
    if (lds > 65536)
        if (int rc = rg_grant_lds(ctx, reinterpret_cast<const void*>(place_pairs_kernel), granted, (static_cast<size_t>(kSortWaves) * kMostExperts + kSortWaves) * sizeof(int32_t))) return rc;
    hipLaunchKernelGGL(place_pairs_kernel, dim3(static_cast<unsigned>(chunks)), dim3(kSortThreads), lds, ctx->stream, expert, n, per_chunk, n_experts, bits, top_k, counts, group_offsets, row_token, slot);
    RG_LAUNCH_CHECK();
    return REGIONE_OK;
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
