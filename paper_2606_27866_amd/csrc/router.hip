// Routing of tokens to experts (gfx950): scores, a bias that only the choice
// sees, groups, the top k, their weights, the tables of rows grouped by expert,
// and the logits' gradient.
//
//   s = softmax(l) or sigmoid(l)      c = s + bias
//   a group's score: the sum of its best one or two c; the best groups stay
//   chosen: the k largest c of the groups that stay, ties to the lower id
//   w = scale s / (normalize ? sum of the chosen s : 1)
//
// An expert whose logit (or bias) is -inf is masked: it is never chosen.  Where
// no expert is left a slot gets the id -1, the weight 0 and no row, so that a
// token of nothing but -inf goes nowhere.
//
// The choice hangs on which of two scores is larger, so it is made on exact
// values: on the logits where the scores are as they are (both functions keep
// their order), else on scores in 64 bits.  Weights are in fp32, the normalised
// ones from differences of log scores, which neither overflow nor vanish.
//
//   route_kernel         one wave per token; a histogram for each few tokens
//   route_tables_kernel  every chunk of tokens sums the histograms before its own
//                        (and all of them, for the experts' starts), then places
//                        its tokens: stable, and no atomic's order is in a result
//   both in one workgroup for few tokens
//
// Latency and instructions, not bytes, bound these launches.  So scores are first
// taken in 32 bits: where the chosen ones and the best of the others (groups too)
// are further apart than those can be wrong, the order is the exact one, and only
// the other tokens (1 in 1000 of usual logits) are routed again in 64 bits.
// One token of 64 experts 4.7 us; 8191 tokens of 256 experts in groups 16.6 us and 8.2
// for the tables (all in 64 bits 82 together); 65536 of 60 experts 38 us.
#include <algorithm>
#include <cmath>

#include "error.h"
#include "flexmoe.h"
#include "rows.h"

using namespace flexmoe;

namespace {

constexpr int kWaves = 16, kThreads = 64 * kWaves;
// Chunks of tokens, at most: workgroups of route_tables_kernel, which read all histograms.  8191 tokens of 256 experts in
// groups, all of a call, 30.3, 29.1, 29.1 and 29.2 us with 32, 64, 128 and 256; 65536 tokens of 60 experts 44.9, 40.1, 37.8 and
// 36.9, of 256 experts with 64, 128 and 256 68.4, 63.9 and 62.5.
constexpr int kChunks = 128;
// Tokens of a workgroup of route_kernel, at most; their counts are bytes.
constexpr int kMostCounted = 128;
// Tokens up to which one workgroup does it all, a wave each: 4, 8 and 16 tokens of 64 experts 4.9, 5.1 and 6.3 us, in two
// launches 7.7, 8.0 and 9.1.
constexpr int kOneWorkgroup = kWaves;
constexpr int kMaxGroups = 64;
constexpr int kQ = kMaxExperts / 64;

struct RouteArgs {
    const void* logits;
    const float* bias;
    int32_t *idx, *counts, *offsets, *perm, *pos;
    float* w;
    uint32_t* hist;  // [histograms][words]: a byte for each expert
    size_t ldl;
    int T, E, k, bf16, sigmoid, normalize, groups, top_groups, best;
    int counted, chunk;  // tokens of a histogram, and of a workgroup of the tables (a multiple)
    int first;           // histogram of a launch's first workgroup
    int words;
    float scale;
};

template <bool kBf16>
__device__ __forceinline__ float load1(const void* p, size_t i) {
    if constexpr (kBf16) return bf16_to_f32(reinterpret_cast<const bf16_t*>(p)[i]);
    else return reinterpret_cast<const float*>(p)[i];
}

// Order of scores as whole numbers: 0 masked, 1 NaN, then ascending (-0 as +0).
__device__ __forceinline__ uint64_t score_key(double c) {
    if (__builtin_isnan(c)) return 1;
    const uint64_t u = (uint64_t)__double_as_longlong(c == 0.0 ? 0.0 : c);
    if (u == 0xfff0000000000000ull) return 0;  // -inf
    return (u >> 63) ? ~u : (u | 0x8000000000000000ull);
}

__device__ __forceinline__ float log_sigmoid(float x) { return fminf(x, 0.f) - log1pf(expf(-fabsf(x))); }

struct RouteScratch {
    double c[kMaxExperts];  // scores in 64 bits, or the first half in 32
    float v[kMaxExperts];   // logits
};

// Order of values that are no NaN as whole numbers: -inf (masked) 0.
__device__ __forceinline__ uint32_t key32(float c) {
    const uint32_t u = __float_as_uint(c + 0.f);  // -0 + 0 = 0
    return c == -INFINITY ? 0u : (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float key32_value(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k); }

// Largest of the wave's keys, in every lane: upper halves first.
__device__ __forceinline__ uint64_t wave_max_key(uint64_t v) {
    const uint32_t hi = wave_max_u((uint32_t)(v >> 32));
    const uint32_t lo = wave_max_u((uint32_t)(v >> 32) == hi ? (uint32_t)v : 0u);
    return ((uint64_t)hi << 32) | lo;
}

// The score of a logit without its bias, in 64 bits; top and z: of the softmax.
__device__ __forceinline__ double exact_score(const RouteArgs& a, float v, double top, double z) {
    return a.sigmoid ? 1.0 / (1.0 + exp(-(double)v)) : exp((double)v - top) / z;
}

template <int NQ>
__device__ __forceinline__ double exact_sum(const float (&v)[NQ], float top) {
    double z = 0.0;
#pragma unroll
    for (int q = 0; q < NQ; ++q) z += v[q] == -INFINITY ? 0.0 : exp((double)v[q] - (double)top);
    return wave_total_d(z);
}

// The choice of one token by one wave, in 64 bits, from its logits v (expert lane NQ + q;
// -inf past E): lane j < k gets the j-th chosen expert (-1: none).
template <int NQ>
__device__ __forceinline__ int choose_exact(const RouteArgs& a, const float (&v)[NQ], int lane, RouteScratch& rs) {
    const bool by_score = a.bias || (a.groups > 1 && a.best > 1);  // scores decide, else logits
    double z = 1.0, c[NQ];
    float top = 0.f;
    if (by_score && !a.sigmoid) {
        top = v[0];
#pragma unroll
        for (int q = 1; q < NQ; ++q) top = fmaxf(top, v[q]);
        top = wave_max(top);
        z = exact_sum<NQ>(v, top);
    }
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        c[q] = v[q];
        if (by_score) {
            c[q] = exact_score(a, v[q], (double)top, z);
            if (a.bias) c[q] += (double)a.bias[min(lane * NQ + q, a.E - 1)];
            if (v[q] == -INFINITY) c[q] = -INFINITY;
        }
    }
    uint64_t kept = ~0ull;
    const int members = a.E / a.groups;
    if (a.groups > 1) {
#pragma unroll
        for (int q = 0; q < NQ; ++q) rs.c[lane * NQ + q] = c[q];
        __builtin_amdgcn_wave_barrier();
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
        uint64_t group = 0;
        if (lane < a.groups) {
            double c1 = -INFINITY, c2 = -INFINITY;
            uint64_t k1 = 0, k2 = 0;
            for (int i = 0, j = lane % members; i < members; ++i, j = j + 1 == members ? 0 : j + 1) {
                const double x = rs.c[lane * members + j];
                const uint64_t kx = score_key(x);
                if (kx > k1) k2 = k1, c2 = c1, k1 = kx, c1 = x;
                else if (kx > k2) k2 = kx, c2 = x;
            }
            group = k1 == 0 ? 0 : a.best > 1 && k2 != 0 ? score_key(c1 + c2) : k1;
        }
        __builtin_amdgcn_wave_barrier();
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
        kept = 0;
        for (int j = 0; j < a.top_groups; ++j) {
            const uint64_t m = wave_max_key(group);
            if (m == 0) break;
            const uint64_t all = __ballot(group == m), first = all & -all;
            kept |= first;
            if ((first >> lane) & 1) group = 0;
        }
    }
    uint64_t key[NQ];
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        const int e = lane * NQ + q;
        key[q] = a.groups == 1 || (e < a.E && ((kept >> (e / members)) & 1)) ? score_key(c[q]) : 0;
    }
    int my_id = -1;
    for (int j = 0; j < a.k; ++j) {
        uint64_t best = key[0];
        int at = lane * NQ;
#pragma unroll
        for (int q = 1; q < NQ; ++q)
            if (key[q] > best) best = key[q], at = lane * NQ + q;  // the lower place of equal ones
        const uint64_t m = wave_max_key(best);
        if (m == 0) break;
        const int from = __ffsll((unsigned long long)__ballot(best == m)) - 1;
        const int id = __builtin_amdgcn_readlane(at, from);
        if (lane == j) my_id = id;
#pragma unroll
        for (int q = 0; q < NQ; ++q)
            if (lane * NQ + q == id) key[q] = 0;
    }
    return my_id;
}

// What decides: the logits themselves, or scores, with a bias or in sums of a group's two best.
enum { kByLogits = 0, kBySigmoid = 1, kBySoftmax = 2 };

// Whether two scores of 32 bits, a >= b, may stand in another order than the exact
// ones.  A score s is off by so many units of 2^-24 of itself: softmax 16 (exp, a sum of 256,
// quotient), sigmoid 5 (exp, a sum, reciprocal), and |ln s| more, the size of the exponent
// that was rounded; with its bias and in a group's sum by one each of what they are.  That
// is below 26 and 15 from 2^-10 on, below 106 down to where fp32 ends.  `bias` is the sum of
// both values' largest possible biases, so that the scores are at most |a| + |b| + bias,
// and s |ln s| falls with s.
template <int kBy>
__device__ __forceinline__ bool too_near(float a, float b, float bias) {
    const float size = fabsf(a) + fabsf(b) + bias;
    return a - b <= (size < 0x1p-10f ? 128.f : kBy == kBySigmoid ? 15.f : 26.f) * 0x1p-24f * size + 0x1p-100f;
}

__device__ __forceinline__ float exp_fast(float x) { return __builtin_amdgcn_exp2f(x * 1.4426950408889634f); }
__device__ __forceinline__ float sigmoid_fast(float x) { return __builtin_amdgcn_rcpf(1.f + exp_fast(-x)); }

// The choice of one token, whose logits are in v (expert lane NQ + q; -inf past E), also
// in rs.v, from values of 32 bits; `unsure`: they do not tell.
template <int NQ, int kBy, bool kGroups>
__device__ __forceinline__ int choose_fast(const RouteArgs& a, const float (&v)[NQ], int lane, RouteScratch& rs, float top, bool& unsure) {
    float c[NQ], bias = 0.f;
    bool again = false;
    if constexpr (kBy == kByLogits) {
#pragma unroll
        for (int q = 0; q < NQ; ++q) c[q] = v[q], again |= __builtin_isnan(v[q]);
    } else {
        float z = 0.f;
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            if constexpr (kBy == kBySigmoid) c[q] = sigmoid_fast(v[q]);
            else z += c[q] = v[q] == -INFINITY ? 0.f : expf(v[q] - top);
        }
        if constexpr (kBy == kBySoftmax) {
            const float inv = 1.f / wave_total_f(z);
#pragma unroll
            for (int q = 0; q < NQ; ++q) c[q] *= inv;
        }
        if (a.bias) {
#pragma unroll
            for (int q = 0; q < NQ; ++q) {
                const float b = a.bias[min(lane * NQ + q, a.E - 1)];
                bias = fmaxf(bias, b > -INFINITY ? 2.f * fabsf(b) : 0.f);
                c[q] += b;
            }
            bias = __uint_as_float(wave_max_u(__float_as_uint(bias)));  // not negative: ordered as its bits
        }
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            c[q] = v[q] == -INFINITY ? -INFINITY : c[q];
            again |= !(c[q] < INFINITY);  // NaN, or +inf from a bias
        }
    }
    unsure = __any(again);
    if (unsure) return -1;
    uint32_t key[NQ];
#pragma unroll
    for (int q = 0; q < NQ; ++q) key[q] = key32(c[q]);
    if constexpr (kGroups) {
        float* const sc = reinterpret_cast<float*>(rs.c);
        if constexpr (kBy != kByLogits) {
#pragma unroll
            for (int q = 0; q < NQ; ++q) sc[lane * NQ + q] = c[q];
            __builtin_amdgcn_wave_barrier();
            __atomic_signal_fence(__ATOMIC_SEQ_CST);
        }
        const float* const of_group = kBy == kByLogits ? rs.v : sc;
        // `share` lanes for each group
        const int members = a.E / a.groups, share = 1 << (31 - __builtin_clz(64 / a.groups)), g = lane / share;
        float c1 = -INFINITY, c2 = -INFINITY;
        if (g < a.groups)
#pragma unroll 4
            for (int i = lane & (share - 1); i < members; i += share) {
                const float x = of_group[g * members + i];
                c2 = fmaxf(c2, fminf(c1, x));
                c1 = fmaxf(c1, x);
            }
        __builtin_amdgcn_wave_barrier();
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
        for (int o = 1; o < share; o <<= 1) {
            const float d1 = __shfl_xor(c1, o, 64), d2 = __shfl_xor(c2, o, 64);
            c2 = fmaxf(fmaxf(c2, d2), fminf(c1, d1));
            c1 = fmaxf(c1, d1);
        }
        const float score = kBy != kByLogits && a.best > 1 && c2 > -INFINITY ? c1 + c2 : c1;
        uint32_t group = g < a.groups && (lane & (share - 1)) == 0 ? key32(score) : 0u;
        // the best groups, one after another
        uint64_t kept = 0;  // bit g share
        uint32_t last = 0;
        for (int j = 0; j < a.top_groups; ++j) {
            const uint32_t m = wave_max_u(group);
            if (m == 0) break;
            const uint64_t all = __ballot(group == m), first = all & -all;
            kept |= first;
            if ((first >> lane) & 1) group = 0;
            last = m;
        }
        if constexpr (kBy != kByLogits) {
            const uint32_t next = wave_max_u(group);
            if (next) unsure |= too_near<kBy>(key32_value(last), key32_value(next), 2.f * bias);
        }
        // lane NQ + q is in group (lane NQ + q) / members: the product is exact below 2^16
        const uint32_t inv = (65536 + members - 1) / members;
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            const uint32_t of = ((uint32_t)(lane * NQ + q) * inv) >> 16;
            if (!((kept >> ((of * share) & 63)) & 1)) key[q] = 0;  // past E all keys are 0
        }
    }
    // each lane's keys in order, the lower place first among equal ones
    uint32_t place[NQ];
#pragma unroll
    for (int q = 0; q < NQ; ++q) place[q] = lane * NQ + q;
    auto order = [&](int i, int j) {
        const bool swap = key[i] < key[j];
        const uint32_t x = key[i], y = place[i];
        key[i] = swap ? key[j] : x, place[i] = swap ? place[j] : y;
        key[j] = swap ? x : key[j], place[j] = swap ? y : place[j];
    };
    if constexpr (NQ == 2) order(0, 1);
    if constexpr (NQ == 4) {  // neighbours only: stable
        order(0, 1), order(1, 2), order(2, 3);
        order(0, 1), order(1, 2);
        order(0, 1);
    }
    // lane j gets the j-th; where scores decide, the list goes on until one is clearly behind
    uint32_t mine = 0, last = 0;
    int my_id = -1, listed = 0;
    for (int j = 0; j < 64; ++j) {
        const uint32_t m = wave_max_u(key[0]);
        if (m == 0) break;
        if (j >= a.k && (kBy == kByLogits || !too_near<kBy>(key32_value(last), key32_value(m), bias))) break;
        const int from = __ffsll((unsigned long long)__ballot(key[0] == m)) - 1;
        const int id = __builtin_amdgcn_readlane((int)place[0], from);
        if (lane == j) mine = m, my_id = id;
        const bool pop = lane == from;
#pragma unroll
        for (int q = 0; q + 1 < NQ; ++q) {
            key[q] = pop ? key[q + 1] : key[q];
            place[q] = pop ? place[q + 1] : place[q];
        }
        key[NQ - 1] = pop ? 0u : key[NQ - 1];
        last = m;
        listed = j + 1;
    }
    if constexpr (kBy != kByLogits) {
        const uint32_t after = (uint32_t)__shfl_down((int)mine, 1, 64);
        const uint64_t close = __ballot(lane + 1 < listed && too_near<kBy>(key32_value(mine), key32_value(after), bias));
        unsure |= listed == 64;  // more of them than lanes
        if (close && !unsure) {  // the listed ones' scores in 64 bits, ranked by counting
            const double z = kBy == kBySoftmax ? exact_sum<NQ>(v, top) : 1.0;
            double exact = -INFINITY;
            if (lane < listed) exact = exact_score(a, rs.v[my_id], (double)top, z) + (a.bias ? (double)a.bias[my_id] : 0.0);
            int rank = 0;
            for (int j = 0; j < listed; ++j) {
                const double other = __longlong_as_double(((long long)__builtin_amdgcn_readlane((int)(__double_as_longlong(exact) >> 32), j) << 32) |
                                                          (uint32_t)__builtin_amdgcn_readlane((int)__double_as_longlong(exact), j));
                const int id = __builtin_amdgcn_readlane(my_id, j);
                rank += other > exact || (other == exact && id < my_id);
            }
            int* const slot = reinterpret_cast<int*>(rs.c);
            __builtin_amdgcn_wave_barrier();
            __atomic_signal_fence(__ATOMIC_SEQ_CST);
            if (lane < listed) slot[rank] = my_id;
            __builtin_amdgcn_wave_barrier();
            __atomic_signal_fence(__ATOMIC_SEQ_CST);
            my_id = lane < listed ? slot[lane] : -1;
            __builtin_amdgcn_wave_barrier();
            __atomic_signal_fence(__ATOMIC_SEQ_CST);
        }
    }
    return lane < a.k ? my_id : -1;
}

// One wave routes token t: lane j < k gets the j-th chosen expert (-1: none) and its weight.
template <int NQ, int kBy, bool kGroups>
__device__ __forceinline__ void route_token(const RouteArgs& a, int t, int lane, RouteScratch& rs, int& my_id, float& my_w) {
    float v[NQ], top = -INFINITY;
    bool nan = false;
    const size_t at = (size_t)t * a.ldl;
    if (a.bf16) {
#pragma unroll
        for (int q = 0; q < NQ; ++q) v[q] = load1<true>(a.logits, at + min(lane * NQ + q, a.E - 1));
    } else {
#pragma unroll
        for (int q = 0; q < NQ; ++q) v[q] = load1<false>(a.logits, at + min(lane * NQ + q, a.E - 1));
    }
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        v[q] = lane * NQ + q < a.E ? v[q] : -INFINITY;
        rs.v[lane * NQ + q] = v[q];
        top = fmaxf(top, v[q]);
        nan |= __builtin_isnan(v[q]);
    }
    __builtin_amdgcn_wave_barrier();
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    const bool whole = !a.sigmoid && !a.normalize;  // weights out of a softmax over all experts
    if (kBy == kBySoftmax || whole) top = wave_max(top);
    bool unsure;
    my_id = choose_fast<NQ, kBy, kGroups>(a, v, lane, rs, top, unsure);
    if (unsure) my_id = choose_exact<NQ>(a, v, lane, rs);
    const float my_logit = my_id < 0 ? -INFINITY : rs.v[my_id];
    __builtin_amdgcn_wave_barrier();  // the scratch is reused by the wave's next token
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    float w;
    if (a.normalize) {
        if (!a.sigmoid) {
            const float m = wave_max(my_logit);
            w = my_id < 0 ? 0.f : exp_fast(my_logit - m);
        } else if (!__any(my_id >= 0 && my_logit < -60.f)) {
            w = my_id < 0 ? 0.f : sigmoid_fast(my_logit);
        } else {  // a score near the end of fp32's range, or past it: differences of their logarithms
            const float ls = my_id < 0 ? -INFINITY : log_sigmoid(my_logit);
            const float most = wave_max(ls);
            w = my_id < 0 ? 0.f : expf(ls - most);
        }
        w /= wave_total_f(w);
    } else if (a.sigmoid) {
        w = 1.f / (1.f + expf(-my_logit));
    } else {
        float z = 0.f;
#pragma unroll
        for (int q = 0; q < NQ; ++q) z += v[q] == -INFINITY ? 0.f : exp_fast(v[q] - top);
        w = exp_fast(my_logit - top) / wave_total_f(z);
    }
    if (!a.sigmoid && __any(nan)) w = NAN;
    my_w = my_id < 0 ? 0.f : w * a.scale;
}

// Tokens [t0, t1), every `step`-th; their experts are counted in hist.
template <int NQ, int kBy, bool kGroups>
__device__ __forceinline__ void route_range(const RouteArgs& a, int t0, int t1, int step, int lane, RouteScratch& rs, int* hist) {
    for (int t = t0; t < t1; t += step) {
        float w;
        int id;
        route_token<NQ, kBy, kGroups>(a, t, lane, rs, id, w);
        if (lane < a.k) {
            a.idx[(size_t)t * a.k + lane] = id;
            a.w[(size_t)t * a.k + lane] = w;
            if (id >= 0) atomicAdd(&hist[id], 1);  // a count: arrival order does not matter
        }
    }
}

template <int NQ, int kBy, bool kGroups>
__global__ __launch_bounds__(kThreads) void route_kernel(const RouteArgs a) {
    __shared__ int hist[kMaxExperts];
    __shared__ RouteScratch rs[kWaves];
    if (threadIdx.x < kMaxExperts) hist[threadIdx.x] = 0;
    __syncthreads();
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int block = a.first + blockIdx.x, t0 = block * a.counted, t1 = min(a.T, t0 + a.counted);
    route_range<NQ, kBy, kGroups>(a, t0 + wave, t1, kWaves, lane, rs[wave], hist);
    if (!a.hist) return;
    __syncthreads();
    const int e = 4 * threadIdx.x;
    if ((int)threadIdx.x < a.words)
        a.hist[(size_t)block * a.words + threadIdx.x] =
            (uint32_t)hist[e] | (uint32_t)hist[e + 1] << 8 | (uint32_t)hist[e + 2] << 16 | (uint32_t)hist[e + 3] << 24;
}

// Places the assignments [a0, a1), one wave: rank among equal ids from ballots, `run`
// the next place of each expert.  first_ids: those of a0 + lane.
__device__ __forceinline__ void place(const RouteArgs& a, long long a0, long long a1, int first_ids, int* run) {
    const int lane = threadIdx.x & 63;
    const uint64_t lower = lane ? (~0ull) >> (64 - lane) : 0ull;
    for (long long r0 = a0; r0 < a1; r0 += 64) {
        const long long i = r0 + lane;
        const int e = i >= a1 ? -1 : r0 == a0 ? first_ids : a.idx[i];
        const bool valid = e >= 0;
        uint64_t match = __ballot(valid);
#pragma unroll
        for (int bit = 0; bit < 8; ++bit) {
            const bool b = (e >> bit) & 1;
            const uint64_t bb = __ballot(valid && b);
            match &= b ? bb : ~bb;
        }
        const int first = valid ? run[e] : 0;
        __builtin_amdgcn_wave_barrier();
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
        if (valid) {
            const int to = first + __popcll(match & lower);
            a.perm[to] = (int32_t)i;
            a.pos[i] = to;
            if ((match & lower) == 0) run[e] = first + __popcll(match);
        } else if (i < a1) {
            a.pos[i] = -1;
        }
        __builtin_amdgcn_wave_barrier();
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
    }
}

// kRoute: the one workgroup routes its tokens too.
template <bool kRoute, int NQ, int kBy, bool kGroups>
__global__ __launch_bounds__(kThreads) void route_tables_kernel(const RouteArgs a) {
    __shared__ int run[kWaves][kMaxExperts];  // counts of each wave's tokens, then where they go
    __shared__ int sums[2][kMaxExperts];      // all histograms, and those of the chunks before this one
    __shared__ int start[kMaxExperts + 1];
    __shared__ RouteScratch rs[kRoute ? kWaves : 1];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, E = a.E;
    const int t0 = blockIdx.x * a.chunk, t1 = min(a.T, t0 + a.chunk);
    const int per = (t1 - t0 + kWaves - 1) / kWaves;
    const int w0 = min(t1, t0 + wave * per), w1 = min(t1, w0 + per);
    const long long a0 = (long long)w0 * a.k, a1 = (long long)w1 * a.k;
    int first_ids = -1;
    if (!kRoute && a0 + lane < a1) first_ids = a.idx[a0 + lane];
    for (int e = lane; e < E; e += 64) run[wave][e] = 0;
    if constexpr (kRoute) {
        __builtin_amdgcn_wave_barrier();
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
        route_range<NQ, kBy, kGroups>(a, w0, w1, 1, lane, rs[wave], run[wave]);
        if (a0 + lane < a1) first_ids = a.idx[a0 + lane];
        __syncthreads();
    } else {
        if (threadIdx.x < kMaxExperts) sums[0][threadIdx.x] = sums[1][threadIdx.x] = 0;
        __syncthreads();
        for (long long i = a0 + lane; i < a1; i += 64) {
            const int e = i == a0 + lane ? first_ids : a.idx[i];
            if (e >= 0) atomicAdd(&run[wave][e], 1);  // a count
        }
        // four experts a lane (expert 4 lane + j at [j 64 + lane], so that no two lanes meet in a bank),
        // every 16th histogram a wave; sums of whole numbers
        const int rows = (a.T + a.counted - 1) / a.counted, mine = t0 / a.counted;
        if (lane < a.words) {
            // 32 of them requested together; two experts' counts in the halves of a word (32 times 128 at most)
            constexpr int kTogether = 32;
            int all[4] = {}, before[4] = {};
            for (int h0 = wave; h0 < rows; h0 += kTogether * kWaves) {
                uint32_t n[kTogether], even[2] = {}, odd[2] = {};
#pragma unroll
                for (int i = 0; i < kTogether; ++i) n[i] = a.hist[(size_t)min(h0 + i * kWaves, rows - 1) * a.words + lane];
                __builtin_amdgcn_sched_barrier(0);  // else the compiler waits for one after another (65536 tokens: 12 us where this takes 8)
#pragma unroll
                for (int i = 0; i < kTogether; ++i) {
                    const int h = h0 + i * kWaves;
                    const uint32_t x = h < rows ? n[i] : 0u, y = h < mine ? x : 0u;
                    even[0] += x & 0x00ff00ffu, odd[0] += (x >> 8) & 0x00ff00ffu;
                    even[1] += y & 0x00ff00ffu, odd[1] += (y >> 8) & 0x00ff00ffu;
                }
                all[0] += even[0] & 0xffff, all[1] += odd[0] & 0xffff, all[2] += even[0] >> 16, all[3] += odd[0] >> 16;
                before[0] += even[1] & 0xffff, before[1] += odd[1] & 0xffff, before[2] += even[1] >> 16, before[3] += odd[1] >> 16;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                atomicAdd(&sums[0][64 * j + lane], all[j]);
                if (mine) atomicAdd(&sums[1][64 * j + lane], before[j]);
            }
        }
        __syncthreads();
    }
    if (wave == 0) {  // the experts' starts: four experts a lane
        int n[kQ], local = 0;
#pragma unroll
        for (int q = 0; q < kQ; ++q) {
            const int e = lane * kQ + q;
            n[q] = 0;
            if (e < E) {
                if constexpr (kRoute)
#pragma unroll
                    for (int w = 0; w < kWaves; ++w) n[q] += run[w][e];
                else
                    n[q] = sums[0][64 * q + lane];
            }
            local += n[q];
        }
        const int inc = wave_incl_scan(local);
        int base = inc - local;
#pragma unroll
        for (int q = 0; q < kQ; ++q) {
            const int e = lane * kQ + q;
            if (e < E) {
                start[e] = base;
                if (blockIdx.x == 0) {
                    a.counts[e] = n[q];
                    a.offsets[e] = base;
                }
            }
            base += n[q];
        }
        if (lane == 63) {
            start[E] = inc;
            if (blockIdx.x == 0) a.offsets[E] = inc;
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += kThreads) {
        int to = start[e];
        if constexpr (!kRoute) to += sums[1][64 * (e & 3) + (e >> 2)];
        int n[kWaves];
#pragma unroll
        for (int w = 0; w < kWaves; ++w) n[w] = run[w][e];
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            run[w][e] = to;
            to += n[w];
        }
    }
    __syncthreads();
    place(a, a0, a1, first_ids, run[wave]);
    // behind the last row
    const long long rows = start[E], A = (long long)a.T * a.k;
    for (long long i = rows + blockIdx.x * (long long)kThreads + threadIdx.x; i < A; i += (long long)gridDim.x * kThreads) a.perm[i] = -1;
}

template <int NQ, int kBy, bool kGroups>
hipError_t launch_route(const RouteArgs& a, bool tables, hipStream_t s) {
    if (tables && a.T <= kOneWorkgroup) {
        route_tables_kernel<true, NQ, kBy, kGroups><<<1, kThreads, 0, s>>>(a);
        return hipGetLastError();
    }
    RouteArgs b = a;
    constexpr int kSlice = 1 << 21;  // a launch's threads are fewer than 2^32
    const int blocks = (a.T + a.counted - 1) / a.counted;
    for (b.first = 0; b.first < blocks; b.first += kSlice) {
        route_kernel<NQ, kBy, kGroups><<<std::min(kSlice, blocks - b.first), kThreads, 0, s>>>(b);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
    }
    if (tables) route_tables_kernel<false, 1, 0, false><<<(a.T + a.chunk - 1) / a.chunk, kThreads, 0, s>>>(a);
    return hipGetLastError();
}
template <int NQ>
hipError_t launch_route(const RouteArgs& a, bool tables, hipStream_t s) {
    if (!a.bias && (a.groups == 1 || a.best == 1))
        return a.groups > 1 ? launch_route<NQ, kByLogits, true>(a, tables, s) : launch_route<NQ, kByLogits, false>(a, tables, s);
    if (a.sigmoid) return a.groups > 1 ? launch_route<NQ, kBySigmoid, true>(a, tables, s) : launch_route<NQ, kBySigmoid, false>(a, tables, s);
    return a.groups > 1 ? launch_route<NQ, kBySoftmax, true>(a, tables, s) : launch_route<NQ, kBySoftmax, false>(a, tables, s);
}

struct RouteGradArgs {
    const void* logits;
    const int32_t* idx;
    const float* dw;
    void* dl;
    size_t ldl, lddl;
    int T, E, k, sigmoid, normalize;
    float scale;
};

// One wave per token.  With g = scale dw:
//   softmax     dl = s (g - sum g s)       normalised: the same over the chosen, 0 elsewhere
//   sigmoid     dl = g s (1 - s)           normalised: w (g - sum g w) (1 - s)
template <bool kBf16>
__global__ __launch_bounds__(256) void route_grad_kernel(const RouteGradArgs a) {
    const int lane = threadIdx.x & 63, t = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (t >= a.T) return;
    float v[kQ], g[kQ] = {};
    bool chosen[kQ] = {};
    const int my = lane < a.k ? a.idx[(size_t)t * a.k + lane] : -1;
    const float my_g = lane < a.k ? a.scale * a.dw[(size_t)t * a.k + lane] : 0.f;
#pragma unroll
    for (int q = 0; q < kQ; ++q) {
        const int e = lane + 64 * q;
        const float x = load1<kBf16>(a.logits, (size_t)t * a.ldl + min(e, a.E - 1));
        v[q] = e < a.E ? x : -INFINITY;
    }
    for (int j = 0; j < a.k; ++j) {
        const int e = __builtin_amdgcn_readlane(my, j);
        const float gj = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(my_g), j));
#pragma unroll
        for (int q = 0; q < kQ; ++q)
            if (lane + 64 * q == e) chosen[q] = true, g[q] += gj;
    }
    float dl[kQ];
    if (a.sigmoid && !a.normalize) {
#pragma unroll
        for (int q = 0; q < kQ; ++q) {
            const float en = expf(-fabsf(v[q])), s = 1.f / (1.f + en);  // s (1 - s) is the same for v and -v
            dl[q] = chosen[q] ? g[q] * (s * (en * s)) : 0.f;
        }
    } else {
        // a softmax over all experts, or over the chosen ones' log scores
        float ls[kQ], top = -INFINITY, z = 0.f, dot = 0.f;
#pragma unroll
        for (int q = 0; q < kQ; ++q) {
            const bool in = a.normalize ? chosen[q] : v[q] != -INFINITY;
            ls[q] = !in ? -INFINITY : a.sigmoid ? log_sigmoid(v[q]) : v[q];
            top = fmaxf(top, ls[q]);
        }
        top = wave_max(top);
#pragma unroll
        for (int q = 0; q < kQ; ++q) {
            const float p = ls[q] == -INFINITY ? 0.f : expf(ls[q] - top);
            ls[q] = p;
            z += p;
            if (chosen[q]) dot += p * g[q];
        }
        z = wave_total_f(z);
        dot = wave_total_f(dot) / z;
#pragma unroll
        for (int q = 0; q < kQ; ++q) {
            float d = ls[q] == 0.f && !chosen[q] ? 0.f : ls[q] / z * (g[q] - dot);
            if (a.sigmoid && chosen[q]) d /= 1.f + expf(v[q]);  // 1 - s
            dl[q] = z == 0.f ? 0.f : d;
        }
    }
#pragma unroll
    for (int q = 0; q < kQ; ++q) {
        const int e = lane + 64 * q;
        if (e >= a.E) continue;
        if constexpr (kBf16) reinterpret_cast<bf16_t*>(a.dl)[(size_t)t * a.lddl + e] = f32_to_bf16(dl[q]);
        else reinterpret_cast<float*>(a.dl)[(size_t)t * a.lddl + e] = dl[q];
    }
}

bool misaligned(const void* p, uintptr_t mask) { return ((uintptr_t)p & mask) != 0; }

constexpr long long kMaxStride = 1 << 21;

int check_router(const flexmoe_router_desc* D, int T, const char* who, long long* ldl) {
    if (!D) return fail(FLEXMOE_EINVAL, "%s: desc is NULL", who);
    if (D->dtype != FLEXMOE_F32 && D->dtype != FLEXMOE_BF16)
        return fail(FLEXMOE_EDTYPE, "%s: dtype %d is neither FLEXMOE_F32 nor FLEXMOE_BF16", who, D->dtype);
    if (D->E < 1 || D->E > kMaxExperts) return fail(FLEXMOE_ESHAPE, "%s: E = %d outside [1, %d]", who, D->E, kMaxExperts);
    if (D->top_k < 1 || D->top_k > D->E || D->top_k > kMaxTopK)
        return fail(FLEXMOE_ESHAPE, "%s: top_k = %d outside [1, min(E, %d)]", who, D->top_k, kMaxTopK);
    if (D->score != FLEXMOE_SOFTMAX && D->score != FLEXMOE_SIGMOID)
        return fail(FLEXMOE_EINVAL, "%s: score = %d is neither FLEXMOE_SOFTMAX nor FLEXMOE_SIGMOID", who, D->score);
    if (D->normalize != 0 && D->normalize != 1) return fail(FLEXMOE_EINVAL, "%s: normalize must be 0 or 1 (got %d)", who, D->normalize);
    if (D->groups < 1 || D->groups > kMaxGroups || D->E % D->groups)
        return fail(FLEXMOE_ESHAPE, "%s: groups = %d must divide E = %d and be at most %d", who, D->groups, D->E, kMaxGroups);
    const int size = D->E / D->groups;
    if (D->top_groups < 1 || D->top_groups > D->groups || D->top_k > size * D->top_groups)
        return fail(FLEXMOE_ESHAPE, "%s: top_groups = %d outside [1, groups], or with fewer experts than top_k", who, D->top_groups);
    if (D->group_best < 1 || D->group_best > 2 || (D->groups > 1 && D->group_best > size))
        return fail(FLEXMOE_ESHAPE, "%s: group_best = %d must be 1 or 2 and at most a group's size", who, D->group_best);
    if (!std::isfinite(D->scale)) return fail(FLEXMOE_EINVAL, "%s: scale must be finite", who);
    if (D->max_tokens < 0 || (long long)D->max_tokens * (D->top_k + 1) > (1LL << 30))
        return fail(FLEXMOE_ESHAPE, "%s: max_tokens = %d is negative or max_tokens * (top_k + 1) exceeds 2^30", who, D->max_tokens);
    *ldl = D->ldl ? D->ldl : D->E;
    if (*ldl < D->E || *ldl > kMaxStride) return fail(FLEXMOE_ESHAPE, "%s: ldl = %lld outside [E, 2^21]", who, *ldl);
    if (T < 0) return fail(FLEXMOE_EINVAL, "%s: T = %d is negative", who, T);
    if (T > D->max_tokens) return fail(FLEXMOE_ESHAPE, "%s: T = %d above max_tokens = %d", who, T, D->max_tokens);
    return FLEXMOE_OK;
}

// Workgroups of route_kernel, a histogram each: one a compute unit (tables read fewer of them), past its tokens two, in
// whole rounds.  8192 tokens of 60 experts 14.2 us with 256, 15.6 with 512; 65536 37.8 with 512, 47.3 and 45.2 with 768 and
// 1024; 131072 98 with 547, 79 with 1024 (of an earlier form of the kernel).
int histograms(int T) { return T <= 256 * kMostCounted ? 256 : (int)(((long long)T + 512 * kMostCounted - 1) / (512 * kMostCounted)) * 512; }

// Tokens of a histogram (a multiple of a workgroup's waves) and of a chunk.
int counted_tokens(int T) {
    const int wanted = histograms(T), per = (T + wanted - 1) / wanted;
    return std::max(1, (per + kWaves - 1) / kWaves) * kWaves;
}
int chunk_tokens(int T, int counted) {
    const int per = (T + kChunks - 1) / kChunks;
    return std::max(1, (per + counted - 1) / counted) * counted;
}

int hist_words(int E) { return (E + 3) / 4; }

size_t route_bytes(const flexmoe_router_desc* D, int T) {
    return ((size_t)histograms(T) * hist_words(D->E) * 4 + 255) & ~size_t(255);
}

}  // namespace

extern "C" {

size_t flexmoe_route_workspace_bytes(const flexmoe_router_desc* desc, int32_t T) {
    long long ldl;
    if (check_router(desc, T, "route_workspace_bytes", &ldl)) return 0;
    return route_bytes(desc, T);
}

int flexmoe_route(const flexmoe_router_desc* desc, int32_t T, const void* logits, const float* bias, const flexmoe_route_out* out,
                  void* workspace, size_t workspace_bytes, void* stream) {
    const char* who = "route";
    long long ldl;
    const int rc = check_router(desc, T, who, &ldl);
    if (rc) return rc;
    if (!out) return fail(FLEXMOE_EINVAL, "%s: out is NULL", who);
    const bool tables = out->counts || out->offsets || out->perm || out->pos;
    if (tables && (!out->counts || !out->offsets || (T > 0 && (!out->perm || !out->pos))))
        return fail(FLEXMOE_EINVAL, "%s: counts, offsets, perm and pos go together", who);
    if (T > 0 && (!logits || !out->topk_idx || !out->topk_w)) return fail(FLEXMOE_EINVAL, "%s: a pointer is NULL", who);
    if (misaligned(logits, desc->dtype == FLEXMOE_BF16 ? 1 : 3)) return fail(FLEXMOE_EINVAL, "%s: logits are not aligned to their elements", who);
    for (const void* p : {(const void*)bias, (const void*)out->topk_idx, (const void*)out->topk_w, (const void*)out->counts,
                          (const void*)out->offsets, (const void*)out->perm, (const void*)out->pos})
        if (misaligned(p, 3)) return fail(FLEXMOE_EINVAL, "%s: bias and results must be 4-byte aligned", who);
    if (T == 0 && !tables) return FLEXMOE_OK;
    RouteArgs a;
    a.logits = logits, a.bias = bias, a.idx = out->topk_idx, a.w = out->topk_w;
    a.counts = out->counts, a.offsets = out->offsets, a.perm = out->perm, a.pos = out->pos;
    a.hist = nullptr, a.ldl = (size_t)ldl, a.first = 0;
    a.T = T, a.E = desc->E, a.k = desc->top_k, a.bf16 = desc->dtype == FLEXMOE_BF16;
    a.sigmoid = desc->score == FLEXMOE_SIGMOID, a.normalize = desc->normalize;
    a.groups = desc->groups, a.top_groups = desc->top_groups, a.best = desc->group_best, a.scale = desc->scale;
    a.counted = counted_tokens(T), a.chunk = chunk_tokens(T, a.counted), a.words = hist_words(a.E);
    if (tables && T > kOneWorkgroup) {
        const size_t need = route_bytes(desc, T);
        if (!workspace || workspace_bytes < need)
            return fail(FLEXMOE_EWORKSPACE, "%s: workspace of %zu bytes, %zu needed", who, workspace ? workspace_bytes : 0, need);
        if (misaligned(workspace, 255)) return fail(FLEXMOE_EWORKSPACE, "%s: workspace must be 256-byte aligned", who);
        a.hist = (uint32_t*)workspace;
    }
    const hipStream_t s = (hipStream_t)stream;
    const hipError_t err = a.E <= 64 ? launch_route<1>(a, tables, s) : a.E <= 128 ? launch_route<2>(a, tables, s) : launch_route<4>(a, tables, s);
    if (err != hipSuccess) return hip_fail(err, who);
    return FLEXMOE_OK;
}

int flexmoe_route_backward(const flexmoe_router_desc* desc, int32_t T, const void* logits, const int32_t* topk_idx, const float* dw,
                           void* dlogits, int64_t lddl, void* stream) {
    const char* who = "route_backward";
    long long ldl;
    const int rc = check_router(desc, T, who, &ldl);
    if (rc) return rc;
    if (!lddl) lddl = desc->E;
    if (lddl < desc->E || lddl > kMaxStride) return fail(FLEXMOE_ESHAPE, "%s: lddl = %lld outside [E, 2^21]", who, (long long)lddl);
    if (T == 0) return FLEXMOE_OK;
    if (!logits || !topk_idx || !dw || !dlogits) return fail(FLEXMOE_EINVAL, "%s: a pointer is NULL", who);
    const uintptr_t mask = desc->dtype == FLEXMOE_BF16 ? 1 : 3;
    if (misaligned(logits, mask) || misaligned(dlogits, mask) || misaligned(topk_idx, 3) || misaligned(dw, 3))
        return fail(FLEXMOE_EINVAL, "%s: a pointer is not aligned to its elements", who);
    RouteGradArgs a;
    a.logits = logits, a.idx = topk_idx, a.dw = dw, a.dl = dlogits, a.ldl = (size_t)ldl, a.lddl = (size_t)lddl;
    a.T = T, a.E = desc->E, a.k = desc->top_k, a.sigmoid = desc->score == FLEXMOE_SIGMOID, a.normalize = desc->normalize, a.scale = desc->scale;
    constexpr int kSlice = 1 << 24;  // a launch's threads are fewer than 2^32
    const size_t es = desc->dtype == FLEXMOE_BF16 ? 2 : 4;
    for (long long at = 0; at < T; at += kSlice) {
        RouteGradArgs b = a;
        b.T = (int)std::min<long long>(kSlice, T - at);
        b.logits = (const char*)logits + (size_t)at * ldl * es, b.dl = (char*)dlogits + (size_t)at * lddl * es;
        b.idx = topk_idx + (size_t)at * a.k, b.dw = dw + (size_t)at * a.k;
        const int grid = (b.T + 3) / 4;
        if (desc->dtype == FLEXMOE_BF16) route_grad_kernel<true><<<grid, 256, 0, (hipStream_t)stream>>>(b);
        else route_grad_kernel<false><<<grid, 256, 0, (hipStream_t)stream>>>(b);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return hip_fail(err, who);
    }
    return FLEXMOE_OK;
}

}  // extern "C"
