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
//   route_kernel         one wave per token; a histogram for each chunk of tokens
//   route_tables_kernel  every chunk sums the histograms before its own (and all
//                        of them, for the experts' starts), then places its
//                        tokens: stable, and no atomic's order is in a result
//   both in one workgroup for few tokens
//
// Latency and instructions, not bytes, bound these launches.
#include <algorithm>
#include <cmath>

#include "error.h"
#include "flexmoe.h"
#include "rows.h"

using namespace flexmoe;

namespace {

constexpr int kWaves = 16, kThreads = 64 * kWaves;
constexpr int kChunks = 128;      // chunks of tokens, at most (a workgroup of route_tables_kernel reads all their histograms)
constexpr int kOneWorkgroup = 16; // tokens up to which one workgroup does it all
constexpr int kMaxGroups = 64;
constexpr int kQ = kMaxExperts / 64;

struct RouteArgs {
    const void* logits;
    const float* bias;
    int32_t *idx, *counts, *offsets, *perm, *pos;
    float* w;
    int32_t* hist;  // [chunks][E]
    size_t ldl;
    int T, E, k, sigmoid, normalize, groups, top_groups, best, chunk;
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

__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const uint64_t u = (uint64_t)__shfl_xor((unsigned long long)v, o, 64);
        v = u > v ? u : v;
    }
    return v;
}

__device__ __forceinline__ float wave_max_f(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    return v;
}

__device__ __forceinline__ double wave_sum_d(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

__device__ __forceinline__ float log_sigmoid(float x) { return fminf(x, 0.f) - log1pf(expf(-fabsf(x))); }

struct RouteScratch {
    double c[kMaxExperts];
};

// One wave routes one token, whose logits are in v (expert lane + 64 q; -inf past E):
// lane j < k gets the j-th chosen expert (-1: none) and its weight.
__device__ void route_token(const RouteArgs& a, const float (&v)[kQ], int lane, RouteScratch& rs, int& my_id, float& my_w) {
    const bool exact = a.bias || (a.groups > 1 && a.best > 1);  // scores decide, else logits
    float top = -INFINITY;
    bool nan = false;
#pragma unroll
    for (int q = 0; q < kQ; ++q) {
        top = fmaxf(top, v[q]);
        nan |= __builtin_isnan(v[q]);
    }
    top = wave_max_f(top);
    const bool any_nan = __any(nan);
    double c[kQ];
    if (!exact) {
#pragma unroll
        for (int q = 0; q < kQ; ++q) c[q] = v[q];
    } else {
        double z = 0.0;
#pragma unroll
        for (int q = 0; q < kQ; ++q) {
            if (a.sigmoid) c[q] = 1.0 / (1.0 + exp(-(double)v[q]));
            else z += c[q] = v[q] == -INFINITY ? 0.0 : exp((double)v[q] - (double)top);
        }
        if (!a.sigmoid) {
            z = wave_sum_d(z);
#pragma unroll
            for (int q = 0; q < kQ; ++q) c[q] /= z;
        }
#pragma unroll
        for (int q = 0; q < kQ; ++q) {
            const int e = lane + 64 * q;
            if (a.bias && e < a.E) c[q] += (double)a.bias[e];
            if (v[q] == -INFINITY) c[q] = -INFINITY;
        }
    }
    uint64_t key[kQ];
#pragma unroll
    for (int q = 0; q < kQ; ++q) key[q] = score_key(c[q]);
    if (a.groups > 1) {
        const int size = a.E / a.groups;
#pragma unroll
        for (int q = 0; q < kQ; ++q)
            if (lane + 64 * q < a.E) rs.c[lane + 64 * q] = c[q];
        __builtin_amdgcn_wave_barrier();
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
        uint64_t group = 0;
        if (lane < a.groups) {
            double c1 = -INFINITY, c2 = -INFINITY;
            uint64_t k1 = 0, k2 = 0;
            for (int i = 0, j = lane % size; i < size; ++i, j = j + 1 == size ? 0 : j + 1) {
                const double x = rs.c[lane * size + j];
                const uint64_t kx = score_key(x);
                if (kx > k1) k2 = k1, c2 = c1, k1 = kx, c1 = x;
                else if (kx > k2) k2 = kx, c2 = x;
            }
            group = k1 == 0 ? 0 : a.best > 1 && k2 != 0 ? score_key(c1 + c2) : k1;
        }
        __builtin_amdgcn_wave_barrier();
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
        int better = 0;
        for (int g = 0; g < a.groups; ++g) {
            const uint64_t other = (uint64_t)__shfl((unsigned long long)group, g, 64);
            better += other > group || (other == group && g < lane);
        }
        const uint64_t kept = __ballot(lane < a.groups && better < a.top_groups);
#pragma unroll
        for (int q = 0; q < kQ; ++q)
            if (!((kept >> ((lane + 64 * q) / size & 63)) & 1)) key[q] = 0;
    }
    my_id = -1;
    float my_logit = -INFINITY;
    for (int j = 0; j < a.k; ++j) {
        uint64_t m = 0;
#pragma unroll
        for (int q = 0; q < kQ; ++q) m = key[q] > m ? key[q] : m;
        m = wave_max(m);
        if (m == 0) break;
        int id = -1;
        float logit = 0.f;
#pragma unroll
        for (int q = kQ - 1; q >= 0; --q) {
            const uint64_t has = __ballot(key[q] == m);
            if (has) {  // the last q that has it is the lowest
                id = 64 * q + __ffsll((unsigned long long)has) - 1;
                logit = __shfl(v[q], id & 63, 64);
            }
        }
#pragma unroll
        for (int q = 0; q < kQ; ++q)
            if (lane + 64 * q == id) key[q] = 0;
        if (lane == j) my_id = id, my_logit = logit;
    }
    float w;
    if (a.normalize) {
        const float ls = my_id < 0 ? -INFINITY : a.sigmoid ? log_sigmoid(my_logit) : my_logit;
        const float m = wave_max_f(ls);
        w = my_id < 0 ? 0.f : expf(ls - m);
        w /= wave_total_f(w);
    } else if (a.sigmoid) {
        w = 1.f / (1.f + expf(-my_logit));
    } else {
        float z = 0.f;
#pragma unroll
        for (int q = 0; q < kQ; ++q) z += v[q] == -INFINITY ? 0.f : expf(v[q] - top);
        w = expf(my_logit - top) / wave_total_f(z);
    }
    if (any_nan && !a.sigmoid) w = NAN;
    my_w = my_id < 0 ? 0.f : w * a.scale;
}

template <bool kBf16>
__device__ __forceinline__ void load_logits(const RouteArgs& a, int t, int lane, float (&v)[kQ]) {
#pragma unroll
    for (int q = 0; q < kQ; ++q) {
        const int e = lane + 64 * q;
        const float x = load1<kBf16>(a.logits, (size_t)t * a.ldl + min(e, a.E - 1));
        v[q] = e < a.E ? x : -INFINITY;
    }
}

// Tokens [t0, t1), one after another; their experts are counted in hist.
template <bool kBf16>
__device__ void route_range(const RouteArgs& a, int t0, int t1, int step, int lane, RouteScratch& rs, int* hist) {
    for (int t = t0; t < t1; t += step) {
        float v[kQ], w;
        int id;
        load_logits<kBf16>(a, t, lane, v);
        route_token(a, v, lane, rs, id, w);
        if (lane < a.k) {
            a.idx[(size_t)t * a.k + lane] = id;
            a.w[(size_t)t * a.k + lane] = w;
            if (hist && id >= 0) atomicAdd(&hist[id], 1);  // a count: arrival order does not matter
        }
    }
}

template <bool kBf16>
__global__ __launch_bounds__(kThreads) void route_kernel(const RouteArgs a) {
    __shared__ int hist[kMaxExperts];
    __shared__ RouteScratch rs[kWaves];
    for (int e = threadIdx.x; e < a.E; e += kThreads) hist[e] = 0;
    __syncthreads();
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int t0 = blockIdx.x * a.chunk, t1 = min(a.T, t0 + a.chunk);
    route_range<kBf16>(a, t0 + wave, t1, kWaves, lane, rs[wave], hist);
    if (!a.hist) return;
    __syncthreads();
    for (int e = threadIdx.x; e < a.E; e += kThreads) a.hist[(size_t)blockIdx.x * a.E + e] = hist[e];
}

// Places the assignments of tokens [t0, t1), one wave: rank among equal ids from
// ballots, `run` the next place of each expert.
__device__ __forceinline__ void place(const RouteArgs& a, const int32_t* idx, long long a0, long long a1, int* run) {
    const int lane = threadIdx.x & 63;
    const uint64_t lower = lane ? (~0ull) >> (64 - lane) : 0ull;
    for (long long r0 = a0; r0 < a1; r0 += 64) {
        const long long i = r0 + lane;
        const int e = i < a1 ? idx[i] : -1;
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
template <bool kBf16, bool kRoute>
__global__ __launch_bounds__(kThreads) void route_tables_kernel(const RouteArgs a) {
    __shared__ int run[kWaves][kMaxExperts];  // counts of each wave's tokens, then where they go
    __shared__ int sums[2][4][kMaxExperts];   // all chunks' counts, and those of the chunks before this one
    __shared__ int start[kMaxExperts + 1];
    __shared__ RouteScratch rs[kRoute ? kWaves : 1];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, E = a.E;
    const int t0 = blockIdx.x * a.chunk, t1 = min(a.T, t0 + a.chunk);
    const int per = (t1 - t0 + kWaves - 1) / kWaves;
    const int w0 = min(t1, t0 + wave * per), w1 = min(t1, w0 + per);
    for (int e = lane; e < E; e += 64) run[wave][e] = 0;
    __builtin_amdgcn_wave_barrier();
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    if constexpr (kRoute) {
        route_range<kBf16>(a, w0, w1, 1, lane, rs[wave], run[wave]);
    } else {
        for (long long i = (long long)w0 * a.k + lane; i < (long long)w1 * a.k; i += 64) {
            const int e = a.idx[i];
            if (e >= 0) atomicAdd(&run[wave][e], 1);  // a count
        }
        const int e = threadIdx.x & 255, part = threadIdx.x >> 8, chunks = gridDim.x;
        const int per_part = (chunks + 3) / 4, c0 = part * per_part, c1 = min(chunks, c0 + per_part);
        int all = 0, before = 0;
        if (e < E)
#pragma unroll 8
            for (int c = c0; c < c1; ++c) {
                const int n = a.hist[(size_t)c * E + e];
                all += n;
                before += c < (int)blockIdx.x ? n : 0;
            }
        sums[0][part][e] = all;
        sums[1][part][e] = before;
    }
    __syncthreads();
    if (wave == 0) {  // the experts' starts: four experts a lane
        int n[kQ], local = 0;
#pragma unroll
        for (int q = 0; q < kQ; ++q) {
            const int e = lane * kQ + q;
            n[q] = 0;
            if (e < E) {
                if constexpr (kRoute)
                    for (int w = 0; w < kWaves; ++w) n[q] += run[w][e];
                else
                    for (int p = 0; p < 4; ++p) n[q] += sums[0][p][e];
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
        if constexpr (!kRoute)
            for (int p = 0; p < 4; ++p) to += sums[1][p][e];
        for (int w = 0; w < kWaves; ++w) {
            const int n = run[w][e];
            run[w][e] = to;
            to += n;
        }
    }
    __syncthreads();
    place(a, a.idx, (long long)w0 * a.k, (long long)w1 * a.k, run[wave]);
    // behind the last row
    const long long rows = start[E], A = (long long)a.T * a.k;
    for (long long i = rows + blockIdx.x * (long long)kThreads + threadIdx.x; i < A; i += (long long)gridDim.x * kThreads) a.perm[i] = -1;
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
        top = wave_max_f(top);
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

// Tokens of a chunk: a multiple of a workgroup's waves.
int chunk_tokens(int T) { return std::max(kWaves, ((T + kChunks - 1) / kChunks + kWaves - 1) / kWaves * kWaves); }

size_t route_bytes(const flexmoe_router_desc* D) { return ((size_t)kChunks * D->E * sizeof(int32_t) + 255) & ~size_t(255); }

}  // namespace

extern "C" {

size_t flexmoe_route_workspace_bytes(const flexmoe_router_desc* desc, int32_t T) {
    long long ldl;
    if (check_router(desc, T, "route_workspace_bytes", &ldl)) return 0;
    return route_bytes(desc);
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
    a.hist = nullptr, a.ldl = (size_t)ldl;
    a.T = T, a.E = desc->E, a.k = desc->top_k, a.sigmoid = desc->score == FLEXMOE_SIGMOID, a.normalize = desc->normalize;
    a.groups = desc->groups, a.top_groups = desc->top_groups, a.best = desc->group_best, a.scale = desc->scale;
    const bool bf16 = desc->dtype == FLEXMOE_BF16;
    const hipStream_t s = (hipStream_t)stream;
    if (tables && T <= kOneWorkgroup) {
        a.chunk = kOneWorkgroup;
        if (bf16) route_tables_kernel<true, true><<<1, kThreads, 0, s>>>(a);
        else route_tables_kernel<false, true><<<1, kThreads, 0, s>>>(a);
        const hipError_t err = hipGetLastError();
        return err == hipSuccess ? FLEXMOE_OK : hip_fail(err, who);
    }
    a.chunk = chunk_tokens(T);
    if (tables) {
        const size_t need = route_bytes(desc);
        if (!workspace || workspace_bytes < need)
            return fail(FLEXMOE_EWORKSPACE, "%s: workspace of %zu bytes, %zu needed", who, workspace ? workspace_bytes : 0, need);
        if (misaligned(workspace, 255)) return fail(FLEXMOE_EWORKSPACE, "%s: workspace must be 256-byte aligned", who);
        a.hist = (int32_t*)workspace;
    }
    const int chunks = (T + a.chunk - 1) / a.chunk;
    if (bf16) route_kernel<true><<<chunks, kThreads, 0, s>>>(a);
    else route_kernel<false><<<chunks, kThreads, 0, s>>>(a);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess) return hip_fail(err, who);
    if (tables) {
        route_tables_kernel<false, false><<<chunks, kThreads, 0, s>>>(a);
        err = hipGetLastError();
        if (err != hipSuccess) return hip_fail(err, who);
    }
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
