// Distillation from a teacher's top log probabilities, with the cross entropy of
// labels, and the gradient of the student's logits (gfx950).
//
//   q = softmax(l / t) over V, q1 = softmax(l)
//   p: the teacher's probabilities of the K listed tokens, renormalised over them,
//      or (tail) as they are, with what they leave as one more class
//   KL = sum p (log p - log q) [+ p_rest (log p_rest - log q_rest)]
//   CE = -log q1[label]         loss = scale (kl_weight t^2 KL + ce_weight CE)
//   dl = scale (kl_weight t (q - p) + ce_weight (q1 - [label]))
//   with a tail: q_v - p_v on the list, q_v (1 - p_rest / q_rest) off it
//
// A divergence is a small difference of large logarithms: what concerns the
// listed tokens is in 64 bits, a row's sum of exponentials in 32.  With a tail
// the listed tokens are left out of the row's maximum and sum (a map of bits says
// which) and joined with them afterwards, so that q_rest is a sum, not a difference,
// and of terms up to 1, however far the listed tokens lie above.
//
// What the teacher's list gives does not hang on the student's maximum M and sum S
// (m and s without the listed tokens): with A = sum p log p [+ p_rest log p_rest] and
// B = sum p (x - y), y the largest listed x,
//   KL = A - (B - (M - y) sum p) / t + (sum p [+ p_rest]) log S [- p_rest (log s + (m - M) / t)]
// and off the list p_rest / q_rest q_v = p_rest e^((x - m) / t) / s.
//
// Many rows that fit the registers of a workgroup (distill_whole_kernel): every row is
// read once; while its gradients leave, the next row's logits come in.  Else:
//   distill_sums_kernel   maximum and sums of each part of a row, and the lists
//   distill_grad_kernel   joins a row's parts, then factor * exp(x) for a part of the
//                         row, then the listed tokens (distill_row_kernel: losses alone)
//
// Bound by memory where rows are many: 4096 x 131072 bf16, 64 listed, 430 us, 5.0 TB/s
// (414 of them whole rows, 16 the lists, whose 64-bit logarithms are bound by instructions
// and their tokens' logits by latency); with tail, labels and t = 2 482, 20 % padding 402. 1021 x
// 50001 fp32 with tail, labels and 20 % padding 120 us, 3.0 TB/s: three or four rows a workgroup, all
// in step, and four exponentials a value, whose instructions take half the time.
// Losses alone of 48 x 131072: 8 us.
#include <algorithm>
#include <cmath>

#include "error.h"
#include "flexmoe.h"
#include "vocab.h"

using namespace flexmoe;

namespace {

// What a row's list gives: sums over its tokens (see above), what it leaves, the label.
struct RowList {
    double a, b, mass, rest;
    float y, e, e1;  // with a tail: sums of 2^(c (x - y)) and 2^(log2(e) (x - y)); 0 where all x are -inf
    float x_label;
    int label;  // -1: none
    int pad;
};

// A token whose gradient is not factor * exp(x): of the list, or the label.
struct Mark {
    int id;  // -1: none
    float p, x;
    int kind;  // kListed, kLabel or both
};
enum { kListed = 1, kLabel = 2 };

struct DistillArgs {
    const void* logits;
    const int32_t *ids, *labels;
    const float *lp, *row_scale;
    float *kl, *ce;
    void* dlogits;
    float* parts;     // [rows][P][4]: m, sum at t, sum at 1
    RowList* lists;   // [rows]
    Mark* marks;      // [rows][K + 1]
    int32_t *order, *counts;  // per kOrder rows: those with a loss, and how many (row_scale given)
    size_t ld, ldd;
    int rows, V, P, length, K, tail, two;  // two: the labels' sum is not that of t
    float c, t, kl_weight, ce_weight;
    double inv_t;
};

constexpr int kOrder = 256;
constexpr float kLog2E = 1.4426950408889634f;

// Sums at t and, where they differ, at 1, while the largest value is still growing.
template <bool kTwo>
struct TwoSums {
    float m = -INFINITY, s = 0.f, r = 0.f, s1 = 0.f, r1 = 0.f, limit = -INFINITY;

    __device__ __forceinline__ void raise(float largest, float c) {
        if (!__any(largest > m)) return;
        if (largest > m) {
            const float to = largest * c, to1 = largest * kLog2E;
            if (m > -INFINITY) {
                s *= exp2_fast(r - to);
                if constexpr (kTwo) s1 *= exp2_fast(r1 - to1);
            }
            m = largest, r = to, r1 = to1;
        }
    }
    // The same for the largest value so far, but that the references stay while values are at most 2^16 times what
    // they stand for: nearly every step has a lane with a new largest one, few have one that is so much larger.
    __device__ __forceinline__ void raise_past(float largest, float c, float margin) {
        m = largest;
        if (!__any(largest > limit)) return;
        if (largest > limit) {
            const float to = largest * c, to1 = largest * kLog2E;
            if (limit > -INFINITY) {
                s *= exp2_fast(r - to);
                if constexpr (kTwo) s1 *= exp2_fast(r1 - to1);
            }
            limit = largest + margin, r = to, r1 = to1;
        }
    }
    __device__ __forceinline__ void add(float v, float c) {
        s += exp2_fast(fmaf(v, c, -r));
        if constexpr (kTwo) s1 += exp2_fast(fmaf(v, kLog2E, -r1));
    }
    // Against c m itself, not c m rounded.
    __device__ __forceinline__ void settle(float c) {
        if (m == -INFINITY) return;
        s *= exp2_fast(-fmaf(m, c, -r));
        if constexpr (kTwo) s1 *= exp2_fast(-fmaf(m, kLog2E, -r1));
    }
    __device__ __forceinline__ void refer(float to, float c) {
        if (m == to) return;
        if (m > -INFINITY) {
            s *= exp2_fast((m - to) * c);
            if constexpr (kTwo) s1 *= exp2_fast((m - to) * kLog2E);
        }
        m = to;
    }
};

// The wave's bits, in every lane.
__device__ __forceinline__ uint32_t wave_or(uint32_t v) {
#define FLEXMOE_OSTEP(C, M) v |= (uint32_t)dpp_shift<C, M>((int)v)
    FLEXMOE_OSTEP(0x111, 0xf);
    FLEXMOE_OSTEP(0x112, 0xf);
    FLEXMOE_OSTEP(0x114, 0xf);
    FLEXMOE_OSTEP(0x118, 0xf);
    FLEXMOE_OSTEP(0x142, 0xa);
    FLEXMOE_OSTEP(0x143, 0xc);
#undef FLEXMOE_OSTEP
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

template <int kThreads, bool kTwo>
__device__ __forceinline__ TwoSums<kTwo> join_threads(TwoSums<kTwo> a, float c, float (*part)[kThreads / 64]) {
    const int wave = threadIdx.x >> 6;
    float m = wave_max(a.m);
    if ((threadIdx.x & 63) == 0) part[0][wave] = m;
    __syncthreads();
    m = part[0][0];
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) m = fmaxf(m, part[0][w]);
    a.refer(m, c);
    a.s = wave_total_f(a.s);
    if constexpr (kTwo) a.s1 = wave_total_f(a.s1);
    if ((threadIdx.x & 63) == 0) part[1][wave] = a.s, part[2][wave] = a.s1;
    __syncthreads();
    a.s = part[1][0], a.s1 = part[2][0];
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) a.s += part[1][w], a.s1 += part[2][w];
    return a;
}

// The listed tokens of [begin, end) as bits.
__device__ __forceinline__ void map_listed(uint32_t* bits, const int32_t* ids, int K, int begin, int end) {
    for (int i = threadIdx.x; i < (end - begin + 31) / 32; i += kVT) bits[i] = 0;
    __syncthreads();
    for (int k = threadIdx.x; k < K; k += kVT) {
        const int id = ids[k];
        if (id >= begin && id < end) atomicOr(&bits[(id - begin) >> 5], 1u << ((id - begin) & 31));
    }
    __syncthreads();
}

// Leaves out those of the values i .. that are listed.
template <bool kBf16>
__device__ __forceinline__ void leave_out(const uint32_t* bits, int i, float (&v)[Vocab<kBf16>::n]) {
    constexpr int n = Vocab<kBf16>::n;
    const uint32_t b = (bits[i >> 5] >> (i & 31)) & ((1u << n) - 1);
    if (b)
#pragma unroll
        for (int k = 0; k < n; ++k) v[k] = (b >> k) & 1 ? -INFINITY : v[k];
}

// One wave writes down what the list of a row with a loss gives, kOwn tokens a lane.  seen: K ints of LDS.
template <bool kBf16, int kOwn>
__device__ __forceinline__ void list_row(const DistillArgs& a, size_t row, int* seen) {
    const int lane = threadIdx.x & 63, K = a.K;
    const void* const logits = reinterpret_cast<const char*>(a.logits) + row * a.ld * elem_size<kBf16>();
    int id[kOwn];
    float lp[kOwn], x[kOwn];
    // all that depends on nothing is asked for at once, then the logits
    int named = *(a.labels ? a.labels + row : a.ids + row * K);
    const float scale = *(a.row_scale ? a.row_scale + row : a.lp + row * K);
#pragma unroll
    for (int q = 0; q < kOwn; ++q) {
        const int k = min(lane + 64 * q, K - 1);
        id[q] = a.ids[row * K + k], lp[q] = a.lp[row * K + k];
    }
    __builtin_amdgcn_sched_barrier(0);
    if (a.row_scale && scale == 0.f) return;
    if (!a.labels) named = -1;
    const int label = named < a.V ? max(named, -1) : -1;
#pragma unroll
    for (int q = 0; q < kOwn; ++q) {
        const bool is = lane + 64 * q < K;
        if (!is || id[q] < 0 || id[q] >= a.V) id[q] = -1;
        if (!is) lp[q] = -INFINITY;
        x[q] = value_at<kBf16>(logits, max(id[q], 0));
        if (is) seen[lane + 64 * q] = id[q];
    }
    const float x_label = value_at<kBf16>(logits, max(label, 0));
    __builtin_amdgcn_wave_barrier();
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    // a token that is named again counts with its first place alone
    bool again[kOwn] = {}, label_listed = false;
#pragma unroll 8
    for (int j = 0; j < K; ++j) {
        const int other = seen[j];
#pragma unroll
        for (int q = 0; q < kOwn; ++q) again[q] |= other == id[q] && j < lane + 64 * q;
        label_listed |= other == label;
    }
    __builtin_amdgcn_wave_barrier();
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    float top = 0.f;
    if (!a.tail) {
        top = -INFINITY;
#pragma unroll
        for (int q = 0; q < kOwn; ++q)
            if (id[q] >= 0) top = fmaxf(top, lp[q]);
        top = wave_max(top);
    }
    double p[kOwn], logp[kOwn], mass = 0.0;
#pragma unroll
    for (int q = 0; q < kOwn; ++q) {
        if (again[q]) id[q] = -1;
        logp[q] = id[q] >= 0 && top > -INFINITY ? (double)lp[q] - (double)top : -INFINITY;
        p[q] = exp(logp[q]);
        mass += p[q];
    }
    mass = wave_total_d(mass);
    RowList out;
    out.rest = 0.0, out.e = out.e1 = 0.f;
    double rest_log = 0.0;
    if (a.tail) {
        out.rest = mass != mass ? mass : fmax(0.0, 1.0 - mass);
        rest_log = out.rest == 0.0 ? 0.0 : out.rest * log(out.rest);
    } else {
        const double log_mass = log(mass);
#pragma unroll
        for (int q = 0; q < kOwn; ++q) {
            p[q] = p[q] == 0.0 ? 0.0 : p[q] / mass;
            logp[q] -= log_mass;
        }
        if (mass > 0.0) mass = 1.0;
    }
    double sum_a = 0.0, sum_b = 0.0;
    float y = -INFINITY;
#pragma unroll
    for (int q = 0; q < kOwn; ++q)
        if (id[q] >= 0) y = fmaxf(y, x[q]);
    y = wave_max(y);
    if (!(fabsf(y) < INFINITY)) y = 0.f;
    if (a.tail) {  // NaN for one of NaN or +inf
        float e = 0.f, e1 = 0.f;
#pragma unroll
        for (int q = 0; q < kOwn; ++q)
            if (id[q] >= 0 && x[q] != -INFINITY) {
                const float d = __builtin_isinf(x[q]) ? NAN : x[q] - y;
                e += exp2_fast(d * a.c);
                e1 += exp2_fast(d * kLog2E);
            }
        out.e = wave_total_f(e), out.e1 = wave_total_f(e1);
    }
    Mark* const marks = a.marks + row * (K + 1);
#pragma unroll
    for (int q = 0; q < kOwn; ++q) {
        if (p[q] != 0.0) sum_a += p[q] * logp[q], sum_b += p[q] * ((double)x[q] - (double)y);
        if (id[q] >= 0 && __builtin_isnan(x[q])) sum_b = NAN;
        if (lane + 64 * q < K) marks[lane + 64 * q] = Mark{id[q], (float)p[q], x[q], kListed | (id[q] == label ? kLabel : 0)};
    }
    out.a = wave_total_d(sum_a) + rest_log, out.b = wave_total_d(sum_b), out.mass = mass;
    out.y = y, out.x_label = x_label, out.label = label;
    if (lane == 0) {
        marks[K] = Mark{label_listed ? -1 : label, 0.f, x_label, kLabel};
        a.lists[row] = out;
    }
}

template <bool kBf16>
__device__ __forceinline__ void list_row(const DistillArgs& a, size_t row, int* seen) {
    static_assert(kMaxTop == 128, "two tokens a lane");
    if (a.K <= 64) list_row<kBf16, 1>(a, row, seen);
    else list_row<kBf16, 2>(a, row, seen);
}

template <bool kBf16, bool kTail, bool kTwo>
__global__ __launch_bounds__(kVT) void distill_sums_kernel(const DistillArgs a) {
    using W = Vocab<kBf16>;
    __shared__ uint32_t bits[kTail ? kRange / 32 : 1];
    __shared__ float part[3][kVT / 64];
    __shared__ int seen[kVT / 64][kMaxTop];
    const size_t parts = (size_t)a.rows * a.P;
    if (blockIdx.x >= parts) {  // lists, four rows a workgroup
        const size_t row = (blockIdx.x - parts) * (kVT / 64) + (threadIdx.x >> 6);
        if (row < (size_t)a.rows) list_row<kBf16>(a, row, seen[threadIdx.x >> 6]);
        return;
    }
    const size_t row = blockIdx.x / a.P;
    const int p = blockIdx.x % a.P, t = threadIdx.x;
    if (a.row_scale && a.row_scale[row] == 0.f) return;
    const void* const logits = reinterpret_cast<const char*>(a.logits) + row * a.ld * elem_size<kBf16>();
    const int begin = p * a.length, end = min(a.V, begin + a.length);
    if constexpr (kTail) map_listed(bits, a.ids + row * a.K, a.K, begin, end);
    TwoSums<kTwo> sums;
    each_step<kBf16>(logits, begin, end, [&](int, int at, float (&v)[W::units][W::n]) {
        float gm = -INFINITY;
#pragma unroll
        for (int u = 0; u < W::units; ++u) {
            const int i = at + u * W::run + t * W::n;
            if constexpr (kTail)
                if (i < end) leave_out<kBf16>(bits, i - begin, v[u]);
            gm = max_of(v[u], gm);
        }
        sums.raise(gm, a.c);
#pragma unroll
        for (int u = 0; u < W::units; ++u)
#pragma unroll
            for (int k = 0; k < W::n; ++k) sums.add(v[u][k], a.c);
    });
    sums.settle(a.c);
    TwoSums<kTwo> all = join_threads<kVT>(sums, a.c, part);
    if (!(all.s < 3.0e38f && all.s1 < 3.0e38f) && all.m > -INFINITY && all.m < INFINITY) {
        // c m may have left fp32's range (or a value is no number): differences first
        TwoSums<kTwo> again;
        again.m = all.m;
        for (int i = begin + t * W::n; i < end; i += W::run) {
            float v[W::n];
            load_values<kBf16>(logits, i, end, v);
            if constexpr (kTail) leave_out<kBf16>(bits, i - begin, v);
#pragma unroll
            for (int k = 0; k < W::n; ++k) {
                again.s += exp2_fast((v[k] - all.m) * a.c);
                if constexpr (kTwo) again.s1 += exp2_fast((v[k] - all.m) * kLog2E);
            }
        }
        __syncthreads();
        all = join_threads<kVT>(again, a.c, part);
    }
    if (t == 0) {
        float* const o = a.parts + 4 * (row * a.P + p);
        o[0] = all.m, o[1] = all.s, o[2] = all.s1;
    }
}

__device__ __forceinline__ float scale_of(const DistillArgs& a, size_t row) { return a.row_scale ? a.row_scale[row] : 1.f; }

// What a row's tokens are multiplied with.
struct RowFactors {
    float m, f, f1;              // tokens off the list: f 2^(c (x - m)) + f1 2^(log2(e) (x - m))
    float M, listed, listed1;    // listed ones: listed 2^(c (x - M)) - p p_k + listed1 2^(log2(e) (x - M))
    float p, label;              // the label: less `label`
};

// The logarithm of a sum to about 2^-25: its power of two is taken off, whose part is exact in 64 bits.
__device__ __forceinline__ double log_of(float s) {
    if (!(s > 0.f && s < INFINITY)) return (double)logf(s);
    int e;
    float f = frexpf(s, &e);
    if (f < 0.70710678f) f *= 2.f, --e;
    return (double)e * 0.6931471805599453 + (double)logf(f);
}

// e^x for x <= 0 to about 2^-32 of itself (an error here is one of all that lies on one side of a gap): its power of two,
// and the exponential series up to u^8 / 8! for what is left, |u| <= 0.35; 0 below 2^-200.
__device__ __forceinline__ double exp_down(double x) {
    const double z = fmax(x * 1.4426950408889634, -200.0), whole = rint(z), u = (z - whole) * 0.6931471805599453;
    double e = 1.0 / 40320;
    for (double c : {1.0 / 5040, 1.0 / 720, 1.0 / 120, 1.0 / 24, 1.0 / 6, 0.5, 1.0, 1.0}) e = fma(e, u, c);
    return x > -138.0 ? ldexp(e, (int)whole) : 0.0;
}

// One wave joins a row's maximum and sums (with a tail: without the listed tokens) with
// its list and marks.  All lanes return the same; lane 0 writes the losses if `writes`.
__device__ __forceinline__ RowFactors end_row(const DistillArgs& a, size_t row, const RowList& list, const Mark* marks, float m, float s, float s1,
                                              float scale, bool writes) {
    const int lane = threadIdx.x & 63;
    float M = m, S = s, S1 = a.two ? s1 : s;
    double down = 1.0, down1 = 1.0;  // e^((m - M) / t), e^(m - M)
    if (a.tail && list.e != 0.f) {
        const double gap = m == -INFINITY ? -INFINITY : -fabs((double)m - (double)list.y);
        const double far = exp_down(gap * a.inv_t), far1 = a.two ? exp_down(gap) : far;
        if (m >= list.y) {
            S = (float)(s + far * list.e), S1 = a.two ? (float)(s1 + far1 * list.e1) : S;
        } else {
            M = list.y, down = far, down1 = far1;
            S = (float)(far * s + list.e), S1 = a.two ? (float)(far1 * s1 + list.e1) : S;
        }
    }
    const bool empty = M == -INFINITY && S == 0.f && list.b == list.b, labelled = list.label >= 0;
    const bool none = s == 0.f && S == S;  // no token off the list has a probability
    const double total = list.mass + list.rest;
    if (writes) {
        double kl = list.mass == 0.0 ? list.a : list.a - (list.b - ((double)M - (double)list.y) * list.mass) * a.inv_t;
        const double log_S = total == 0.0 ? 0.0 : log_of(S);
        kl += total * log_S;
        if (list.rest != 0.0) {
            // log probabilities in 32 bits leave about 1e-6 of their own: nothing, where there is no token for it
            if (none) kl = list.rest <= 1e-5 ? kl - list.rest * (log(list.rest) + log_S) : INFINITY;
            else kl -= list.rest * (log_of(s) + ((double)m - (double)M) * a.inv_t);
        }
        if (empty) kl = list.mass > 0.0 || list.rest > 1e-5 ? INFINITY : 0.0;
        const double ce = !labelled ? 0.0 : empty ? INFINITY : log_of(S1) - ((double)list.x_label - (double)M);
        if (lane == 0) {
            a.kl[row] = (float)kl;
            a.ce[row] = (float)ce;
        }
    }
    // s is at least about 1: neither quotient leaves fp32's range
    double dense = total;
    if (a.tail) dense = total * down - (list.rest != 0.0 ? list.rest * ((double)S / (double)s) : 0.0);
    const float by_kl = scale * a.kl_weight * a.t, by_ce = labelled ? scale * a.ce_weight : 0.f;
    const bool no_dense = empty || (a.tail && none);
    RowFactors o;
    o.m = m;
    o.f = no_dense ? 0.f : by_kl * (float)dense / S;
    o.f1 = no_dense ? 0.f : by_ce * (float)down1 / S1;
    o.M = M;
    o.listed = empty ? 0.f : by_kl * (float)total / S;
    o.listed1 = empty ? 0.f : by_ce / S1;
    o.p = empty ? 0.f : by_kl;
    o.label = empty ? 0.f : by_ce;
    return o;
}

__device__ __forceinline__ float marked(const DistillArgs& a, const RowFactors& r, const Mark& k) {
    const bool listed = k.kind & kListed;
    const float d = k.x == -INFINITY ? -INFINITY : k.x - (listed ? r.M : r.m);
    const float e = exp2_fast(d * a.c), e1 = a.two ? exp2_fast(d * kLog2E) : e;
    const float of_kl = listed ? r.listed * e - r.p * k.p : r.f * e;
    return of_kl + (listed ? r.listed1 : r.f1) * e1 - (k.kind & kLabel ? r.label : 0.f);
}

// A row's sums out of its parts', the same in all lanes.
__device__ __forceinline__ TwoSums<true> join_parts(const DistillArgs& a, size_t row) {
    const int lane = threadIdx.x & 63;
    const float* const parts = a.parts + 4 * row * a.P;
    TwoSums<true> all;
    for (int p = lane; p < a.P; p += 64) all.m = fmaxf(all.m, parts[4 * p]);
    all.m = wave_max(all.m);
    for (int p = lane; p < a.P; p += 64) {
        TwoSums<true> one;
        one.m = parts[4 * p], one.s = parts[4 * p + 1], one.s1 = parts[4 * p + 2];
        one.refer(all.m, a.c);
        all.s += one.s;
        all.s1 += one.s1;
    }
    all.s = wave_total_f(all.s);
    all.s1 = wave_total_f(all.s1);
    return all;
}

// Losses alone: a wave for each row.
__global__ __launch_bounds__(256) void distill_row_kernel(const DistillArgs a) {
    const size_t row = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= (size_t)a.rows) return;
    if (a.row_scale && a.row_scale[row] == 0.f) {
        if ((threadIdx.x & 63) == 0) a.kl[row] = a.ce[row] = 0.f;
        return;
    }
    const TwoSums<true> all = join_parts(a, row);
    end_row(a, row, a.lists[row], a.marks + row * (a.K + 1), all.m, all.s, all.s1, scale_of(a, row), true);
}

// 16 bytes of gradients at value i of a row that ends at `end`.
template <bool kBf16>
__device__ __forceinline__ void store_unit(char* out, int i, int end, const u32x4& w) {
    constexpr int n = Vocab<kBf16>::n;
    if (i + n <= end) {
        *reinterpret_cast<u32x4*>(out + (size_t)i * elem_size<kBf16>()) = w;
    } else {
#pragma unroll
        for (int k = 0; k < n - 1; ++k)
            if (i + k < end) {
                if constexpr (kBf16) reinterpret_cast<bf16_t*>(out)[i + k] = (bf16_t)(w[k >> 1] >> (16 * (k & 1)));
                else reinterpret_cast<uint32_t*>(out)[i + k] = w[k];
            }
    }
}

// Gradients of a unit's values; f1 is in f where the temperature is 1.
template <bool kBf16, bool kTwo>
__device__ __forceinline__ void gradients(const DistillArgs& a, float m, float f, float f1, float (&v)[Vocab<kBf16>::n]) {
#pragma unroll
    for (int k = 0; k < Vocab<kBf16>::n; ++k) {
        float g = f * exp2_fast((v[k] - m) * a.c);
        if constexpr (kTwo) g = fmaf(f1, exp2_fast((v[k] - m) * kLog2E), g);
        v[k] = g;
    }
}

template <bool kBf16>
__device__ __forceinline__ u32x4 pack_unit(const float (&v)[Vocab<kBf16>::n]) {
    u32x4 w;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (kBf16) w[k] = pack_bf16x2(v[2 * k], v[2 * k + 1]);
        else w[k] = __float_as_uint(v[k]);
    }
    return w;
}

template <bool kBf16, bool kTwo>
__global__ __launch_bounds__(kVT) void distill_grad_kernel(const DistillArgs a) {
    using W = Vocab<kBf16>;
    __shared__ RowFactors shared;
    const size_t row = blockIdx.x / a.P;
    const int p = blockIdx.x % a.P, t = threadIdx.x;
    const char* const logits = reinterpret_cast<const char*>(a.logits) + row * a.ld * elem_size<kBf16>();
    char* const out = reinterpret_cast<char*>(a.dlogits) + row * a.ldd * elem_size<kBf16>();
    const int begin = p * a.length, end = min(a.V, begin + a.length);
    if (a.row_scale && a.row_scale[row] == 0.f) {  // padding is not read
        for (int i = begin + t * W::n; i < end; i += W::run) store_unit<kBf16>(out, i, end, u32x4{0, 0, 0, 0});
        if (p == 0 && t == 0) a.kl[row] = a.ce[row] = 0.f;
        return;
    }
    if (t < 64) {
        const TwoSums<true> all = join_parts(a, row);
        const RowFactors r = end_row(a, row, a.lists[row], a.marks + row * (a.K + 1), all.m, all.s, all.s1, scale_of(a, row), p == 0);
        if (t == 0) shared = r;
    }
    __syncthreads();
    const RowFactors r = shared;
    const float f = kTwo ? r.f : r.f + r.f1;
    const bool zero = f == 0.f && (!kTwo || r.f1 == 0.f);  // nothing off the list
    if (zero)
        for (int i = begin + t * W::n; i < end; i += W::run) store_unit<kBf16>(out, i, end, u32x4{0, 0, 0, 0});
    each_step<kBf16>(logits, begin, zero ? begin : end, [&](int, int at, float (&v)[W::units][W::n]) {
#pragma unroll
        for (int u = 0; u < W::units; ++u) {
            const int i = at + u * W::run + t * W::n;
            gradients<kBf16, kTwo>(a, r.m, f, r.f1, v[u]);
            if (i < end) store_unit<kBf16>(out, i, end, pack_unit<kBf16>(v[u]));
        }
    });
    __syncthreads();  // the marked tokens' gradients go over what was written there
    if (r.p == 0.f && r.label == 0.f) return;
    for (int k = t; k <= a.K; k += kVT) {
        const Mark mark = a.marks[row * (a.K + 1) + k];
        if (mark.id < begin || mark.id >= end) continue;
        const float g = marked(a, r, mark);
        if constexpr (kBf16) reinterpret_cast<bf16_t*>(out)[mark.id] = f32_to_bf16(g);
        else reinterpret_cast<float*>(out)[mark.id] = g;
    }
}

// The lists of rows whose gradients distill_whole_kernel makes, a wave each; rows without
// a loss get their zeros here, each from a workgroup, and are left out of `order`.
template <bool kBf16>
__global__ __launch_bounds__(kOrder) void distill_list_kernel(const DistillArgs a) {
    constexpr int n = Vocab<kBf16>::n;
    __shared__ int seen[4][kMaxTop], waves[4];
    auto live = [&](int row) { return !(a.row_scale && a.row_scale[row] == 0.f); };
    if (a.row_scale && blockIdx.x % kOrder == 0) {
        const int row = blockIdx.x + threadIdx.x, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
        const bool is = row < a.rows && live(row);
        const uint64_t all = __ballot(is);
        if (lane == 0) waves[wave] = __popcll(all);
        __syncthreads();
        int at = __popcll(all & ((1ull << lane) - 1)), count = 0;
        for (int w = 0; w < 4; ++w) {
            if (w < wave) at += waves[w];
            count += waves[w];
        }
        if (is) a.order[blockIdx.x + at] = row;
        if (threadIdx.x == 0) a.counts[blockIdx.x / kOrder] = count;
    }
    const int listed = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (listed < a.rows) list_row<kBf16>(a, listed, seen[threadIdx.x >> 6]);
    const int row = blockIdx.x;
    if (live(row)) return;
    char* const out = reinterpret_cast<char*>(a.dlogits) + row * a.ldd * elem_size<kBf16>();
    for (int i = threadIdx.x * n; i < a.V; i += kOrder * n) store_unit<kBf16>(out, i, a.V, u32x4{0, 0, 0, 0});
    if (threadIdx.x == 0) a.kl[row] = a.ce[row] = 0.f;
}

// A scalar load of what no kernel writes meanwhile: as a vector load it would be the last
// of those in flight, and waiting for it would be waiting for the next row.
template <typename T>
__device__ __forceinline__ T load_scalar(const T* p) {
    struct Words {
        uint32_t w[sizeof(T) / 4];
    } words;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 4); ++i) words.w[i] = ((const uint32_t __attribute__((address_space(4)))*)(uintptr_t)p)[i];
    return __builtin_bit_cast(T, words);
}

// Whole rows in a workgroup's registers, one after another: each is read once.  While the
// gradients of a row leave unit by unit, the next row's units come into the registers
// that get free, and kLag units later they are summed: so memory is busy throughout,
// where it would wait for the first pass of each row.  Unit 0 of a thread is the row's
// last one, so that only it may be ragged.  A thread knows the marked tokens of its own
// units from a list in LDS (which is in no order, and need not be); the first of them is
// in registers.
// kHeld units a thread: 32 leave registers for two waves of a SIMD (207 to 216 of 256 are in use, and 145 to 193 scalar ones are
// spilled to lanes of vector registers), 16 for three.  kLag: what comes sooner is waited for,
// what comes later is summed when no store is left to hide it (4096 x 131072 bf16, with tail, labels and a temperature
// 485, 483, 489, 499 and 537 us with 4, 6, 8, 12 and 16; plain 430, 427, 429, 431, 436).
constexpr int waves_of(int held) { return held > 16 ? 2 : 3; }
template <bool kBf16, int kThreads, int kHeld, bool kTail, bool kTwo>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(waves_of(kHeld), waves_of(kHeld)))) void distill_whole_kernel(const DistillArgs a) {
    constexpr int n = Vocab<kBf16>::n, run = kThreads * n, kLag = kHeld * 3 / 16;
    __shared__ float part[3][kThreads / 64];
    __shared__ RowFactors shared;
    __shared__ Mark marks[2][kMaxTop + 1];  // of this row and of the next
    __shared__ int after[2][kMaxTop + 1], head[2][kThreads];
    __shared__ float mark_gradient[kMaxTop + 1];
    const int t = threadIdx.x, whole = a.V / n, held = (a.V + run - 1) / run;
    int tn = t * n;
    u32x4 raw[kHeld];
    // Rows as buffers: the units that a row does not have are read as zeros and not written, so that every unit is one
    // request and one store, which the compiler counts; under a condition it would wait for half of those in flight.
    auto buffer = [&](const char* row, int units) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(row), (short)0, units * 16, 0x00020000); };
    auto offset = [&](int i) { return (uint32_t)((held - 1 - i) * (run * 16 / n) + tn * (16 / n)); };
    auto logits_of = [&](int row) { return reinterpret_cast<const char*>(a.logits) + row * a.ld * elem_size<kBf16>(); };
    auto request = [&](__amdgpu_buffer_rsrc_t logits, int i) {
        raw[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(logits, offset(i), 0, 0));
    };
    const int units = (a.V + n - 1) / n;
    auto request_mark = [&](int row) { return a.marks[(size_t)row * (a.K + 1) + min(t, a.K)]; };
    auto keep_mark = [&](int set, const Mark& mark) {
        if (t > a.K) return;
        marks[set][t] = mark;
        if (mark.id >= 0) after[set][t] = atomicExch(&head[set][mark.id / n % kThreads], t);
    };
    // a thread's own marked tokens: one of them (most have one or none) as its place in the thread's units, and which of
    // those hold others
    struct Own {
        int at, leave, k;
        uint32_t units, others;  // units: of all threads of the wave
    };
    auto own_marks = [&](int set) {
        Own o{-1, -1, head[set][t], 0, 0};
        if (o.k >= 0) {
            const Mark mark = marks[set][o.k];
            o.at = (held - 1 - mark.id / run) * n + mark.id % n;
            o.leave = mark.kind & kListed ? o.at : -1;
            for (int k = after[set][o.k]; k >= 0; k = after[set][k]) o.others |= 1u << (held - 1 - marks[set][k].id / run);
            o.units = o.others | 1u << (o.at / n);
        }
        o.units = wave_or(o.units);
        return o;
    };
    // the row that is number `place` of those with a loss, or the end; places only grow
    int block = 0, before = 0;
    auto row_at = [&](int place) {
        if (!a.row_scale) return place;
        for (; block * kOrder < a.rows; ++block) {
            const int count = load_scalar(a.counts + block);
            if (place - before < count) return load_scalar(a.order + block * kOrder + place - before);
            before += count;
        }
        return a.rows;
    };
    auto leave_out = [&](int set, int i, float (&v)[n]) {
        for (int k = head[set][t]; k >= 0; k = after[set][k]) {
            const int at = marks[set][k].kind & kListed ? marks[set][k].id - i : -1;
#pragma unroll
            for (int j = 0; j < n; ++j) v[j] = j == at ? -INFINITY : v[j];
        }
    };
    TwoSums<true> sums;
    const float margin = 16.f / fmaxf(a.c, kLog2E);
    auto add_unit = [&](int i, int set, const Own& own) {
        if (i >= held) return;
        const int base = (held - 1 - i) * run + tn;
        float v[n];
        unpack_unit<kBf16>(raw[i], v);
        if (i == 0)
#pragma unroll
            for (int k = 0; k < n; ++k) v[k] = base + k < a.V ? v[k] : -INFINITY;
        if (kTail && ((own.units >> i) & 1)) {  // the listed ones are left out, of the maximum too
            int at = own.leave - i * n, k = (own.others >> i) & 1 ? own.k : -1;
            for (;;) {
#pragma unroll
                for (int j = 0; j < n; ++j) v[j] = j == at ? -INFINITY : v[j];
                if (k < 0) break;
                at = marks[set][k].kind & kListed ? marks[set][k].id - base : -1, k = after[set][k];
            }
        }
        sums.raise_past(max_of(v, sums.m), a.c, margin);
        float e[n], e1[n];
#pragma unroll
        for (int k = 0; k < n; ++k) {
            e[k] = exp2_fast(fmaf(v[k], a.c, -sums.r));
            if constexpr (kTwo) e1[k] = exp2_fast(fmaf(v[k], kLog2E, -sums.r1));
        }
        float s = e[0], s1 = kTwo ? e1[0] : 0.f;
#pragma unroll
        for (int k = 1; k < n; ++k) {
            s += e[k];
            if constexpr (kTwo) s1 += e1[k];
        }
        sums.s += s;
        if constexpr (kTwo) sums.s1 += s1;
    };
    int place = blockIdx.x, row = row_at(place), next = row_at(place += gridDim.x), set = 0;
    if (row >= a.rows) return;
    auto or_last = [&](int r) { return r < a.rows ? r : row; };
    Mark mark = request_mark(row), mark_ahead = request_mark(or_last(next));
#pragma unroll
    for (int i = 0; i < kHeld; ++i) request(buffer(logits_of(row), units), i);
    head[0][t] = -1;
    __syncthreads();
    keep_mark(0, mark);
    __syncthreads();
    Own own = own_marks(0);
#pragma unroll
    for (int i = 0; i < kHeld - kLag; ++i) add_unit(i, 0, own);
    for (;;) {
        const int ahead = or_last(next), after_next = row_at(place += gridDim.x);
        const RowList list = load_scalar(a.lists + row);
        const float scale = a.row_scale ? load_scalar(a.row_scale + row) : 1.f;
        head[set ^ 1][t] = -1;
#pragma unroll
        for (int i = kHeld - kLag; i < kHeld; ++i) add_unit(i, set, own);
        sums.settle(a.c);
        TwoSums<true> all = join_threads<kThreads>(sums, a.c, part);
        const bool wide = !(all.s < 3.0e38f && all.s1 < 3.0e38f);  // c m may have left fp32's range, or a value is no number
        if (wide && all.m > -INFINITY && all.m < INFINITY) {  // differences first
            TwoSums<true> again;
            again.m = all.m;
#pragma unroll 1
            for (int at = t * n; at < a.V; at += run) {
                float v[n];
                load_values<kBf16>(logits_of(row), at, a.V, v);
                if (kTail) leave_out(set, at, v);
#pragma unroll
                for (int k = 0; k < n; ++k) {
                    again.s += exp2_fast((v[k] - all.m) * a.c);
                    again.s1 += kTwo ? exp2_fast((v[k] - all.m) * kLog2E) : 0.f;
                }
            }
            __syncthreads();
            all = join_threads<kThreads>(again, a.c, part);
        }
        keep_mark(set ^ 1, mark_ahead);  // the heads were cleared before join_threads' barriers
        if (t < 64) {
            const RowFactors r = end_row(a, row, list, marks[set], all.m, all.s, all.s1, scale, true);
            for (int k = t; k <= a.K; k += 64) mark_gradient[k] = marked(a, r, marks[set][k]);
            if (t == 0) shared = r;
        }
        __syncthreads();
        const RowFactors r = shared;
        const Own own_next = own_marks(set ^ 1);
        const float own_gradient = mark_gradient[max(own.k, 0)];
        float f = kTwo ? r.f : r.f + r.f1, f1 = kTwo ? r.f1 : 0.f;
        const bool zero = f == 0.f && f1 == 0.f;  // nothing off the list
        char* const out = reinterpret_cast<char*>(a.dlogits) + row * a.ldd * elem_size<kBf16>();
        const __amdgpu_buffer_rsrc_t logits_ahead = buffer(logits_of(ahead), units), gradients_of = buffer(out, whole);
        sums = TwoSums<true>();
        mark_ahead = request_mark(or_last(after_next));  // before the stores: waiting for it is waiting for what was asked before
        if (wide || zero) {
#pragma unroll 1
            for (int at = t * n; at < a.V; at += run) {
                float v[n];
                load_values<kBf16>(logits_of(row), at, a.V, v);
                gradients<kBf16, true>(a, r.m, f, f1, v);
                u32x4 w = pack_unit<kBf16>(v);
                if (zero) w = u32x4{0, 0, 0, 0};
                store_unit<kBf16>(out, at, a.V, w);
            }
            __syncthreads();  // the marked tokens' gradients go over what was written there
            for (int k = t; k <= a.K; k += kThreads) {
                const int id = r.p == 0.f && r.label == 0.f ? -1 : marks[set][k].id;
                if (id < 0) continue;
                if constexpr (kBf16) reinterpret_cast<bf16_t*>(out)[id] = f32_to_bf16(mark_gradient[k]);
                else reinterpret_cast<float*>(out)[id] = mark_gradient[k];
            }
            if (next >= a.rows) return;
#pragma unroll
            for (int i = 0; i < kHeld; ++i) request(logits_ahead, i);
#pragma unroll 1
            for (int once = 0; once < 1; ++once)
#pragma unroll
                for (int i = 0; i < kHeld - kLag; ++i) add_unit(i, set ^ 1, own_next);
        } else {
            // exponents against c m rounded, what that is off in the factor
            const float R = r.m * a.c, R1 = r.m * kLog2E;
            f *= exp2_fast(-fmaf(r.m, a.c, -R)), f1 *= exp2_fast(-fmaf(r.m, kLog2E, -R1));
            // without this the compiler keeps what it took apart, and compared, for the sums, which no registers hold
            asm volatile("" : "+v"(tn));
#pragma unroll
            for (int i = 0; i < kHeld; ++i) asm volatile("" : "+v"(raw[i]));
#pragma unroll
            for (int i = 0; i < kHeld; ++i) {
                u32x4 w{};
                const int base = (held - 1 - i) * run + tn;
                if (i < held) {
                    float v[n];
                    unpack_unit<kBf16>(raw[i], v);
                    if (kTwo) {
#pragma unroll
                        for (int k = 0; k < n; ++k)
                            v[k] = fmaf(f1, exp2_fast(fmaf(v[k], kLog2E, -R1)), f * exp2_fast(fmaf(v[k], a.c, -R)));
                    } else {
#pragma unroll
                        for (int k = 0; k < n; ++k) v[k] = f * exp2_fast(fmaf(v[k], a.c, -R));
                    }
                    w = pack_unit<kBf16>(v);
                    if ((own.units >> i) & 1) {
                        int at = own.at - i * n, k = (own.others >> i) & 1 ? own.k : -1;
                        float g = own_gradient;
                        for (;;) {  // at outside [0, n): nothing
                            if constexpr (kBf16) {
                                const uint32_t bits = (uint32_t)f32_to_bf16(g) << (16 * (at & 1)), mask = 0xffffu << (16 * (at & 1));
#pragma unroll
                                for (int j = 0; j < 4; ++j) w[j] = j == at >> 1 ? (w[j] & ~mask) | bits : w[j];
                            } else {
#pragma unroll
                                for (int j = 0; j < 4; ++j) w[j] = j == at ? __float_as_uint(g) : w[j];
                            }
                            if (k < 0) break;
                            at = marks[set][k].id - base, g = mark_gradient[k], k = after[set][k];
                        }
                    }
                }
                if (i == 0 && base / n == whole && base < a.V) store_unit<kBf16>(out, base, a.V, w);
                __builtin_amdgcn_raw_buffer_store_b128(w, gradients_of, offset(i), 0, 0);
                request(logits_ahead, i);
                if (i >= kLag) add_unit(i - kLag, set ^ 1, own_next);
            }
            if (next >= a.rows) return;
        }
        row = next, next = after_next;
        set ^= 1;
        own = own_next;
    }
}

bool misaligned(const void* p, uintptr_t mask) { return ((uintptr_t)p & mask) != 0; }

constexpr int kMaxV = 1 << 21;

int check_distill(const flexmoe_distill_desc* D, int rows, const char* who, long long* ld, long long* ldd) {
    if (!D) return fail(FLEXMOE_EINVAL, "%s: desc is NULL", who);
    if (D->dtype != FLEXMOE_F32 && D->dtype != FLEXMOE_BF16)
        return fail(FLEXMOE_EDTYPE, "%s: dtype %d is neither FLEXMOE_F32 nor FLEXMOE_BF16", who, D->dtype);
    if (D->V < 1 || D->V > kMaxV) return fail(FLEXMOE_ESHAPE, "%s: V = %d outside [1, 2^21]", who, D->V);
    if (D->top < 1 || D->top > kMaxTop) return fail(FLEXMOE_ESHAPE, "%s: top = %d outside [1, %d]", who, D->top, kMaxTop);
    if (D->max_rows < 0 || D->max_rows > (1 << 24)) return fail(FLEXMOE_ESHAPE, "%s: max_rows = %d outside [0, 2^24]", who, D->max_rows);
    if (!(D->temperature >= 1e-6f && D->temperature <= 1e6f))
        return fail(FLEXMOE_EINVAL, "%s: temperature = %g outside [1e-6, 1e6]", who, (double)D->temperature);
    if (D->tail != 0 && D->tail != 1) return fail(FLEXMOE_EINVAL, "%s: tail must be 0 or 1 (got %d)", who, D->tail);
    if (!std::isfinite(D->kl_weight) || !std::isfinite(D->ce_weight)) return fail(FLEXMOE_EINVAL, "%s: weights must be finite", who);
    const int unit = D->dtype == FLEXMOE_BF16 ? 8 : 4;
    *ld = D->ld ? D->ld : D->V;
    *ldd = D->ldd ? D->ldd : D->V;
    for (long long s : {*ld, *ldd})
        if (s < D->V || s > 2LL * kMaxV || s % unit)
            return fail(FLEXMOE_ESHAPE, "%s: ld, ldd = %lld must be a multiple of %d in [V = %d, 2^22]", who, s, unit, D->V);
    if (rows < 0) return fail(FLEXMOE_EINVAL, "%s: rows = %d is negative", who, rows);
    if (rows > D->max_rows) return fail(FLEXMOE_ESHAPE, "%s: rows = %d above max_rows = %d", who, rows, D->max_rows);
    return FLEXMOE_OK;
}

int unit_run(int dtype) { return dtype == FLEXMOE_BF16 ? Vocab<true>::run : Vocab<false>::run; }

constexpr int kComputeUnits = 256;
// Workgroups of parts of rows, while there are few: 131072 tokens in bf16, losses and with the gradient, 16 rows 7.3 and
// 9.1 us with 256, 7.7 and 10.0 with 512, 9.2 and 11.8 with 2048; 200 rows 13.9 and 29.8, 15.6 and 31.7, 16.5 and 31.8.
constexpr int kWanted = 256;

struct DistillLayout {
    size_t lists, marks, order, counts, total;
};

DistillLayout distill_layout(const flexmoe_distill_desc* D, int rows) {
    auto up = [](size_t n) { return (n + 255) & ~size_t(255); };
    const size_t parts = most_parts(rows, D->V, kWanted);
    DistillLayout L;
    L.lists = up(parts * 16);
    L.marks = L.lists + up((size_t)rows * sizeof(RowList));
    L.order = L.marks + up((size_t)rows * (D->top + 1) * sizeof(Mark));
    L.counts = L.order + up((size_t)rows * sizeof(int32_t));
    L.total = L.counts + up((size_t)(rows + kOrder - 1) / kOrder * sizeof(int32_t)) + 256;
    return L;
}

// Workgroups that are at work together.
int whole_grid(int threads, int held) { return kComputeUnits * waves_of(held) * 256 / threads; }

template <bool kBf16, int kThreads, int kHeld>
hipError_t launch_whole(const DistillArgs& a, hipStream_t s) {
    distill_list_kernel<kBf16><<<a.row_scale ? a.rows : (a.rows + 3) / 4, kOrder, 0, s>>>(a);
    const int grid = std::min(a.rows, whole_grid(kThreads, kHeld));
    if (a.tail && a.two) distill_whole_kernel<kBf16, kThreads, kHeld, true, true><<<grid, kThreads, 0, s>>>(a);
    else if (a.tail) distill_whole_kernel<kBf16, kThreads, kHeld, true, false><<<grid, kThreads, 0, s>>>(a);
    else if (a.two) distill_whole_kernel<kBf16, kThreads, kHeld, false, true><<<grid, kThreads, 0, s>>>(a);
    else distill_whole_kernel<kBf16, kThreads, kHeld, false, false><<<grid, kThreads, 0, s>>>(a);
    return hipGetLastError();
}

// Whether rows are held whole by workgroups of `threads` times `held` units.  One read
// pays where the second one would not find the logits in the last cache: from 96 MB of
// them on (131072 tokens in bf16, 256, 512, 1024, 4096 rows: 52, 73, 129, 429 us against
// 37, 66, 167, 638 in parts; 32000 tokens, 1024, 2048, 4096 rows: 36, 60, 121 against 38,
// 71, 176; 50001 in fp32, 512, 1024, 4096: 52, 103, 353 against 53, 119, 537); of rows
// that are long beside what is done once for each (16384 rows in bf16 of 5000 tokens 162
// against 129, of 12800 227 against 300; with a tail, labels and a temperature 12800 tokens
// 329 against 287, 32000 tokens 528 against 682); and unless the last round of workgroups
// leaves many idle.
bool holds(const DistillArgs& a, int n, int threads, int held) {
    const size_t row = (size_t)a.V * 16 / n;
    if (!a.dlogits || a.V > threads * held * n || row * a.rows < (96u << 20) || row < (a.tail || a.two ? 48u << 10 : 24u << 10)) return false;
    const long long grid = whole_grid(threads, held), rounds = (a.rows + grid - 1) / grid;
    return 4 * rounds * grid <= 5LL * a.rows;
}

template <bool kBf16>
hipError_t launch_distill(const DistillArgs& a, hipStream_t s) {
    constexpr int n = Vocab<kBf16>::n;
    if (holds(a, n, 256, 16)) return launch_whole<kBf16, 256, 16>(a, s);
    if (holds(a, n, 256, 32)) return launch_whole<kBf16, 256, 32>(a, s);
    if (holds(a, n, 512, 32)) return launch_whole<kBf16, 512, 32>(a, s);
    const unsigned parts = (unsigned)a.rows * a.P, grid = parts + (a.rows + 3) / 4;
    if (a.tail && a.two) distill_sums_kernel<kBf16, true, true><<<grid, kVT, 0, s>>>(a);
    else if (a.tail) distill_sums_kernel<kBf16, true, false><<<grid, kVT, 0, s>>>(a);
    else if (a.two) distill_sums_kernel<kBf16, false, true><<<grid, kVT, 0, s>>>(a);
    else distill_sums_kernel<kBf16, false, false><<<grid, kVT, 0, s>>>(a);
    if (!a.dlogits) distill_row_kernel<<<(a.rows + 3) / 4, 256, 0, s>>>(a);
    else if (a.two) distill_grad_kernel<kBf16, true><<<parts, kVT, 0, s>>>(a);
    else distill_grad_kernel<kBf16, false><<<parts, kVT, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

extern "C" {

size_t flexmoe_distill_workspace_bytes(const flexmoe_distill_desc* desc, int32_t rows) {
    long long ld, ldd;
    if (check_distill(desc, rows, "distill_workspace_bytes", &ld, &ldd)) return 0;
    return distill_layout(desc, rows).total;
}

int flexmoe_distill(const flexmoe_distill_desc* desc, int32_t rows, const void* logits, const int32_t* ids, const float* logprobs,
                    const int32_t* labels, const float* row_scale, float* kl, float* ce, void* dlogits, void* workspace,
                    size_t workspace_bytes, void* stream) {
    const char* who = "distill";
    long long ld, ldd;
    const int rc = check_distill(desc, rows, who, &ld, &ldd);
    if (rc) return rc;
    if (rows == 0) return FLEXMOE_OK;
    if (!logits || !ids || !logprobs || !kl || !ce) return fail(FLEXMOE_EINVAL, "%s: a pointer is NULL", who);
    if (dlogits == logits && ld != ldd) return fail(FLEXMOE_EINVAL, "%s: gradients in the place of the logits need their stride", who);
    if (misaligned(logits, 15) || misaligned(dlogits, 15)) return fail(FLEXMOE_EINVAL, "%s: logits and gradients must be 16-byte aligned", who);
    for (const void* p : {(const void*)ids, (const void*)logprobs, (const void*)labels, (const void*)row_scale, (const void*)kl, (const void*)ce})
        if (misaligned(p, 3)) return fail(FLEXMOE_EINVAL, "%s: lists, labels, scales and losses must be 4-byte aligned", who);
    const DistillLayout L = distill_layout(desc, rows);
    if (!workspace || workspace_bytes < L.total)
        return fail(FLEXMOE_EWORKSPACE, "%s: workspace of %zu bytes, %zu needed", who, workspace ? workspace_bytes : 0, L.total);
    if (misaligned(workspace, 255)) return fail(FLEXMOE_EWORKSPACE, "%s: workspace must be 256-byte aligned", who);
    DistillArgs a;
    a.logits = logits, a.ids = ids, a.labels = labels, a.lp = logprobs, a.row_scale = row_scale, a.kl = kl, a.ce = ce, a.dlogits = dlogits;
    char* const ws = (char*)workspace;
    a.parts = (float*)ws, a.lists = (RowList*)(ws + L.lists), a.marks = (Mark*)(ws + L.marks);
    a.order = (int32_t*)(ws + L.order), a.counts = (int32_t*)(ws + L.counts);  // of a launch's rows
    a.ld = (size_t)ld, a.ldd = (size_t)ldd, a.V = desc->V, a.K = desc->top, a.tail = desc->tail;
    a.P = row_parts(rows, desc->V, unit_run(desc->dtype), kWanted);
    a.length = part_length(desc->V, a.P, unit_run(desc->dtype));
    a.two = labels && desc->temperature != 1.f;
    a.t = desc->temperature, a.inv_t = 1.0 / desc->temperature, a.c = (float)(1.4426950408889634 / desc->temperature);
    a.kl_weight = desc->kl_weight, a.ce_weight = desc->ce_weight;
    const bool bf16 = desc->dtype == FLEXMOE_BF16;
    const size_t es = bf16 ? 2 : 4;
    const int slice = (1 << 23) / a.P;  // a launch's threads are fewer than 2^32
    for (int done = 0; done < rows; done += slice) {
        const int n = a.rows = std::min(slice, rows - done);
        const hipError_t err = bf16 ? launch_distill<true>(a, (hipStream_t)stream) : launch_distill<false>(a, (hipStream_t)stream);
        if (err != hipSuccess) return hip_fail(err, who);
        a.logits = (const char*)a.logits + (size_t)n * ld * es;
        if (a.dlogits) a.dlogits = (char*)a.dlogits + (size_t)n * ldd * es;
        a.ids += (size_t)n * a.K, a.lp += (size_t)n * a.K, a.kl += n, a.ce += n;
        if (labels) a.labels += n;
        if (row_scale) a.row_scale += n;
        a.parts += (size_t)4 * n * a.P, a.lists += n, a.marks += (size_t)n * (a.K + 1);
    }
    return FLEXMOE_OK;
}

}  // extern "C"
