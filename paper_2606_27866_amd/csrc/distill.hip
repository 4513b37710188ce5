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
// the listed tokens are left out of that sum (a map of bits says which) and added
// to it afterwards, so that q_rest is a sum and not a difference.
//
//   distill_sums_kernel   maximum and sums of each part of a row
//   distill_row_kernel    a wave joins them: losses, factors, gradients of the listed tokens
//   distill_grad_kernel   factor * exp(x) for a part of a row, then the listed tokens
#include <algorithm>
#include <cmath>

#include "error.h"
#include "flexmoe.h"
#include "vocab.h"

using namespace flexmoe;

namespace {

struct DistillArgs {
    const void* logits;
    const int32_t *ids, *labels;
    const float *lp, *row_scale;
    float *kl, *ce;
    void* dlogits;
    float* parts;     // [rows][P][4]: m, sum at t, sum at 1
    float* factors;   // [rows][4]: m, factor at t, factor at 1
    int2* marks;      // [rows][K + 1]: token (-1: none), bits of its gradient
    size_t ld, ldd;
    int V, P, length, K, tail, two;  // two: the labels' sum is not that of t
    float c, inv_t, t, kl_weight, ce_weight;
};

constexpr float kLog2E = 1.4426950408889634f;

// Sums at t and, where they differ, at 1, while the largest value is still growing.
template <bool kTwo>
struct TwoSums {
    float m = -INFINITY, s = 0.f, r = 0.f, s1 = 0.f, r1 = 0.f;

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

template <bool kTwo>
__device__ __forceinline__ TwoSums<kTwo> join_threads(TwoSums<kTwo> a, float c, float (*part)[kVT / 64]) {
    const int wave = threadIdx.x >> 6;
    float m = wave_max(a.m);
    if ((threadIdx.x & 63) == 0) part[0][wave] = m;
    __syncthreads();
    m = part[0][0];
#pragma unroll
    for (int w = 1; w < kVT / 64; ++w) m = fmaxf(m, part[0][w]);
    a.refer(m, c);
    a.s = wave_total_f(a.s);
    if constexpr (kTwo) a.s1 = wave_total_f(a.s1);
    if ((threadIdx.x & 63) == 0) part[1][wave] = a.s, part[2][wave] = a.s1;
    __syncthreads();
    a.s = part[1][0], a.s1 = part[2][0];
#pragma unroll
    for (int w = 1; w < kVT / 64; ++w) a.s += part[1][w], a.s1 += part[2][w];
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

template <bool kBf16, bool kTail, bool kTwo>
__global__ __launch_bounds__(kVT) void distill_sums_kernel(const DistillArgs a) {
    using W = Vocab<kBf16>;
    __shared__ uint32_t bits[kTail ? kRange / 32 : 1];
    __shared__ float part[3][kVT / 64];
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
        for (int u = 0; u < W::units; ++u) gm = max_of(v[u], gm);
        sums.raise(gm, a.c);
#pragma unroll
        for (int u = 0; u < W::units; ++u) {
            const int i = at + u * W::run + t * W::n;
            if constexpr (kTail)
                if (i < end) leave_out<kBf16>(bits, i - begin, v[u]);
#pragma unroll
            for (int k = 0; k < W::n; ++k) sums.add(v[u][k], a.c);
        }
    });
    sums.settle(a.c);
    TwoSums<kTwo> all = join_threads(sums, a.c, part);
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
        all = join_threads(again, a.c, part);
    }
    if (t == 0) {
        float* const o = a.parts + 4 * (row * a.P + p);
        o[0] = all.m, o[1] = all.s, o[2] = all.s1;
    }
}

__device__ __forceinline__ double wave_sum_d(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

constexpr int kOwn = kMaxTop / 64;  // listed tokens of a lane

// One wave ends a row whose largest logit is m and whose sums (with a tail: without
// the listed tokens) are s and s1.  seen: K + 1 ints of LDS.
template <bool kBf16>
__device__ void end_row(const DistillArgs& a, size_t row, const void* logits, float m, float s, float s1, int* seen) {
    const int lane = threadIdx.x & 63, K = a.K;
    const double scale = a.row_scale ? (double)a.row_scale[row] : 1.0, inv_t = (double)a.inv_t;
    const int32_t* const ids = a.ids + row * K;
    const int label = a.labels ? a.labels[row] : -1;
    const bool labelled = label >= 0 && label < a.V;
    int id[kOwn];
    float lp[kOwn];
#pragma unroll
    for (int q = 0; q < kOwn; ++q) {
        const int k = lane + 64 * q;
        id[q] = k < K ? ids[k] : -1;
        lp[q] = k < K ? a.lp[row * K + k] : -INFINITY;
        if (id[q] < 0 || id[q] >= a.V) id[q] = -1;
        if (k < K) seen[k] = id[q];
    }
    __builtin_amdgcn_wave_barrier();
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    // a token that is named again counts with its first place alone
    bool again[kOwn] = {}, label_listed = false;
    for (int j = 0; j < K; ++j) {
        const int other = seen[j];
#pragma unroll
        for (int q = 0; q < kOwn; ++q) again[q] |= other == id[q] && j < lane + 64 * q;
        label_listed |= other == label;
    }
    __builtin_amdgcn_wave_barrier();
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    double e[kOwn], e1[kOwn], logq[kOwn], p[kOwn], logp[kOwn];
    double listed = 0.0, listed1 = 0.0;
    bool nan = false;
#pragma unroll
    for (int q = 0; q < kOwn; ++q) {
        if (again[q]) id[q] = -1;
        const double x = id[q] >= 0 ? (double)value_at<kBf16>(logits, id[q]) - (double)m : -INFINITY;
        nan |= id[q] >= 0 && __builtin_isnan(value_at<kBf16>(logits, id[q]));
        logq[q] = x * inv_t;
        e[q] = id[q] >= 0 ? exp(logq[q]) : 0.0;
        e1[q] = !a.two ? e[q] : id[q] >= 0 ? exp(x) : 0.0;
        listed += e[q];
        listed1 += e1[q];
    }
    double S = (double)s, S1 = a.two ? (double)s1 : S;
    if (a.tail) {
        S += wave_sum_d(listed);
        S1 = a.two ? S1 + wave_sum_d(listed1) : S;
    }
    const bool empty = m == -INFINITY && s == 0.f && !__any(nan);
    // the teacher
    double mass = 0.0, rest = 0.0, kl = 0.0;
    if (a.tail) {
#pragma unroll
        for (int q = 0; q < kOwn; ++q) {
            logp[q] = id[q] >= 0 ? (double)lp[q] : -INFINITY;
            p[q] = exp(logp[q]);
            mass += p[q];
        }
        mass = wave_sum_d(mass);
        rest = mass != mass ? mass : fmax(0.0, 1.0 - mass);
    } else {
        float top = -INFINITY;
#pragma unroll
        for (int q = 0; q < kOwn; ++q)
            if (id[q] >= 0) top = fmaxf(top, lp[q]);
        top = wave_max(top);
#pragma unroll
        for (int q = 0; q < kOwn; ++q) {
            logp[q] = id[q] >= 0 && top > -INFINITY ? (double)lp[q] - (double)top : -INFINITY;
            p[q] = exp(logp[q]);
            mass += p[q];
        }
        mass = wave_sum_d(mass);
        const double log_mass = log(mass);
#pragma unroll
        for (int q = 0; q < kOwn; ++q) {
            p[q] = p[q] == 0.0 ? 0.0 : p[q] / mass;
            logp[q] -= log_mass;
        }
        if (mass > 0.0) mass = 1.0;
    }
    const double log_s = log(S), total = mass + rest;
#pragma unroll
    for (int q = 0; q < kOwn; ++q) {
        logq[q] -= log_s;
        if (p[q] != 0.0) kl += p[q] * (logp[q] - logq[q]);
    }
    kl = wave_sum_d(kl);
    double dense = total;
    if (a.tail && rest != 0.0) {
        const double q_rest = (double)s / S;
        // log probabilities in 32 bits leave about 1e-6 of their own
        if (s == 0.f) kl += rest <= 1e-5 ? 0.0 : INFINITY;
        else kl += rest * (log(rest) - log(q_rest));
        dense = s == 0.f ? 0.0 : total - rest / q_rest;
    }
    if (empty) kl = mass > 0.0 || rest > 1e-5 ? INFINITY : 0.0;
    const double x_label = labelled ? (double)value_at<kBf16>(logits, label) - (double)m : 0.0;
    const double ce = !labelled ? 0.0 : empty ? INFINITY : log(S1) - x_label;
    if (lane == 0) {
        a.kl[row] = (float)kl;
        a.ce[row] = (float)ce;
    }
    if (!a.dlogits) return;
    const double by_kl = scale * (double)a.kl_weight * (double)a.t, by_ce = labelled ? scale * (double)a.ce_weight : 0.0;
    const double f = by_kl * dense / S, f1 = by_ce / S1;
    if (lane == 0) {
        float* const o = a.factors + 4 * row;
        o[0] = m;
        o[1] = empty ? 0.f : (float)(a.two ? f : f + f1);
        o[2] = empty || !a.two ? 0.f : (float)f1;
    }
    int2* const marks = a.marks + row * (K + 1);
#pragma unroll
    for (int q = 0; q < kOwn; ++q) {
        const int k = lane + 64 * q;
        if (k >= K) continue;
        double g = by_kl * (total * e[q] / S - p[q]) + f1 * e1[q];
        if (id[q] == label) g -= by_ce;
        marks[k] = make_int2(empty ? -1 : id[q], __float_as_int((float)g));
    }
    if (lane == 0) {
        const double g = f * exp(x_label * inv_t) + f1 * exp(x_label) - by_ce;
        marks[K] = make_int2(!labelled || label_listed || empty ? -1 : label, __float_as_int((float)g));
    }
}

template <bool kBf16>
__global__ __launch_bounds__(64) void distill_row_kernel(const DistillArgs a) {
    __shared__ int seen[kMaxTop + 1];
    const size_t row = blockIdx.x;
    if (a.row_scale && a.row_scale[row] == 0.f) {
        if (threadIdx.x == 0) {
            a.kl[row] = a.ce[row] = 0.f;
            if (a.dlogits) a.factors[4 * row + 1] = a.factors[4 * row + 2] = 0.f;
        }
        if (a.dlogits)
            for (int k = threadIdx.x; k <= a.K; k += 64) a.marks[row * (a.K + 1) + k] = make_int2(-1, 0);
        return;
    }
    const float* const parts = a.parts + 4 * row * a.P;
    TwoSums<true> all;
    for (int p = 0; p < a.P; ++p) all.m = fmaxf(all.m, parts[4 * p]);
    for (int p = 0; p < a.P; ++p) {
        TwoSums<true> one;
        one.m = parts[4 * p], one.s = parts[4 * p + 1], one.s1 = parts[4 * p + 2];
        one.refer(all.m, a.c);
        all.s += one.s;
        all.s1 += one.s1;
    }
    end_row<kBf16>(a, row, reinterpret_cast<const char*>(a.logits) + row * a.ld * elem_size<kBf16>(), all.m, all.s, all.s1, seen);
}

template <bool kBf16, bool kTwo>
__global__ __launch_bounds__(kVT) void distill_grad_kernel(const DistillArgs a) {
    using W = Vocab<kBf16>;
    const size_t row = blockIdx.x / a.P;
    const int p = blockIdx.x % a.P, t = threadIdx.x;
    const char* const logits = reinterpret_cast<const char*>(a.logits) + row * a.ld * elem_size<kBf16>();
    char* const out = reinterpret_cast<char*>(a.dlogits) + row * a.ldd * elem_size<kBf16>();
    const int begin = p * a.length, end = min(a.V, begin + a.length);
    const float m = a.factors[4 * row], f = a.factors[4 * row + 1], f1 = kTwo ? a.factors[4 * row + 2] : 0.f;
    auto write = [&](int i, const u32x4& w) {
        if (i + W::n <= end) {
            *reinterpret_cast<u32x4*>(out + (size_t)i * elem_size<kBf16>()) = w;
        } else {
#pragma unroll
            for (int k = 0; k < W::n - 1; ++k)
                if (i + k < end) {
                    if constexpr (kBf16) reinterpret_cast<bf16_t*>(out)[i + k] = (bf16_t)(w[k >> 1] >> (16 * (k & 1)));
                    else reinterpret_cast<uint32_t*>(out)[i + k] = w[k];
                }
        }
    };
    const bool zero = f == 0.f && f1 == 0.f;  // padding, which is not read, or nothing off the list
    if (zero)
        for (int i = begin + t * W::n; i < end; i += W::run) write(i, u32x4{0, 0, 0, 0});
    each_step<kBf16>(logits, begin, zero ? begin : end, [&](int, int at, float (&v)[W::units][W::n]) {
#pragma unroll
        for (int u = 0; u < W::units; ++u) {
            const int i = at + u * W::run + t * W::n;
#pragma unroll
            for (int k = 0; k < W::n; ++k) {
                float g = f * exp2_fast((v[u][k] - m) * a.c);
                if constexpr (kTwo) g = fmaf(f1, exp2_fast((v[u][k] - m) * kLog2E), g);
                v[u][k] = g;
            }
            u32x4 w;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if constexpr (kBf16) w[k] = pack_bf16x2(v[u][2 * k], v[u][2 * k + 1]);
                else w[k] = __float_as_uint(v[u][k]);
            }
            if (i < end) write(i, w);
        }
    });
    __syncthreads();  // the listed tokens' gradients go over what was written there
    for (int k = t; k <= a.K; k += kVT) {
        const int2 mark = a.marks[row * (a.K + 1) + k];
        if (mark.x < begin || mark.x >= end) continue;
        const float g = __int_as_float(mark.y);
        if constexpr (kBf16) reinterpret_cast<bf16_t*>(out)[mark.x] = f32_to_bf16(g);
        else reinterpret_cast<float*>(out)[mark.x] = g;
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

struct DistillLayout {
    size_t factors, marks, total;
};

DistillLayout distill_layout(const flexmoe_distill_desc* D, int rows) {
    auto up = [](size_t n) { return (n + 255) & ~size_t(255); };
    const size_t least = (D->V + kRange - 1) / kRange;
    const size_t parts = std::max<size_t>(rows * least, std::min<size_t>((size_t)std::min(rows, kWantedWorkgroups) * std::max(1, D->V / kLeastRange),
                                                                         2 * kWantedWorkgroups));
    DistillLayout L;
    L.factors = up(parts * 16);
    L.marks = L.factors + up((size_t)rows * 16);
    L.total = L.marks + up((size_t)rows * (D->top + 1) * 8) + 256;
    return L;
}

template <bool kBf16>
hipError_t launch_distill(const DistillArgs& a, int rows, hipStream_t s) {
    const unsigned grid = (unsigned)rows * a.P;
    if (a.tail && a.two) distill_sums_kernel<kBf16, true, true><<<grid, kVT, 0, s>>>(a);
    else if (a.tail) distill_sums_kernel<kBf16, true, false><<<grid, kVT, 0, s>>>(a);
    else if (a.two) distill_sums_kernel<kBf16, false, true><<<grid, kVT, 0, s>>>(a);
    else distill_sums_kernel<kBf16, false, false><<<grid, kVT, 0, s>>>(a);
    distill_row_kernel<kBf16><<<rows, 64, 0, s>>>(a);
    if (a.dlogits) {
        if (a.two) distill_grad_kernel<kBf16, true><<<grid, kVT, 0, s>>>(a);
        else distill_grad_kernel<kBf16, false><<<grid, kVT, 0, s>>>(a);
    }
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
    a.parts = (float*)ws, a.factors = (float*)(ws + L.factors), a.marks = (int2*)(ws + L.marks);
    a.ld = (size_t)ld, a.ldd = (size_t)ldd, a.V = desc->V, a.K = desc->top, a.tail = desc->tail;
    a.P = row_parts(rows, desc->V, unit_run(desc->dtype));
    a.length = part_length(desc->V, a.P, unit_run(desc->dtype));
    a.two = labels && desc->temperature != 1.f;
    a.t = desc->temperature, a.inv_t = (float)(1.0 / desc->temperature), a.c = (float)(1.4426950408889634 / desc->temperature);
    a.kl_weight = desc->kl_weight, a.ce_weight = desc->ce_weight;
    const bool bf16 = desc->dtype == FLEXMOE_BF16;
    const size_t es = bf16 ? 2 : 4;
    const int slice = (1 << 23) / a.P;  // a launch's threads are fewer than 2^32
    for (int done = 0; done < rows; done += slice) {
        const int n = std::min(slice, rows - done);
        const hipError_t err = bf16 ? launch_distill<true>(a, n, (hipStream_t)stream) : launch_distill<false>(a, n, (hipStream_t)stream);
        if (err != hipSuccess) return hip_fail(err, who);
        a.logits = (const char*)a.logits + (size_t)n * ld * es;
        if (a.dlogits) a.dlogits = (char*)a.dlogits + (size_t)n * ldd * es;
        a.ids += (size_t)n * a.K, a.lp += (size_t)n * a.K, a.kl += n, a.ce += n;
        if (labels) a.labels += n;
        if (row_scale) a.row_scale += n;
        a.parts += (size_t)4 * n * a.P, a.factors += (size_t)4 * n, a.marks += (size_t)n * (a.K + 1);
    }
    return FLEXMOE_OK;
}

}  // extern "C"
