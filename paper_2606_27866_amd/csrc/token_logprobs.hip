// Log probabilities of given tokens, entropy and the most likely tokens of rows
// of logits (gfx950), in one pass over the logits.
//
//   x = l / temperature       lse = log sum exp x        logprob = x_token - lse
//   entropy = lse - sum p x   top: the K largest l, ties to the lower id
//
// Every thread keeps the maximum and the sums of its values, and the maximum of
// each group of 32 of them in LDS.  The K-th largest of the threads' maxima is a
// bound that at least K values reach; the few groups that reach it are read
// again (from the caches, all at once) for the values that do, and those are ranked
// by counting.  Where ties or an unlucky order leave more candidates than their
// buffer holds, the K-th largest (value, place) is found digit by digit in
// further passes over the row, which is exact for any input.
//
// Rows are split over workgroups while there are few; a second launch joins the
// parts' sums and lists.
//
// Bound by memory where rows are many: 4096 x 131072 bf16, 32 listed, 198 us, 5.4 TB/s
// (128 listed 226, none 191).  One row is two launches and the latency of their chains of
// loads, barriers and ranks: 11.4 us with 20 listed.
#include <algorithm>
#include <cmath>

#include "error.h"
#include "flexmoe.h"
#include "vocab.h"

using namespace flexmoe;

namespace {

constexpr int kCandidates = 1024;
constexpr int kJoined = 8;        // keys of a thread that joins the parts' lists
constexpr int kMostKeys = kJoined * kVT;
static_assert(kMostKeys >= ((1 << 21) / kRange) * kMaxTop, "the lists of the longest row's parts");
// Workgroups while there are few rows: more parts are more to join.  131072 tokens in bf16, 20 listed, 8, 64 and 256 rows
// 11.6, 14.1 and 18.9 us with 256, 12.6, 13.4 and 22.7 with 512; 64 rows of 100003 in fp32, 64 listed, 16.8 with both, 20.7
// with 128, 23.4 with 2048.
constexpr int kWanted = 256;

struct LogprobArgs {
    const void* logits;
    const int32_t* tokens;
    float *logprob, *entropy, *lse;
    int32_t* top_ids;
    float* top_logprobs;
    float* parts;      // [rows][P][4]: m, s, h of each part of a row
    uint64_t* lists;   // [rows][P][K]: their largest, in order; 0 past their number
    size_t ld;
    int V, P, length, K;
    float c, inv_t;    // log2(e) / temperature, 1 / temperature
};

struct TopScratch {
    uint64_t list[kCandidates];
    uint32_t key[kVT];
    uint32_t bound;
    int count, items;
    int hist[256];
    uint64_t prefix;
    int left;
    uint16_t item[kCandidates];  // groups that reach the bound
};

// The K-th largest of the threads' keys by their upper halves (one wave): at least K of
// the keys reach it.
__device__ __forceinline__ uint32_t kth_key(const uint32_t* key, int K) {
    const int lane = threadIdx.x & 63;
    uint32_t k[kVT / 64], at = 0;
#pragma unroll
    for (int q = 0; q < kVT / 64; ++q) k[q] = key[lane + 64 * q];
#pragma unroll 4
    for (int bit = 31; bit >= 16; --bit) {
        const uint32_t trial = at | (1u << bit);
        int n = 0;
#pragma unroll
        for (int q = 0; q < kVT / 64; ++q) n += __popcll(__ballot(k[q] >= trial));
        if (n >= K) at = trial;
    }
    return at;
}

// The `want` largest of the candidates that each(f) hands out as f(key), in order, to
// put(rank, key).  `own`: the largest value's key of this thread's candidates;
// near(bound, f) hands out those whose value may reach the bound, by whichever thread.
template <typename Each, typename Near, typename Put>
__device__ __forceinline__ void top_of(TopScratch& ts, uint32_t own, int want, Each&& each, Near&& near, Put&& put) {
    ts.key[threadIdx.x] = own;
    if (threadIdx.x == 0) ts.count = ts.items = 0;
    __syncthreads();
    if (threadIdx.x < 64) {
        const uint32_t b = kth_key(ts.key, want);
        if (threadIdx.x == 0) ts.bound = b;
    }
    __syncthreads();
    const uint32_t bound = ts.bound;
    near(bound, [&](uint64_t k) {
        if ((uint32_t)(k >> 32) < bound) return;
        const int at = atomicAdd(&ts.count, 1);  // the order in the list does not matter: it is ranked
        if (at < kCandidates) ts.list[at] = k;
    });
    __syncthreads();
    if (ts.count < want || ts.count > kCandidates) {
        // digit by digit from the top: how many keys with the prefix so far have which next digit
        if (threadIdx.x == 0) ts.prefix = 0, ts.left = want;
        for (int shift = 56; shift >= 0; shift -= 8) {
            ts.hist[threadIdx.x] = 0;
            __syncthreads();
            const uint64_t prefix = ts.prefix;
            each([&](uint64_t k) {
                const bool in = shift == 56 || (k >> (shift + 8)) == (prefix >> (shift + 8));
                const int digit = (int)(k >> shift) & 255;
                // many equal values would meet in one counter: a wave that agrees adds once
                const uint64_t all = __ballot(1), with = __ballot(in);
                if (!with) return;
                const int first = __shfl(digit, __ffsll((unsigned long long)with) - 1, 64);
                if (__ballot(in && digit == first) == with) {
                    if ((int)(threadIdx.x & 63) == __ffsll((unsigned long long)all) - 1) atomicAdd(&ts.hist[first], (int)__popcll(with));
                } else if (in) {
                    atomicAdd(&ts.hist[digit], 1);
                }
            });
            __syncthreads();
            if (threadIdx.x < 64) {  // four digits a lane, the largest first
                const int lane = threadIdx.x, left = ts.left;
                int n[4], sum = 0;
#pragma unroll
                for (int q = 0; q < 4; ++q) sum += n[q] = ts.hist[255 - 4 * lane - q];
                const int upto = wave_incl_scan(sum);
                if (lane == __ffsll((unsigned long long)__ballot(upto >= left)) - 1) {
                    int rest = left - (upto - sum), q = 0;
                    while (q < 3 && n[q] < rest) rest -= n[q++];
                    ts.left = rest;
                    ts.prefix = prefix | ((uint64_t)(255 - 4 * lane - q) << shift);
                    ts.count = 0;
                }
            }
            __syncthreads();
        }
        const uint64_t least = ts.prefix;
        each([&](uint64_t k) {
            if (k < least) return;
            const int at = atomicAdd(&ts.count, 1);
            if (at < kCandidates) ts.list[at] = k;  // `want` keys: they all differ
        });
        __syncthreads();
    }
    const int n = min(ts.count, kCandidates);
    for (int i = threadIdx.x; i < n; i += kVT) {
        const uint64_t k = ts.list[i];
        int rank = 0;
#pragma unroll 8
        for (int j = 0; j < n; ++j) rank += ts.list[j] > k;
        if (rank < want) put(rank, k);
    }
}

// Sums of a workgroup's threads, in every thread.
__device__ __forceinline__ Sums join_threads(Sums t, float c, float (*part)[kVT / 64]) {
    const int wave = threadIdx.x >> 6;
    float m = wave_max(t.m);
    if ((threadIdx.x & 63) == 0) part[0][wave] = m;
    __syncthreads();
    m = part[0][0];
#pragma unroll
    for (int w = 1; w < kVT / 64; ++w) m = fmaxf(m, part[0][w]);
    t.refer(m, c);
    t.s = wave_total_f(t.s);
    t.h = wave_total_f(t.h);
    if ((threadIdx.x & 63) == 0) part[1][wave] = t.s, part[2][wave] = t.h;
    __syncthreads();
    t.s = part[1][0], t.h = part[2][0];
#pragma unroll
    for (int w = 1; w < kVT / 64; ++w) t.s += part[1][w], t.h += part[2][w];
    return t;
}

// A row's results from its sums.
struct RowEnd {
    float m, inv_t, log_s;
    bool empty;  // nothing but -inf
    __device__ __forceinline__ RowEnd(const Sums& t, float inv_t_) : m(t.m), inv_t(inv_t_), log_s(logf(t.s)), empty(t.s == 0.f) {}
    __device__ __forceinline__ float logprob(float x) const { return empty ? -INFINITY : (x - m) * inv_t - log_s; }
};

__device__ __forceinline__ void write_row(const LogprobArgs& a, size_t row, const Sums& t, const RowEnd& end, float token_logit) {
    a.lse[row] = end.empty ? -INFINITY : t.m * a.inv_t + end.log_s;
    a.entropy[row] = end.empty ? 0.f : end.log_s - t.h / t.s * 0.6931471805599453f;
    if (a.tokens) {
        const int tok = a.tokens[row];
        a.logprob[row] = tok < 0 || tok >= a.V ? 0.f : end.logprob(token_logit);
    }
}

template <bool kBf16>
__device__ __forceinline__ float token_logit(const LogprobArgs& a, size_t row, const void* logits) {
    if (!a.tokens) return 0.f;
    const int tok = a.tokens[row];
    return tok < 0 || tok >= a.V ? 0.f : value_at<kBf16>(logits, tok);
}

template <bool kBf16, bool kTop>
__global__ __launch_bounds__(kVT) void logprob_kernel(const LogprobArgs a) {
    using W = Vocab<kBf16>;
    __shared__ float group[kTop ? kRange / 32 : 1];
    __shared__ float part[3][kVT / 64];
    __shared__ TopScratch ts;
    const size_t row = blockIdx.x / a.P;
    const int p = blockIdx.x % a.P, t = threadIdx.x;
    const void* const logits = reinterpret_cast<const char*>(a.logits) + row * a.ld * elem_size<kBf16>();
    const int begin = p * a.length, end = min(a.V, begin + a.length);
    const float of_token = a.P == 1 ? token_logit<kBf16>(a, row, logits) : 0.f;  // on its way early
    RunningSums sums;
    each_step<kBf16>(logits, begin, end, [&](int it, int, const float (&v)[W::units][W::n]) {
        float gm = -INFINITY;
#pragma unroll
        for (int u = 0; u < W::units; ++u) gm = max_of(v[u], gm);
        if constexpr (kTop) group[it * kVT + t] = gm;
        sums.raise(gm, a.c);
#pragma unroll
        for (int u = 0; u < W::units; ++u)
#pragma unroll
            for (int k = 0; k < W::n; ++k) sums.add(v[u][k], a.c);
    });
    const uint32_t own = value_key(sums.t.m);
    Sums all = join_threads(sums.exact(a.c), a.c, part);
    if (!(all.s < 3.0e38f) && all.m > -INFINITY && all.m < INFINITY) {
        // c m may have left fp32's range (or a value is no number): differences first
        Sums again;
        again.m = all.m;
        for (int i = begin + t * W::n; i < end; i += W::run) {
            float v[W::n];
            load_values<kBf16>(logits, i, end, v);
#pragma unroll
            for (int k = 0; k < W::n; ++k) {
                const float d = (v[k] - all.m) * a.c, e = exp2_fast(d);
                again.s += e;
                again.h = fmaf(e, fmaxf(d, -200.f), again.h);
            }
        }
        __syncthreads();
        all = join_threads(again, a.c, part);
    }
    const RowEnd result(all, a.inv_t);
    if (t == 0) {
        if (a.P == 1) {
            write_row(a, row, all, result, of_token);
        } else {
            float* const o = a.parts + 4 * (row * a.P + p);
            o[0] = all.m, o[1] = all.s, o[2] = all.h;
        }
    }
    if constexpr (kTop) {
        const int want = min(a.K, end - begin);
        auto each = [&](auto&& f) {
            for (int i = begin + t * W::n; i < end; i += W::run) {
                float v[W::n];
                load_values<kBf16>(logits, i, end, v);
#pragma unroll
                for (int k = 0; k < W::n; ++k)
                    if (i + k < end) f(place_key(v[k], i + k));
            }
        };
        auto near = [&](uint32_t bound, auto&& f) {
            for (int at = begin, it = 0; at < end; at += W::step, ++it)
                if (value_key(group[it * kVT + t]) >= bound) {
                    const int i = atomicAdd(&ts.items, 1);
                    if (i < kCandidates) ts.item[i] = (uint16_t)(it * kVT + t);
                }
            __syncthreads();
            if (ts.items > kCandidates) {  // digit by digit
                if (t == 0) ts.count = kCandidates + 1;
                return;
            }
            for (int i = t / W::units; i < ts.items; i += kVT / W::units) {
                const int item = ts.item[i], at = begin + item / kVT * W::step + t % W::units * W::run + item % kVT * W::n;
                float v[W::n];
                load_values<kBf16>(logits, at, end, v);
#pragma unroll
                for (int k = 0; k < W::n; ++k)
                    if (at + k < end) f(place_key(v[k], at + k));
            }
        };
        uint64_t* const list = a.P > 1 ? a.lists + (row * a.P + p) * a.K : nullptr;
        top_of(ts, own, want, each, near, [&](int rank, uint64_t k) {
            if (list) {
                list[rank] = k;
            } else {
                a.top_ids[row * a.K + rank] = (int32_t)~(uint32_t)k;
                a.top_logprobs[row * a.K + rank] = result.logprob(key_value((uint32_t)(k >> 32)));
            }
        });
        if (list)
            for (int i = want + t; i < a.K; i += kVT) list[i] = 0;
    }
}

template <bool kBf16, bool kTop>
__global__ __launch_bounds__(kVT) void logprob_join_kernel(const LogprobArgs a) {
    __shared__ TopScratch ts;
    const size_t row = blockIdx.x;
    const int t = threadIdx.x;
    const void* const logits = reinterpret_cast<const char*>(a.logits) + row * a.ld * elem_size<kBf16>();
    const float* const parts = a.parts + 4 * row * a.P;
    const float of_token = token_logit<kBf16>(a, row, logits);  // on its way early
    uint64_t key[kJoined];
    const int keys = kTop ? a.P * a.K : 0;
    if constexpr (kTop) {
        const uint64_t* const lists = a.lists + row * a.P * a.K;
        // each list turned by some places, else a thread's keys would be of one rank, and the bound a poor one
#pragma unroll
        for (int j = 0; j < kJoined; ++j) {
            const int i = min(t + j * kVT, keys - 1), p = i / a.K;
            key[j] = lists[p * a.K + (i + 37 * p) % a.K];
        }
    }
    // every wave joins the sums, a part a lane
    Sums all;
    const int lane = t & 63;
    for (int p = lane; p < a.P; p += 64) all.m = fmaxf(all.m, parts[4 * p]);
    all.m = wave_max(all.m);
    for (int p = lane; p < a.P; p += 64) {
        Sums one;
        one.m = parts[4 * p], one.s = parts[4 * p + 1], one.h = parts[4 * p + 2];
        one.refer(all.m, a.c);
        all.s += one.s;
        all.h += one.h;
    }
    all.s = wave_total_f(all.s);
    all.h = wave_total_f(all.h);
    const RowEnd result(all, a.inv_t);
    if (t == 0) write_row(a, row, all, result, of_token);
    if constexpr (kTop) {
        uint32_t own = 0;
        auto each = [&](auto&& f) {
#pragma unroll
            for (int j = 0; j < kJoined; ++j)
                if (t + j * kVT < keys && key[j]) f(key[j]);  // 0: a part of fewer values
        };
        each([&](uint64_t k) { own = max(own, (uint32_t)(k >> 32)); });
        top_of(ts, own, a.K, each, [&](uint32_t, auto&& f) { each(f); }, [&](int rank, uint64_t k) {
            a.top_ids[row * a.K + rank] = (int32_t)~(uint32_t)k;
            a.top_logprobs[row * a.K + rank] = result.logprob(key_value((uint32_t)(k >> 32)));
        });
    }
}

bool misaligned(const void* p, uintptr_t mask) { return ((uintptr_t)p & mask) != 0; }

constexpr int kMaxV = 1 << 21;

int check_vocab(const flexmoe_logprob_desc* D, int rows, const char* who, long long* ld) {
    if (!D) return fail(FLEXMOE_EINVAL, "%s: desc is NULL", who);
    if (D->dtype != FLEXMOE_F32 && D->dtype != FLEXMOE_BF16)
        return fail(FLEXMOE_EDTYPE, "%s: dtype %d is neither FLEXMOE_F32 nor FLEXMOE_BF16", who, D->dtype);
    if (D->V < 1 || D->V > kMaxV) return fail(FLEXMOE_ESHAPE, "%s: V = %d outside [1, 2^21]", who, D->V);
    if (D->top < 0 || D->top > kMaxTop || D->top > D->V) return fail(FLEXMOE_ESHAPE, "%s: top = %d outside [0, min(V, %d)]", who, D->top, kMaxTop);
    if (D->max_rows < 0 || D->max_rows > (1 << 24)) return fail(FLEXMOE_ESHAPE, "%s: max_rows = %d outside [0, 2^24]", who, D->max_rows);
    if (!(D->temperature >= 1e-6f && D->temperature <= 1e6f))
        return fail(FLEXMOE_EINVAL, "%s: temperature = %g outside [1e-6, 1e6]", who, (double)D->temperature);
    const int unit = D->dtype == FLEXMOE_BF16 ? 8 : 4;
    *ld = D->ld ? D->ld : D->V;
    if (*ld < D->V || *ld > 2LL * kMaxV || *ld % unit)
        return fail(FLEXMOE_ESHAPE, "%s: ld = %lld must be a multiple of %d in [V = %d, 2^22]", who, *ld, unit, D->V);
    if (rows < 0) return fail(FLEXMOE_EINVAL, "%s: rows = %d is negative", who, rows);
    if (rows > D->max_rows) return fail(FLEXMOE_ESHAPE, "%s: rows = %d above max_rows = %d", who, rows, D->max_rows);
    return FLEXMOE_OK;
}

int unit_run(int dtype) { return dtype == FLEXMOE_BF16 ? Vocab<true>::run : Vocab<false>::run; }

size_t list_offset(size_t parts) { return (parts * 16 + 255) & ~size_t(255); }

size_t logprob_bytes(const flexmoe_logprob_desc* D, int rows) {
    const size_t parts = D->V < 2 * kLeastRange ? 0 : most_parts(rows, D->V, kWanted);  // else rows are whole
    return std::max<size_t>(256, list_offset(parts) + parts * D->top * 8);
}

template <bool kBf16, bool kTop>
hipError_t launch_logprobs(const LogprobArgs& a, int rows, hipStream_t s) {
    logprob_kernel<kBf16, kTop><<<(unsigned)rows * a.P, kVT, 0, s>>>(a);
    if (a.P > 1) logprob_join_kernel<kBf16, kTop><<<rows, kVT, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

extern "C" {

size_t flexmoe_token_logprobs_workspace_bytes(const flexmoe_logprob_desc* desc, int32_t rows) {
    long long ld;
    if (check_vocab(desc, rows, "token_logprobs_workspace_bytes", &ld)) return 0;
    return logprob_bytes(desc, rows);
}

int flexmoe_token_logprobs(const flexmoe_logprob_desc* desc, int32_t rows, const void* logits, const int32_t* tokens, float* logprob,
                           float* entropy, float* lse, int32_t* top_ids, float* top_logprobs, void* workspace, size_t workspace_bytes,
                           void* stream) {
    const char* who = "token_logprobs";
    long long ld;
    const int rc = check_vocab(desc, rows, who, &ld);
    if (rc) return rc;
    if (rows == 0) return FLEXMOE_OK;
    if (!logits || !entropy || !lse) return fail(FLEXMOE_EINVAL, "%s: a pointer is NULL", who);
    if (!tokens != !logprob) return fail(FLEXMOE_EINVAL, "%s: tokens and logprob go together", who);
    if ((desc->top > 0) != (top_ids && top_logprobs) || (desc->top == 0 && (top_ids || top_logprobs)))
        return fail(FLEXMOE_EINVAL, "%s: top_ids and top_logprobs go with top", who);
    if (misaligned(logits, 15)) return fail(FLEXMOE_EINVAL, "%s: logits must be 16-byte aligned", who);
    for (const void* p : {(const void*)tokens, (const void*)logprob, (const void*)entropy, (const void*)lse, (const void*)top_ids, (const void*)top_logprobs})
        if (misaligned(p, 3)) return fail(FLEXMOE_EINVAL, "%s: tokens and results must be 4-byte aligned", who);
    LogprobArgs a;
    a.logits = logits, a.tokens = tokens, a.logprob = logprob, a.entropy = entropy, a.lse = lse, a.top_ids = top_ids, a.top_logprobs = top_logprobs;
    a.parts = nullptr, a.lists = nullptr, a.ld = (size_t)ld, a.V = desc->V, a.K = desc->top;
    a.P = row_parts(rows, desc->V, unit_run(desc->dtype), kWanted, desc->top ? kMostKeys / desc->top : 1 << 20);
    a.length = part_length(desc->V, a.P, unit_run(desc->dtype));
    a.inv_t = (float)(1.0 / desc->temperature), a.c = (float)(1.4426950408889634 / desc->temperature);
    if (a.P > 1) {
        const size_t need = logprob_bytes(desc, rows);
        if (!workspace || workspace_bytes < need)
            return fail(FLEXMOE_EWORKSPACE, "%s: workspace of %zu bytes, %zu needed", who, workspace ? workspace_bytes : 0, need);
        if (misaligned(workspace, 255)) return fail(FLEXMOE_EWORKSPACE, "%s: workspace must be 256-byte aligned", who);
        a.parts = (float*)workspace;
        a.lists = (uint64_t*)((char*)workspace + list_offset((size_t)rows * a.P));
    }
    const bool bf16 = desc->dtype == FLEXMOE_BF16;
    const int slice = (1 << 23) / a.P;  // a launch's threads are fewer than 2^32
    for (int done = 0; done < rows; done += slice) {
        const int n = std::min(slice, rows - done);
        const hipStream_t s = (hipStream_t)stream;
        const hipError_t err = bf16 ? (a.K ? launch_logprobs<true, true>(a, n, s) : launch_logprobs<true, false>(a, n, s))
                                    : (a.K ? launch_logprobs<false, true>(a, n, s) : launch_logprobs<false, false>(a, n, s));
        if (err != hipSuccess) return hip_fail(err, who);
        a.logits = (const char*)a.logits + (size_t)n * ld * (bf16 ? 2 : 4);
        if (tokens) a.tokens += n, a.logprob += n;
        a.entropy += n, a.lse += n;
        if (a.K) a.top_ids += (size_t)n * a.K, a.top_logprobs += (size_t)n * a.K;
        if (a.P > 1) a.parts += (size_t)4 * n * a.P, a.lists += (size_t)n * a.P * a.K;
    }
    return FLEXMOE_OK;
}

}  // extern "C"
