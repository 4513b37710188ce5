// Rows over a vocabulary (gfx950): the running maximum and sums of a softmax in
// one pass, and the joining of parts of a row.
//
// A row, or a part of it of up to kRange values, is a workgroup's.  A thread
// takes kUnits 16-byte units at a time, one from each run of the workgroup's
// accesses, so that every access of a wave covers whole cache lines.
#pragma once

#include <algorithm>

#include "rows.h"

namespace flexmoe {

constexpr int kVT = 256;            // threads of a workgroup
constexpr int kRange = 1 << 17;     // values of a workgroup, at most
constexpr int kLeastRange = 2048;   // and at least, where a row has more
constexpr int kMaxTop = 128;        // listed tokens of a row

template <bool kBf16>
struct Vocab {
    static constexpr int n = kBf16 ? 8 : 4;            // values of a unit
    static constexpr int units = kBf16 ? 4 : 8;        // of a thread at a time: 32 values
    static constexpr int run = kVT * n;                // values of a workgroup's access
    static constexpr int step = run * units;
};

template <bool kBf16>
__device__ __forceinline__ u32x4 load_unit(const void* row, int i) {
    return *reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(row) + (size_t)i * elem_size<kBf16>());
}

template <bool kBf16>
__device__ __forceinline__ void unpack_unit(const u32x4& w, float (&v)[Vocab<kBf16>::n]) {
    if constexpr (kBf16) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[2 * k] = __uint_as_float(w[k] << 16);
            v[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = __uint_as_float(w[k]);
    }
}

// Values i .. i + n - 1 of a row whose values end at `end`; -inf past it.
template <bool kBf16>
__device__ __forceinline__ void load_values(const void* row, int i, int end, float (&v)[Vocab<kBf16>::n]) {
    constexpr int n = Vocab<kBf16>::n;
    if (i >= end) {
#pragma unroll
        for (int k = 0; k < n; ++k) v[k] = -INFINITY;
        return;
    }
    unpack_unit<kBf16>(load_unit<kBf16>(row, i), v);
    if (i + n > end)
#pragma unroll
        for (int k = 0; k < n; ++k) v[k] = i + k < end ? v[k] : -INFINITY;
}

// f(step, its first value's index, the values of this thread's units) for the steps of
// [begin, end): -inf past the end.  A step's loads have no conditions, so that all of
// them are in flight together (addresses past the end are those of the last unit); in
// bf16 those of the next step too, in fp32 they would take too many registers.
template <bool kBf16, typename F>
__device__ __forceinline__ void each_step(const void* row, int begin, int end, F&& f) {
    using W = Vocab<kBf16>;
    const int t = threadIdx.x, last = (end - 1) / W::n * W::n;
    u32x4 next[W::units];
    auto request = [&](int at) {
#pragma unroll
        for (int u = 0; u < W::units; ++u) next[u] = load_unit<kBf16>(row, min(at + u * W::run + t * W::n, last));
    };
    if (begin < end) request(begin);
    for (int at = begin, it = 0; at < end; at += W::step, ++it) {
        float v[W::units][W::n];
        u32x4 now[W::units];
#pragma unroll
        for (int u = 0; u < W::units; ++u) now[u] = next[u];
        if (kBf16 && at + W::step < end) request(at + W::step);
#pragma unroll
        for (int u = 0; u < W::units; ++u) unpack_unit<kBf16>(now[u], v[u]);
        if (at + W::step > end) {
#pragma unroll
            for (int u = 0; u < W::units; ++u)
#pragma unroll
                for (int k = 0; k < W::n; ++k) v[u][k] = at + u * W::run + t * W::n + k < end ? v[u][k] : -INFINITY;
        }
        f(it, at, v);
        if (!kBf16 && at + W::step < end) request(at + W::step);
    }
}

template <bool kBf16>
__device__ __forceinline__ float value_at(const void* row, int i) {
    if constexpr (kBf16) return bf16_to_f32(reinterpret_cast<const bf16_t*>(row)[i]);
    else return reinterpret_cast<const float*>(row)[i];
}

// Largest value, NaN left out.
template <int N>
__device__ __forceinline__ float max_of(const float (&v)[N], float m) {
#pragma unroll
    for (int k = 0; k < N; ++k) m = fmaxf(m, v[k]);
    return m;
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// sum of 2^(c (x - m)) and, weighted by it, of c (x - m): of values whose largest is m.
struct Sums {
    float m = -INFINITY, s = 0.f, h = 0.f;

    // The same sums with the reference `to` >= m.
    __device__ __forceinline__ void refer(float to, float c) {
        if (m == to) return;
        if (m == -INFINITY) {  // nothing but -inf so far (or NaN, which s keeps)
            m = to;
            return;
        }
        const float d = (m - to) * c, f = exp2_fast(d);
        h = f * (h + s * fmaxf(d, -200.f));
        s *= f;
        m = to;
    }
};

// A thread's sums while its largest value is still growing: exponents are taken
// against r = c m rounded, one fused operation for each value.
struct RunningSums {
    Sums t;
    float r = 0.f;

    // The largest of the next values is at most `largest`.
    __device__ __forceinline__ void raise(float largest, float c) {
        if (!__any(largest > t.m)) return;
        if (largest > t.m) {
            const float to = largest * c;
            if (t.m > -INFINITY) {
                const float d = r - to, f = exp2_fast(d);
                t.h = f * (t.h + t.s * fmaxf(d, -200.f));
                t.s *= f;
            }
            t.m = largest;
            r = to;
        }
    }
    __device__ __forceinline__ void add(float v, float c) {
        const float d = fmaf(v, c, -r), e = exp2_fast(d);
        t.s += e;
        t.h = fmaf(e, fmaxf(d, -200.f), t.h);  // a product of 0 and -inf would be no number
    }
    // Against c m itself.
    __device__ __forceinline__ Sums exact(float c) const {
        if (t.m == -INFINITY) return t;
        Sums o = t;
        const float d = fmaf(t.m, c, -r), f = exp2_fast(-d);
        o.h = f * (t.h - d * t.s);
        o.s = f * t.s;
        return o;
    }
};

// Order of logits as whole numbers: NaN 0, then ascending, -0 as +0.
__device__ __forceinline__ uint32_t value_key(float v) {
    uint32_t u = __float_as_uint(v);
    u = u == 0x80000000u ? 0u : u;
    const uint32_t k = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
    return __builtin_isnan(v) ? 0u : k;
}
__device__ __forceinline__ float key_value(uint32_t k) {
    if (k == 0) return __uint_as_float(0x7fc00000u);
    return __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k);
}
// Larger value first, then lower place first.
__device__ __forceinline__ uint64_t place_key(float v, int i) { return ((uint64_t)value_key(v) << 32) | (uint32_t)~i; }

// Parts of a row: as few as kRange allows, and while there are few rows as many as make
// `wanted` workgroups, `limit` at most.
inline int row_parts(int rows, int V, int unit_run, int wanted, int limit = 1 << 20) {
    const int least = (V + kRange - 1) / kRange;
    const int most = std::max(1, std::min(V / kLeastRange, limit));
    const int parts = std::max(least, std::min(most, rows > 0 ? (wanted + rows - 1) / rows : 1));
    const int length = ((V + parts - 1) / parts + unit_run - 1) / unit_run * unit_run;
    return (V + length - 1) / length;
}
// Parts of all rows of any call of up to `rows` rows: rows that have to be in parts, or
// few rows in at most `wanted` and one more each.
inline size_t most_parts(int rows, int V, int wanted) {
    const size_t least = (V + kRange - 1) / kRange, most = std::max(1, V / kLeastRange), few = std::min(rows, wanted);
    return std::max(rows * least, std::min<size_t>(few * most, 2 * (size_t)wanted));
}
inline int part_length(int V, int parts, int unit_run) { return ((V + parts - 1) / parts + unit_run - 1) / unit_run * unit_run; }

}  // namespace flexmoe
