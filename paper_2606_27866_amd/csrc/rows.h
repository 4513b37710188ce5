// Rows of bf16 or fp32 values read and written 8 at a time, and sums over a
// workgroup: shared by the kernels that take one row after another (norms,
// log probabilities, distillation).
//
// Rows start on 16-byte boundaries.  A row is read up to the 16-byte unit that
// its last value lies in; nothing past it is written.
#pragma once

#include "common.h"

namespace flexmoe {

template <bool kBf16>
__host__ __device__ constexpr int elem_size() { return kBf16 ? 2 : 4; }

// The 16-byte units of 8 values as they lie in memory.
template <bool kBf16>
struct Raw8 {
    u32x4 w[kBf16 ? 1 : 2];
};

// Values i .. i + 7 of the row at p, the first `left` of which exist (left >= 1).
template <bool kBf16>
__device__ __forceinline__ Raw8<kBf16> load_raw8(const void* p, size_t i, int left) {
    Raw8<kBf16> r;
    const u32x4* u = reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(p) + i * elem_size<kBf16>());
    r.w[0] = u[0];
    if constexpr (!kBf16) r.w[1] = left > 4 ? u[1] : u32x4{0, 0, 0, 0};
    return r;
}

template <bool kBf16>
__device__ __forceinline__ void unpack8(const Raw8<kBf16>& r, float (&v)[8]) {
    if constexpr (kBf16) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[2 * k] = __uint_as_float(r.w[0][k] << 16);
            v[2 * k + 1] = __uint_as_float(r.w[0][k] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = __uint_as_float(r.w[k >> 2][k & 3]);
    }
}

// As load_raw8, as fp32, with `fill` past the row's end.
template <bool kBf16>
__device__ __forceinline__ void load8(const void* p, size_t i, int left, float (&v)[8], float fill = 0.f) {
    unpack8<kBf16>(load_raw8<kBf16>(p, i, left), v);
    if (left < 8)
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = k < left ? v[k] : fill;
}

template <bool kBf16>
__device__ __forceinline__ Raw8<kBf16> pack8(const float (&v)[8]) {
    Raw8<kBf16> r;
    if constexpr (kBf16) {
#pragma unroll
        for (int k = 0; k < 4; ++k) r.w[0][k] = pack_bf16x2(v[2 * k], v[2 * k + 1]);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) r.w[k >> 2][k & 3] = __float_as_uint(v[k]);
    }
    return r;
}

template <bool kBf16>
__device__ __forceinline__ void store_raw8(void* p, size_t i, int left, const Raw8<kBf16>& r) {
    char* const at = reinterpret_cast<char*>(p) + i * elem_size<kBf16>();
    if (left >= 8) {
        u32x4* u = reinterpret_cast<u32x4*>(at);
        u[0] = r.w[0];
        if constexpr (!kBf16) u[1] = r.w[1];
    } else {
#pragma unroll
        for (int k = 0; k < 7; ++k)
            if (k < left) {
                if constexpr (kBf16) reinterpret_cast<bf16_t*>(at)[k] = (bf16_t)(r.w[0][k >> 1] >> (16 * (k & 1)));
                else reinterpret_cast<uint32_t*>(at)[k] = r.w[k >> 2][k & 3];
            }
    }
}

template <bool kBf16>
__device__ __forceinline__ void store8(void* p, size_t i, int left, const float (&v)[8]) {
    store_raw8<kBf16>(p, i, left, pack8<kBf16>(v));
}

// Largest of the wave's whole numbers, and of its values (NaN left out), in every lane: the steps of wave_total_f.
__device__ __forceinline__ uint32_t wave_max_u(uint32_t v) {
#define FLEXMOE_USTEP(C, M) v = max(v, (uint32_t)dpp_shift<C, M>((int)v))
    FLEXMOE_USTEP(0x111, 0xf);
    FLEXMOE_USTEP(0x112, 0xf);
    FLEXMOE_USTEP(0x114, 0xf);
    FLEXMOE_USTEP(0x118, 0xf);
    FLEXMOE_USTEP(0x142, 0xa);
    FLEXMOE_USTEP(0x143, 0xc);
#undef FLEXMOE_USTEP
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
__device__ __forceinline__ float wave_max(float v) {
    // a lane without a source keeps its own
#define FLEXMOE_MSTEP(C, M) v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), C, M, 0xf, false)))
    FLEXMOE_MSTEP(0x111, 0xf);
    FLEXMOE_MSTEP(0x112, 0xf);
    FLEXMOE_MSTEP(0x114, 0xf);
    FLEXMOE_MSTEP(0x118, 0xf);
    FLEXMOE_MSTEP(0x142, 0xa);
    FLEXMOE_MSTEP(0x143, 0xc);
#undef FLEXMOE_MSTEP
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// Sum of a double over the wave, in every lane: the steps of wave_total_f.
__device__ __forceinline__ double wave_total_d(double v) {
    union Halves {
        double d;
        int w[2];
    };
#define FLEXMOE_DSTEP(C, M)                                            \
    {                                                                  \
        Halves h{v};                                                   \
        h.w[0] = dpp_shift<C, M>(h.w[0]), h.w[1] = dpp_shift<C, M>(h.w[1]); \
        v += h.d;                                                      \
    }
    FLEXMOE_DSTEP(0x111, 0xf);
    FLEXMOE_DSTEP(0x112, 0xf);
    FLEXMOE_DSTEP(0x114, 0xf);
    FLEXMOE_DSTEP(0x118, 0xf);
    FLEXMOE_DSTEP(0x142, 0xa);
    FLEXMOE_DSTEP(0x143, 0xc);
#undef FLEXMOE_DSTEP
    Halves h{v};
    h.w[0] = __builtin_amdgcn_readlane(h.w[0], 63), h.w[1] = __builtin_amdgcn_readlane(h.w[1], 63);
    return h.d;
}

// Sum over kWaves waves, in every thread: the waves' sums in order.  `part`
// holds kWaves floats that no other sum uses before the next barrier.
template <int kWaves>
__device__ __forceinline__ float sum_over_waves(float v, float* part) {
    v = wave_total_f(v);
    if constexpr (kWaves > 1) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
        __syncthreads();
        v = part[0];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) v += part[w];
    }
    return v;
}

template <int kWaves>
__device__ __forceinline__ uint32_t max_over_waves(uint32_t m, uint32_t* part) {
    m = wave_max_u(m);
    if constexpr (kWaves > 1) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) m = max(m, part[w]);
    }
    return m;
}

}  // namespace flexmoe
