// One AdamW step over many tensors (gfx950), states in 32 or in 8 bits.
//
//   g = grad * grad_scale
//   m = beta1 m + (1 - beta1) g         v = beta2 v + (1 - beta2) g^2
//   p = p (1 - lr decay) - lr / (1 - beta1^t) * m / (sqrt(v / (1 - beta2^t)) + eps)
//
// in fp32.  A bf16 parameter has an fp32 master copy that the step works on, or
// is itself read, stepped and rounded to nearest.
//
// 8-bit states: blocks of 256 consecutive values share an fp32 scale each.
//   m: a sign bit and k = 0 .. 127, which stands for the float with the bits
//      (896 + k) << 20 (three mantissa bits, 16 binades up to 1.875; 0 for k =
//      0) times the scale, the power of two that brings the block's largest
//      value into (0.9375, 1.875].
//   v: k = 0 .. 255 stands for (k * scale)^2, scale = sqrt(largest) / 255.
// A step changes a running mean by a small part of itself, less than half the
// distance of neighbouring codes; rounded to nearest it would stand still.  So
// both are rounded up with the probability that keeps their mean, from 32 bits
// hashed from the seed, the step, the tensor's number and the value's index.
// v's linear code for its root keeps large values finely (that noise adds up
// over 1 / (1 - beta2) steps).  A v above zero never becomes zero: it would
// blow up the next update; it becomes at least the smallest code, which makes
// updates smaller.  A block with a NaN or an infinity gets the scale NaN.
//
// Bound by memory: 28 bytes per value with 32-bit states (bf16 parameter,
// master copy, bf16 gradient), 16 with 8-bit ones.  A wave takes 256
// consecutive values at a time (4 per lane: 16-byte accesses of fp32), with 8-bit
// states one of those, with 32-bit ones four, or two in lists of less than 2^24
// values (100 M values, bf16 with master: 8 bits 267 us for one, 276 for two, 279
// for four with sums fused as the compiler likes, 278 for one with every rounding
// kept, on another card: 5.8 TB/s; 32 bits 483, 481, 468: 6.0 TB/s; 1.5 M values in 192
// tensors, 32 bits: 19, 17, 22 us).  Every value is read once and written once,
// with the non-temporal hint (8 bits 307 -> 279 us, 32 bits 525 -> 468).  The
// list travels in the kernel's arguments, 56 tensors a launch.
#include <algorithm>
#include <cmath>

#include "common.h"
#include "error.h"

namespace flexmoe {

namespace {

constexpr int AT = 256;            // threads
constexpr int kBlock = 256;        // values of a block of states

// Values of a workgroup whose waves take `unroll` blocks each.
constexpr int chunk(int unroll) { return AT / 64 * unroll * kBlock; }
constexpr int64_t kMaxValues = 1LL << 33;   // of a tensor: its workgroups' threads are fewer than 2^32
constexpr uint64_t kMaxGroups = 1u << 24;  // of a launch, for the same reason
constexpr int kTensors = 56;       // per launch: the arguments stay below 4 KB

struct AdamwArgs {
    flexmoe_adamw_tensor t[kTensors];
    uint32_t first[kTensors + 1];  // first workgroup of each tensor
    float beta1, beta2, one_minus_beta1, one_minus_beta2, grad_scale, keep, step_size, inv_bias2, eps;
    uint32_t key;                  // seed and step
    int tensor0;                   // number of t[0] in the list
    const flexmoe_adamw_clock* clock;  // holds step_size, inv_bias2 and key, or NULL
};
static_assert(sizeof(AdamwArgs) <= 4096, "kernel arguments");

constexpr uint32_t kTensorStep = 0x6C8E9CF5u, kSeedStep = 0x3504F335u, kTimeStep = 0x5851F42Du;

__device__ __forceinline__ uint32_t random_bits(uint32_t h) {
    h = (h ^ (h >> 16)) * 0x45D9F3B5u;
    h = (h ^ (h >> 15)) * 0x2C1B3C6Du;
    return h ^ (h >> 16);
}

// Largest of a wave's non-negative floats by their bits (a NaN is above all).
__device__ __forceinline__ uint32_t wave_max_bits(uint32_t v) {
#define FLEXMOE_MSTEP(C, M) v = max(v, (uint32_t)dpp_shift<C, M>((int)v))
    FLEXMOE_MSTEP(0x111, 0xf);
    FLEXMOE_MSTEP(0x112, 0xf);
    FLEXMOE_MSTEP(0x114, 0xf);
    FLEXMOE_MSTEP(0x118, 0xf);
    FLEXMOE_MSTEP(0x142, 0xa);
    FLEXMOE_MSTEP(0x143, 0xc);
#undef FLEXMOE_MSTEP
    return (uint32_t)lane63((int)v);
}

__device__ __forceinline__ float m_value(uint32_t code, float scale) {
    const uint32_t k = code & 127u;
    const float y = (k ? __uint_as_float((896u + k) << 20) : 0.f) * scale;
    return code > 127u ? -y : y;
}
__device__ __forceinline__ float v_value(uint32_t code, float scale) {
    const float s = (float)code * scale;
    return s * s;
}

typedef uint32_t uintx2 __attribute__((ext_vector_type(2)));

// 4 values of lane-contiguous memory; n of them exist (kFull: all, and aligned).
template <bool kFull>
__device__ __forceinline__ void load4(const float* p, int n, float (&v)[4]) {
    if constexpr (kFull) {
        const floatx4 w = __builtin_nontemporal_load(reinterpret_cast<const floatx4*>(p));
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = w[k];
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = k < n ? p[k] : 0.f;
    }
}
template <bool kFull>
__device__ __forceinline__ void load4(const bf16_t* p, int n, float (&v)[4]) {
    if constexpr (kFull) {
        const uintx2 w = __builtin_nontemporal_load(reinterpret_cast<const uintx2*>(p));
        v[0] = __uint_as_float(w.x << 16), v[1] = __uint_as_float(w.x & 0xffff0000u);
        v[2] = __uint_as_float(w.y << 16), v[3] = __uint_as_float(w.y & 0xffff0000u);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = k < n ? bf16_to_f32(p[k]) : 0.f;
    }
}
template <bool kFull>
__device__ __forceinline__ void load4(const uint8_t* p, int n, uint32_t& v) {
    if constexpr (kFull) {
        v = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(p));
    } else {
        v = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k < n) v |= (uint32_t)p[k] << (8 * k);
    }
}
template <bool kFull>
__device__ __forceinline__ void store4(float* p, int n, const float (&v)[4]) {
    if constexpr (kFull) {
        __builtin_nontemporal_store(floatx4{v[0], v[1], v[2], v[3]}, reinterpret_cast<floatx4*>(p));
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k < n) p[k] = v[k];
    }
}
template <bool kFull>
__device__ __forceinline__ void store4(bf16_t* p, int n, const float (&v)[4]) {
    if constexpr (kFull) {
        const bf16x2_t a = __builtin_convertvector(float2_t{v[0], v[1]}, bf16x2_t), b = __builtin_convertvector(float2_t{v[2], v[3]}, bf16x2_t);
        __builtin_nontemporal_store(uintx2{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)}, reinterpret_cast<uintx2*>(p));
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k < n) p[k] = f32_to_bf16(v[k]);
    }
}
template <bool kFull>
__device__ __forceinline__ void store4(uint8_t* p, int n, uint32_t v) {
    if constexpr (kFull) {
        __builtin_nontemporal_store(v, reinterpret_cast<uint32_t*>(p));
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k < n) p[k] = (uint8_t)(v >> (8 * k));
    }
}

// The hardware root takes a denormal, whose root is below 1.1e-19, for 0.  That
// shows beside an eps below kSmallest only, 2^24 times as much: there small values
// are lifted by a power of four (in every step it would take 1 to 2 % longer).
constexpr double kSmallest = 2e-12;
template <bool kSmallEps>
__device__ __forceinline__ float root(float x) {
    if constexpr (!kSmallEps) return __builtin_amdgcn_sqrtf(x);
    const bool small = x < 0x1p-96f;
    const float r = __builtin_amdgcn_sqrtf(small ? x * 0x1p+64f : x);
    return small ? r * 0x1p-32f : r;
}

// What a step's number decides.
struct StepNumbers {
    float step_size, inv_bias2;
    uint32_t key;
};
__host__ __device__ inline StepNumbers numbers_of(uint32_t seed, int64_t step, double lr, double beta1, double beta2) {
    return StepNumbers{(float)(lr / (1.0 - pow(beta1, (double)step))), (float)(1.0 / (1.0 - pow(beta2, (double)step))),
                       seed * kSeedStep + (uint32_t)step * kTimeStep};
}

// A step counted on the device: its number and what follows from it.
__global__ void adamw_clock_kernel(flexmoe_adamw_clock* clock, uint32_t seed, double lr, double beta1, double beta2) {
    const int64_t step = clock->step + 1;
    const StepNumbers n = numbers_of(seed, step, lr, beta1, beta2);
    clock->step = step;
    clock->step_size = n.step_size;
    clock->inv_bias2 = n.inv_bias2;
    clock->key = n.key;
}

// The parameter that is read and stepped: the master copy where there is one.
template <typename P>
struct Values {
    float p[4], g[4], m[4], v[4];
    uint32_t mc, vc;
    float ms, vs;
};

template <typename P, typename G, int kBits, bool kFull, bool kMaster>
__device__ __forceinline__ void read_values(const flexmoe_adamw_tensor& t, size_t i, int n, Values<P>& x) {
    if constexpr (kMaster) load4<kFull>(t.master + i, n, x.p);
    else load4<kFull>(reinterpret_cast<const P*>(t.param) + i, n, x.p);
    load4<kFull>(reinterpret_cast<const G*>(t.grad) + i, n, x.g);
    if constexpr (kBits == 32) {
        load4<kFull>(reinterpret_cast<const float*>(t.m) + i, n, x.m);
        load4<kFull>(reinterpret_cast<const float*>(t.v) + i, n, x.v);
    } else {
        load4<kFull>(reinterpret_cast<const uint8_t*>(t.m) + i, n, x.mc);
        load4<kFull>(reinterpret_cast<const uint8_t*>(t.v) + i, n, x.vc);
        x.ms = t.m_scale[i / kBlock];
        x.vs = t.v_scale[i / kBlock];
    }
}

template <typename P, typename G, int kBits, bool kFull, bool kMaster, bool kSmallEps>
__device__ __forceinline__ void step_values(const AdamwArgs& a, const flexmoe_adamw_tensor& t, size_t i, int n,
                                            const StepNumbers& step, Values<P>& x) {
    // every product and sum rounded by itself: whether a code is rounded up hangs
    // on the last bit, and the formula's own roundings decide, not which of them
    // the compiler fuses
#pragma clang fp contract(off)
    uint32_t top_m = 0, top_v = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (kBits == 8) {
            x.m[k] = m_value((x.mc >> (8 * k)) & 255u, x.ms);
            x.v[k] = v_value((x.vc >> (8 * k)) & 255u, x.vs);
        }
        const float g = x.g[k] * a.grad_scale;
        x.m[k] = x.m[k] * a.beta1 + g * a.one_minus_beta1;
        x.v[k] = x.v[k] * a.beta2 + g * g * a.one_minus_beta2;
        // the hardware root and reciprocal (1 ulp each): a few ulps of the
        // update, which is itself a small part of p
        const float den = root<kSmallEps>(x.v[k] * step.inv_bias2) + a.eps;
        x.p[k] = x.p[k] * a.keep - step.step_size * (x.m[k] * __builtin_amdgcn_rcpf(den));
        if constexpr (kBits == 8)
            if (kFull || k < n) {
                top_m = max(top_m, __float_as_uint(x.m[k]) & 0x7fffffffu);
                top_v = max(top_v, __float_as_uint(x.v[k]) & 0x7fffffffu);
            }
    }
    if constexpr (kMaster) store4<kFull>(t.master + i, n, x.p);
    store4<kFull>(reinterpret_cast<P*>(t.param) + i, n, x.p);
    if constexpr (kBits == 32) {
        store4<kFull>(reinterpret_cast<float*>(t.m) + i, n, x.m);
        store4<kFull>(reinterpret_cast<float*>(t.v) + i, n, x.v);
    } else {
        top_m = wave_max_bits(top_m);
        top_v = wave_max_bits(top_v);
        float tv = __uint_as_float(top_v);
        const float nan = __uint_as_float(0x7fc00000u);
        // scale of m: the power of two that top is at most 1.875 times of
        const uint32_t sb = max((top_m + 0xfffffu) & 0x7f800000u, 0x00800000u);
        const int down = 127 - (int)(sb >> 23);
        // 65025 / tv leaves fp32's range below 1.9e-34: such a block (all zeros is
        // one too) is lifted by a power of two first
        if (tv < 0x1p-100f) {
            tv *= 0x1p+64f;
#pragma unroll
            for (int k = 0; k < 4; ++k) x.v[k] *= 0x1p+64f;
        }
        const float per_v = 65025.f * (1.f / tv);
        constexpr float kLeast = 1.125f / 32768.f;  // code 1
        uint32_t mc = 0, vc = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t r = random_bits(step.key + (uint32_t)i + k);
            const float y = __builtin_amdgcn_ldexpf(fabsf(x.m[k]), down);
            int c = (int)((__float_as_uint(y) + ((r >> 16) << 4)) >> 20) - 896;
            c = y < kLeast ? (int)((float)(r >> 16) * (kLeast / 65536.f) < y) : min(max(c, 0), 127);
            mc |= ((uint32_t)c | (x.m[k] < 0.f ? 128u : 0u)) << (8 * k);
            const float z = x.v[k] * per_v;
            const float f = floorf(__builtin_amdgcn_sqrtf(z));
            const float up = (float)(r & 0xffffu) * (1.f / 65536.f) * (2.f * f + 1.f) < z - f * f ? f + 1.f : f;
            vc |= (x.v[k] > 0.f ? (uint32_t)fminf(fmaxf(up, 1.f), 255.f) : 0u) << (8 * k);
        }
        store4<kFull>(reinterpret_cast<uint8_t*>(t.m) + i, n, mc);
        store4<kFull>(reinterpret_cast<uint8_t*>(t.v) + i, n, vc);
        if ((threadIdx.x & 63) == 0) {
            t.m_scale[i / kBlock] = top_m >= 0x7f800000u ? nan : top_m ? __uint_as_float(sb) : 0.f;
            t.v_scale[i / kBlock] = top_v >= 0x7f800000u ? nan : sqrtf(__uint_as_float(top_v)) / 255.f;
        }
    }
}

template <typename P, typename G, int kBits, int kUnroll, bool kMaster, bool kSmallEps>
__device__ __forceinline__ void step_chunk(const AdamwArgs& a, const flexmoe_adamw_tensor& t, size_t at, const StepNumbers& step) {
    const int lane = threadIdx.x & 63;
    const size_t left = (size_t)t.n - at;  // from this wave's first value on
    const uintptr_t bits = (uintptr_t)t.param | (uintptr_t)t.grad | (uintptr_t)t.m | (uintptr_t)t.v | (uintptr_t)t.master;
    if (left >= (size_t)kUnroll * kBlock && (bits & 15) == 0) {
        Values<P> x[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) read_values<P, G, kBits, true, kMaster>(t, at + u * kBlock + lane * 4, 4, x[u]);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) step_values<P, G, kBits, true, kMaster, kSmallEps>(a, t, at + u * kBlock + lane * 4, 4, step, x[u]);
    } else {
        for (int u = 0; u < kUnroll && (size_t)u * kBlock < left; ++u) {
            // every lane stays: the block's largest value is the wave's
            const int n = (int)min((long long)4, max((long long)0, (long long)left - u * kBlock - lane * 4));
            Values<P> x;
            read_values<P, G, kBits, false, kMaster>(t, at + u * kBlock + lane * 4, n, x);
            step_values<P, G, kBits, false, kMaster, kSmallEps>(a, t, at + u * kBlock + lane * 4, n, step, x);
        }
    }
}

template <typename P, typename G, int kBits, int kUnroll, bool kSmallEps>
__global__ __launch_bounds__(AT) void adamw_kernel(AdamwArgs a) {
    static_assert(kTensors < 64, "one lane per tensor");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t f = a.first[min(lane, kTensors)];
    const int j = __popcll(__ballot(lane < kTensors && f <= blockIdx.x)) - 1;  // tensors without values share their start
    const flexmoe_adamw_tensor& t = a.t[j];
    const size_t at = (size_t)(blockIdx.x - a.first[j]) * chunk(kUnroll) + wave * (kUnroll * kBlock);
    if (at >= (size_t)t.n) return;
    StepNumbers step{a.step_size, a.inv_bias2, a.key};
    if (a.clock) step = StepNumbers{a.clock->step_size, a.clock->inv_bias2, a.clock->key};
    step.key += (uint32_t)(a.tensor0 + j) * kTensorStep;
    if (sizeof(P) == 2 && t.master) step_chunk<P, G, kBits, kUnroll, true, kSmallEps>(a, t, at, step);
    else step_chunk<P, G, kBits, kUnroll, false, kSmallEps>(a, t, at, step);
}

template <typename O>
__global__ __launch_bounds__(AT) void adamw_read_kernel(const uint8_t* m, const uint8_t* v, const float* ms, const float* vs, O* om, O* ov,
                                                        size_t n, bool aligned) {
    const size_t i = ((size_t)blockIdx.x * AT + threadIdx.x) * 4;
    if (i >= n) return;
    const float sm = ms[i / kBlock], sv = vs[i / kBlock];
    const int c = (int)min((size_t)4, n - i);
    const bool full = aligned && c == 4;
    uint32_t a, b;
    if (full) load4<true>(m + i, 4, a), load4<true>(v + i, 4, b);
    else load4<false>(m + i, c, a), load4<false>(v + i, c, b);
    float x[4], y[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = m_value((a >> (8 * k)) & 255u, sm), y[k] = v_value((b >> (8 * k)) & 255u, sv);
    if (full) store4<true>(om + i, 4, x), store4<true>(ov + i, 4, y);
    else store4<false>(om + i, c, x), store4<false>(ov + i, c, y);
}

// hipLaunchKernel itself: the arguments, 4 KB, are not copied on the way, and the
// error is the launch's own.
template <int kBits, int kUnroll, bool kSmallEps>
hipError_t launch(AdamwArgs& a, bool param_bf16, bool grad_bf16, unsigned grid, hipStream_t s) {
    auto* const f = param_bf16 && grad_bf16 ? adamw_kernel<bf16_t, bf16_t, kBits, kUnroll, kSmallEps>
                    : param_bf16            ? adamw_kernel<bf16_t, float, kBits, kUnroll, kSmallEps>
                    : grad_bf16             ? adamw_kernel<float, bf16_t, kBits, kUnroll, kSmallEps>
                                            : adamw_kernel<float, float, kBits, kUnroll, kSmallEps>;
    void* args[] = {&a};
    return hipLaunchKernel(reinterpret_cast<const void*>(f), dim3(grid), dim3(AT), args, 0, s);
}
template <int kBits, int kUnroll>
hipError_t launch(AdamwArgs& a, bool param_bf16, bool grad_bf16, unsigned grid, hipStream_t s) {
    return a.eps < (float)kSmallest ? launch<kBits, kUnroll, true>(a, param_bf16, grad_bf16, grid, s)
                                    : launch<kBits, kUnroll, false>(a, param_bf16, grad_bf16, grid, s);
}

bool misaligned(const void* p, uintptr_t mask) { return ((uintptr_t)p & mask) != 0; }

}  // namespace

}  // namespace flexmoe

using namespace flexmoe;

extern "C" {

int flexmoe_adamw_step(const flexmoe_adamw_desc* D, const flexmoe_adamw_tensor* tensors, int32_t count, void* stream) {
    if (!D) return fail(FLEXMOE_EINVAL, "adamw_step: desc is NULL");
    for (int dt : {D->param_dtype, D->grad_dtype})
        if (dt != FLEXMOE_F32 && dt != FLEXMOE_BF16)
            return fail(FLEXMOE_EDTYPE, "adamw_step: dtype %d is neither FLEXMOE_F32 nor FLEXMOE_BF16", dt);
    if (D->state_bits != 8 && D->state_bits != 32) return fail(FLEXMOE_EINVAL, "adamw_step: state_bits = %d is neither 8 nor 32", D->state_bits);
    if (count < 0 || (count > 0 && !tensors)) return fail(FLEXMOE_EINVAL, "adamw_step: count = %d, or tensors is NULL", count);
    if (D->clock && misaligned(D->clock, 7)) return fail(FLEXMOE_EINVAL, "adamw_step: clock must be 8-byte aligned");
    if (!D->clock && D->step < 1) return fail(FLEXMOE_EINVAL, "adamw_step: step = %lld must be at least 1", (long long)D->step);
    if (!(D->beta1 >= 0 && D->beta1 < 1 && D->beta2 >= 0 && D->beta2 < 1))
        return fail(FLEXMOE_EINVAL, "adamw_step: beta1 = %g, beta2 = %g outside [0, 1)", D->beta1, D->beta2);
    if (!(D->eps >= 1e-30 && std::isfinite(D->eps))) return fail(FLEXMOE_EINVAL, "adamw_step: eps = %g must be at least 1e-30", D->eps);
    if (!std::isfinite(D->lr) || !std::isfinite(D->weight_decay) || !std::isfinite(D->grad_scale))
        return fail(FLEXMOE_EINVAL, "adamw_step: lr, weight_decay and grad_scale must be finite");
    const uintptr_t pm = D->param_dtype == FLEXMOE_BF16 ? 1 : 3, gm = D->grad_dtype == FLEXMOE_BF16 ? 1 : 3;
    for (int i = 0; i < count; ++i) {
        const flexmoe_adamw_tensor& t = tensors[i];
        if (t.n < 0) return fail(FLEXMOE_EINVAL, "adamw_step: tensor %d has n = %lld", i, (long long)t.n);
        if (t.n > kMaxValues) return fail(FLEXMOE_ESHAPE, "adamw_step: tensor %d has n = %lld above 2^33", i, (long long)t.n);
        if (t.n == 0) continue;
        if (!t.param || !t.grad || !t.m || !t.v) return fail(FLEXMOE_EINVAL, "adamw_step: tensor %d has a NULL pointer", i);
        if ((D->state_bits == 8) != (t.m_scale && t.v_scale) || (D->state_bits == 32 && (t.m_scale || t.v_scale)))
            return fail(FLEXMOE_EINVAL, "adamw_step: tensor %d: scales go with 8-bit states", i);
        if (t.master && D->param_dtype != FLEXMOE_BF16)
            return fail(FLEXMOE_EINVAL, "adamw_step: tensor %d: a master copy goes with bf16 parameters", i);
        if (misaligned(t.param, pm) || misaligned(t.grad, gm) || misaligned(t.master, 3) || misaligned(t.m_scale, 3) ||
            misaligned(t.v_scale, 3) || (D->state_bits == 32 && (misaligned(t.m, 3) || misaligned(t.v, 3))))
            return fail(FLEXMOE_EINVAL, "adamw_step: tensor %d is not aligned to its elements", i);
    }
    AdamwArgs a;
    a.beta1 = (float)D->beta1;
    a.beta2 = (float)D->beta2;
    a.one_minus_beta1 = (float)(1.0 - D->beta1);
    a.one_minus_beta2 = (float)(1.0 - D->beta2);
    a.grad_scale = (float)D->grad_scale;
    a.keep = (float)(1.0 - D->lr * D->weight_decay);
    const StepNumbers numbers = D->clock ? StepNumbers{} : numbers_of(D->seed, D->step, D->lr, D->beta1, D->beta2);
    a.step_size = numbers.step_size;
    a.inv_bias2 = numbers.inv_bias2;
    a.eps = (float)D->eps;
    a.key = numbers.key;
    a.clock = D->clock;
    const hipStream_t s = (hipStream_t)stream;
    if (D->clock) {
        adamw_clock_kernel<<<1, 1, 0, s>>>(D->clock, D->seed, D->lr, D->beta1, D->beta2);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return hip_fail(err, "adamw_step launch");
    }
    uint64_t total = 0;
    for (int i = 0; i < count; ++i) total += (uint64_t)tensors[i].n;
    const int unroll = D->state_bits == 8 ? 1 : total < (1u << 24) ? 2 : 4;
    const uint64_t per = (uint64_t)chunk(unroll);
    for (int i = 0; i < count;) {
        // as many tensors as the arguments and a grid hold
        uint64_t groups = 0;
        int n = 0;
        a.tensor0 = i;
        for (; i + n < count && n < kTensors; ++n) {
            const uint64_t g = ((uint64_t)tensors[i + n].n + per - 1) / per;
            if (n > 0 && groups + g >= kMaxGroups) break;
            a.t[n] = tensors[i + n];
            a.first[n] = (uint32_t)groups;
            groups += g;
        }
        i += n;
        for (int k = n; k <= kTensors; ++k) a.first[k] = 0xffffffffu;
        if (!groups) continue;
        const unsigned grid = (unsigned)groups;
        const bool pb = D->param_dtype == FLEXMOE_BF16, gb = D->grad_dtype == FLEXMOE_BF16;
        const hipError_t err = unroll == 1   ? launch<8, 1>(a, pb, gb, grid, s)
                               : unroll == 2 ? launch<32, 2>(a, pb, gb, grid, s)
                                             : launch<32, 4>(a, pb, gb, grid, s);
        if (err != hipSuccess) return hip_fail(err, "adamw_step launch");
    }
    return FLEXMOE_OK;
}

int flexmoe_adamw_read_state(int64_t n, const void* m, const void* v, const float* m_scale, const float* v_scale, int32_t dtype,
                             void* m_out, void* v_out, void* stream) {
    if (dtype != FLEXMOE_F32 && dtype != FLEXMOE_BF16)
        return fail(FLEXMOE_EDTYPE, "adamw_read_state: dtype %d is neither FLEXMOE_F32 nor FLEXMOE_BF16", dtype);
    if (n < 0) return fail(FLEXMOE_EINVAL, "adamw_read_state: n = %lld is negative", (long long)n);
    if (n > kMaxValues) return fail(FLEXMOE_ESHAPE, "adamw_read_state: n = %lld above 2^33", (long long)n);
    if (n == 0) return FLEXMOE_OK;
    if (!m || !v || !m_scale || !v_scale || !m_out || !v_out) return fail(FLEXMOE_EINVAL, "adamw_read_state: a pointer is NULL");
    const uintptr_t om = dtype == FLEXMOE_BF16 ? 1 : 3;
    if (misaligned(m_out, om) || misaligned(v_out, om) || misaligned(m_scale, 3) || misaligned(v_scale, 3))
        return fail(FLEXMOE_EINVAL, "adamw_read_state: a pointer is not aligned to its elements");
    const bool aligned = (((uintptr_t)m | (uintptr_t)v | (uintptr_t)m_out | (uintptr_t)v_out) & 15) == 0;
    const unsigned grid = (unsigned)(((uint64_t)n + 4 * AT - 1) / (4 * AT));
    const uint8_t *mc = (const uint8_t*)m, *vc = (const uint8_t*)v;
    if (dtype == FLEXMOE_BF16)
        adamw_read_kernel<<<grid, AT, 0, (hipStream_t)stream>>>(mc, vc, m_scale, v_scale, (bf16_t*)m_out, (bf16_t*)v_out, (size_t)n, aligned);
    else
        adamw_read_kernel<<<grid, AT, 0, (hipStream_t)stream>>>(mc, vc, m_scale, v_scale, (float*)m_out, (float*)v_out, (size_t)n, aligned);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return hip_fail(err, "adamw_read_state launch");
    return FLEXMOE_OK;
}

}  // extern "C"
