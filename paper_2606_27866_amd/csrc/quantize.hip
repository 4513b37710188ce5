// Rows rounded to 8 bits with a scale each (gfx950): s = max|v| / 127 over the
// row, q = round(v * ((1 / max|v|) * 127)) in fp32, ties to even, for v = x or
// silu(x) * x2.
// A row that holds a NaN or an infinity gets the scale NaN and zeros, so that
// what is computed from it is NaN; a row of zeros the scale 0.
//
// Bound by memory: a row is read once and kept in registers between its
// maximum and its rounding (up to 16384 values; longer rows are read twice).
// Rows of up to 512 values take one wave each, in calls of 1024 rows and more
// also those of up to 2048; longer ones a workgroup.  A workgroup against a wave
// for each of 32768 bf16 rows: of 600 values 24.9 and 15.8 us, 1408 35.2 and
// 29.2, 2048 41.9 and 40.9, 3584 61.4 and 68.4, 4096 68.0 and 76.9; of 1024 gated
// rows of 3584 values 6.9 and 10.0.  8192 rows of 3584: 15.6 us, 5.6 TB/s.
#include "grouped.h"

namespace flexmoe {

namespace {

constexpr int QT = 256;
constexpr int kManyRows = 1024;  // rows from which a wave takes a row of up to 2048 values

template <bool kBf16>
__device__ __forceinline__ void load8(const void* p, size_t i, bool upper, float (&v)[8]) {
    if constexpr (kBf16) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(reinterpret_cast<const bf16_t*>(p) + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[2 * k] = __uint_as_float(w[k] << 16);
            v[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
        }
    } else {
        const float* f = reinterpret_cast<const float*>(p) + i;
        const floatx4 a = *reinterpret_cast<const floatx4*>(f);
        const floatx4 b = upper ? *reinterpret_cast<const floatx4*>(f + 4) : floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = a[k], v[k + 4] = b[k];
    }
}

// Values 8c .. 8c + 7 of the row; zeros past its end.
template <bool kBf16, bool kGated>
__device__ __forceinline__ void row_chunk(const void* x, const void* x2, size_t at, int c, int cols, float (&v)[8]) {
    load8<kBf16>(x, at + 8 * c, 8 * c + 4 < cols, v);
    if constexpr (kGated) {
        float u[8];
        load8<kBf16>(x2, at + 8 * c, 8 * c + 4 < cols, u);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = v[k] / (1.f + expf(-v[k])) * u[k];
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = 8 * c + k < cols ? v[k] : 0.f;
}

__device__ __forceinline__ uint32_t max_bits(const float (&v)[8], uint32_t m) {
#pragma unroll
    for (int k = 0; k < 8; ++k) m = max(m, __float_as_uint(v[k]) & 0x7fffffffu);
    return m;
}

// Whole numbers of 8 values, the first cols - at of which exist (kWhole: all).
template <bool kWhole>
__device__ __forceinline__ void store_q(int8_t* q, const float (&v)[8], float inv, int at, int cols) {
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int n = (int)fminf(fmaxf(rintf(v[k] * inv), -127.f), 127.f);
        w[k >> 2] |= (uint32_t)(n & 255) << (8 * (k & 3));
    }
    if (kWhole || at + 8 <= cols) {
        *reinterpret_cast<uint2*>(q) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
        for (int k = 0; k < 7; ++k)
            if (at + k < cols) q[k] = (int8_t)(w[k >> 2] >> (8 * (k & 3)));
    }
}

// kWaves waves per row, kChunks 8-value chunks per lane in registers (0: read
// again).  kWhole: rows of whole chunks (the test for the last one in every store
// takes 2 % longer).
template <bool kBf16, bool kGated, int kWaves, int kChunks, bool kWhole>
__global__ __launch_bounds__(QT) void quantize_kernel(const void* x, const void* x2, size_t ldx, int8_t* q, size_t ldq, float* scale,
                                                      int rows, int cols) {
    constexpr int kLanes = 64 * kWaves, kRows = QT / kLanes;
    __shared__ uint32_t part[QT / 64];
    const int row = blockIdx.x * kRows + (kWaves == 1 ? (int)threadIdx.x / 64 : 0);
    if (row >= rows) return;  // whole waves, and whole workgroups where they meet at a barrier
    const int t = threadIdx.x % kLanes, chunks = (cols + 7) / 8;
    const size_t at = (size_t)row * ldx;
    int8_t* const qr = q + (size_t)row * ldq;
    float v[kChunks ? kChunks : 1][8];
    uint32_t m = 0;
    if constexpr (kChunks > 0) {
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            const int c = t + i * kLanes;
            if (c < chunks) {
                row_chunk<kBf16, kGated>(x, x2, at, c, cols, v[i]);
                m = max_bits(v[i], m);
            }
        }
    } else {
        for (int c = t; c < chunks; c += kLanes) {
            row_chunk<kBf16, kGated>(x, x2, at, c, cols, v[0]);
            m = max_bits(v[0], m);
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, 64));
    if constexpr (kWaves > 1) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) m = max(m, part[w]);
    }
    const float top = __uint_as_float(m);
    const bool finite = m < 0x7f800000u;
    // 127 / top leaves fp32's range below 3.7e-37: the values of such a row (of
    // zeros too) are lifted by a power of two first
    const bool low = top < 0x1p-100f;
    const float inv = finite && m ? 1.f / (low ? top * 0x1p+64f : top) * 127.f : 0.f;
    if (t == 0) scale[row] = finite ? top / 127.f : __uint_as_float(0x7fc00000u);
    if constexpr (kChunks > 0) {
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            const int c = t + i * kLanes;
            if (c < chunks) {
                if (!finite || low)
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[i][k] = finite ? v[i][k] * 0x1p+64f : 0.f;
                store_q<kWhole>(qr + 8 * c, v[i], inv, 8 * c, cols);
            }
        }
    } else {
        for (int c = t; c < chunks; c += kLanes) {
            row_chunk<kBf16, kGated>(x, x2, at, c, cols, v[0]);
            if (!finite || low)
#pragma unroll
                for (int k = 0; k < 8; ++k) v[0][k] = finite ? v[0][k] * 0x1p+64f : 0.f;
            store_q<kWhole>(qr + 8 * c, v[0], inv, 8 * c, cols);
        }
    }
}

template <bool kBf16, bool kGated, bool kWhole>
void launch(const void* x, const void* x2, size_t ldx, int8_t* q, size_t ldq, float* scale, int rows, int cols, hipStream_t s) {
    const int by4 = (rows + 3) / 4;
    if (cols <= 512)
        quantize_kernel<kBf16, kGated, 1, 1, kWhole><<<by4, QT, 0, s>>>(x, x2, ldx, q, ldq, scale, rows, cols);
    else if (rows >= kManyRows && cols <= 2048)
        quantize_kernel<kBf16, kGated, 1, 4, kWhole><<<by4, QT, 0, s>>>(x, x2, ldx, q, ldq, scale, rows, cols);
    else if (cols <= 2048)
        quantize_kernel<kBf16, kGated, 4, 1, kWhole><<<rows, QT, 0, s>>>(x, x2, ldx, q, ldq, scale, rows, cols);
    else if (cols <= 4096)
        quantize_kernel<kBf16, kGated, 4, 2, kWhole><<<rows, QT, 0, s>>>(x, x2, ldx, q, ldq, scale, rows, cols);
    else if (cols <= 16384)
        quantize_kernel<kBf16, kGated, 4, 8, kWhole><<<rows, QT, 0, s>>>(x, x2, ldx, q, ldq, scale, rows, cols);
    else
        quantize_kernel<kBf16, kGated, 4, 0, kWhole><<<rows, QT, 0, s>>>(x, x2, ldx, q, ldq, scale, rows, cols);
}
template <bool kBf16, bool kGated>
void launch(const void* x, const void* x2, size_t ldx, int8_t* q, size_t ldq, float* scale, int rows, int cols, hipStream_t s) {
    if (cols % 8 == 0) launch<kBf16, kGated, true>(x, x2, ldx, q, ldq, scale, rows, cols, s);
    else launch<kBf16, kGated, false>(x, x2, ldx, q, ldq, scale, rows, cols, s);
}

}  // namespace

hipError_t launch_quantize_rows(const void* x, const void* x2, size_t ldx, int8_t* q, size_t ldq, float* scale, int rows, int cols,
                                bool bf16, hipStream_t s) {
    if (rows <= 0) return hipSuccess;
    constexpr int kSlice = 1 << 22;  // a launch's threads are fewer than 2^32
    for (; rows > kSlice; rows -= kSlice) {
        const hipError_t err = launch_quantize_rows(x, x2, ldx, q, ldq, scale, kSlice, cols, bf16, s);
        if (err != hipSuccess) return err;
        const size_t step = kSlice * ldx * (bf16 ? 2 : 4);
        x = reinterpret_cast<const char*>(x) + step;
        if (x2) x2 = reinterpret_cast<const char*>(x2) + step;
        q += kSlice * ldq;
        scale += kSlice;
    }
    if (bf16 && x2) launch<true, true>(x, x2, ldx, q, ldq, scale, rows, cols, s);
    else if (bf16) launch<true, false>(x, x2, ldx, q, ldq, scale, rows, cols, s);
    else if (x2) launch<false, true>(x, x2, ldx, q, ldq, scale, rows, cols, s);
    else launch<false, false>(x, x2, ldx, q, ldq, scale, rows, cols, s);
    return hipGetLastError();
}

}  // namespace flexmoe
