// Root-mean-square norm of rows (gfx950), after the addition of a residual, as
// bf16 or fp32 rows, as rows in 8 bits with a scale each, or both; and its
// backward.
//
//   r = x + residual (rounded to the rows' type)    n = r / sqrt(mean(r^2) + eps)
//   y = n w          q = round(y * ((1 / m) * 127)), scale = m / 127, m = max|y|
//
//   g = dy w         dx = rstd (g - n mean(g n)) + dr         dw = sum of dy n
//
// y is rounded once; the 8-bit rows are rounded from the fp32 y.  What is
// normalised is the rounded r, which is what the backward has in hand.
//
// Bound by memory.  A row is read once and kept in registers between its sum and
// its output (up to 16384 values; longer rows are read again); all of a row's
// values, its residual's and the weights are asked for before the first is used.
// Rows of up to 512 values, in large calls 1024, take one wave each, longer ones a
// workgroup.  8192 x 4096 bf16 with a residual: 42 us, 6.4 TB/s of rows that in part
// lie in the last cache; 64 x 4096 in 8 bits: 4.4 us.
//
// The backward's workgroups take every G-th row, ask for the next one before this
// one's sum (rows of up to 8192 bf16 values: the registers end there) and keep their
// part of dw in registers; the parts are summed in order by a second launch, so that
// the result does not depend on which workgroup ends first.  4133 x 2048 bf16: 17.3 us
// with the join, 3.9 TB/s; 16384 x 8192: 212 us, 5.1 TB/s.
#include <algorithm>

#include "error.h"
#include "flexmoe.h"
#include "rows.h"

using namespace flexmoe;

namespace {

constexpr int NT = 256;
constexpr int kManyRows = 1024;
constexpr int kInRegisters = 16384;  // values of a row
// Workgroups of the backward: fewer ask for too little at once, more write and join more parts of dw.  4133 x 2048 bf16:
// 19.7 us with 256, 17.4 with 512, 19.0 with 1024, 24.4 with 2048.
constexpr int kParts = 512;

struct NormArgs {
    const void *x, *res, *w;
    void *r, *y;
    int8_t* q;
    float *scale, *rstd;
    size_t ldx, ldres, ldr, ldy, ldq;
    int rows, cols;
    float eps, inv_cols;
};

template <bool kBf16>
__device__ __forceinline__ float add_rounded(float a, float b) {
    return kBf16 ? bf16_to_f32(f32_to_bf16(a + b)) : a + b;
}

// Chunk c of row `row` as it lies in memory.  Chunks behind the row's last are asked for as that one: a request
// that depends on no condition waits for none before it, so all of a row's are on their way at once.
template <bool kBf16>
__device__ __forceinline__ Raw8<kBf16> request(const void* p, size_t at, int c, int cols) {
    const int last = (cols - 1) / 8, cc = min(c, last), left = cols - 8 * cc;
    const u32x4* u = reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(p) + (at + 8 * cc) * elem_size<kBf16>());
    Raw8<kBf16> r;
    r.w[0] = u[0];
    if constexpr (!kBf16) r.w[1] = u[left > 4];
    return r;
}

// A requested chunk's values, 0 behind the row's end.
template <bool kBf16>
__device__ __forceinline__ void arrived(const Raw8<kBf16>& raw, int c, int cols, float (&v)[8]) {
    unpack8<kBf16>(raw, v);
    const int left = cols - 8 * c;
    if (left < 8)
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = k < left ? v[k] : 0.f;
}

// v += the residual's chunk c, rounded, and written as r's.
template <bool kBf16>
__device__ __forceinline__ void add_chunk(const NormArgs& a, size_t row, int c, const Raw8<kBf16>& res, float (&v)[8]) {
    float u[8];
    arrived<kBf16>(res, c, a.cols, u);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = add_rounded<kBf16>(v[k], u[k]);
    store8<kBf16>(a.r, row * a.ldr + 8 * c, a.cols - 8 * c, v);
}

__device__ __forceinline__ float squares(const float (&v)[8], float lift, float s) {
#pragma unroll
    for (int k = 0; k < 8; ++k) s = fmaf(v[k] * lift, v[k] * lift, s);
    return s;
}

template <bool kWBf16>
__device__ __forceinline__ void normed(const Raw8<kWBf16>& raw, int c, int cols, float rstd, float (&v)[8]) {
    float w[8];
    arrived<kWBf16>(raw, c, cols, w);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = v[k] * rstd * w[k];
}

__device__ __forceinline__ uint32_t max_bits(const float (&v)[8], uint32_t m) {
#pragma unroll
    for (int k = 0; k < 8; ++k) m = max(m, __float_as_uint(v[k]) & 0x7fffffffu);
    return m;
}

__device__ __forceinline__ void store_q(int8_t* q, int left, const float (&v)[8], float inv) {
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int n = (int)fminf(fmaxf(rintf(v[k] * inv), -127.f), 127.f);
        w[k >> 2] |= (uint32_t)(n & 255) << (8 * (k & 3));
    }
    if (left >= 8) {
        *reinterpret_cast<uint2*>(q) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
        for (int k = 0; k < 7; ++k)
            if (k < left) q[k] = (int8_t)(w[k >> 2] >> (8 * (k & 3)));
    }
}

// kWaves waves per row, kChunks 8-value chunks per lane in registers (0: read again).
template <bool kBf16, bool kWBf16, int kWaves, int kChunks>
__global__ __launch_bounds__(NT) void norm_kernel(const NormArgs a) {
    constexpr int kLanes = 64 * kWaves, kRows = NT / kLanes;
    __shared__ float part[3][NT / 64];
    const int row = blockIdx.x * kRows + (kWaves == 1 ? (int)threadIdx.x / 64 : 0);
    if (row >= a.rows) return;  // whole waves, and whole workgroups where they meet at a barrier
    const int t = threadIdx.x % kLanes, chunks = (a.cols + 7) / 8;
    float v[kChunks ? kChunks : 1][8];
    const void* const again = a.res ? a.r : a.x;  // where a row that is too long for the registers is read again
    const size_t again_at = (size_t)row * (a.res ? a.ldr : a.ldx);

    // the weights are on their way, too, before the first sum
    Raw8<kWBf16> w[kChunks ? kChunks : 1];
    Raw8<kBf16> x[kChunks ? kChunks : 1], res[kChunks ? kChunks : 1];
    if constexpr (kChunks > 0) {
#pragma unroll
        for (int i = 0; i < kChunks; ++i) x[i] = request<kBf16>(a.x, (size_t)row * a.ldx, t + i * kLanes, a.cols);
        if (a.res)
#pragma unroll
            for (int i = 0; i < kChunks; ++i) res[i] = request<kBf16>(a.res, (size_t)row * a.ldres, t + i * kLanes, a.cols);
#pragma unroll
        for (int i = 0; i < kChunks; ++i) w[i] = request<kWBf16>(a.w, 0, t + i * kLanes, a.cols);
        __builtin_amdgcn_sched_barrier(0);
    }

    // f(chunk, its values, its weights) for the chunks of this lane; `first`: from x and the residual
    auto each = [&](bool first, auto&& f) {
        if constexpr (kChunks > 0) {
#pragma unroll
            for (int i = 0; i < kChunks; ++i) {
                const int c = t + i * kLanes;
                if (c < chunks) {
                    if (first) {
                        arrived<kBf16>(x[i], c, a.cols, v[i]);
                        if (a.res) add_chunk<kBf16>(a, row, c, res[i], v[i]);
                    }
                    f(c, v[i], w[i]);
                }
            }
        } else {
            for (int c = t; c < chunks; c += kLanes) {
                x[0] = first ? request<kBf16>(a.x, (size_t)row * a.ldx, c, a.cols) : request<kBf16>(again, again_at, c, a.cols);
                if (first && a.res) res[0] = request<kBf16>(a.res, (size_t)row * a.ldres, c, a.cols);
                if (!first) w[0] = request<kWBf16>(a.w, 0, c, a.cols);
                arrived<kBf16>(x[0], c, a.cols, v[0]);
                if (first && a.res) add_chunk<kBf16>(a, row, c, res[0], v[0]);
                f(c, v[0], w[0]);
            }
        }
    };

    float s = 0.f;
    each(true, [&](int, const float (&u)[8], const Raw8<kWBf16>&) { s = squares(u, 1.f, s); });
    s = sum_over_waves<kWaves>(s, part[0]);
    float rstd = 1.f / sqrtf(s * a.inv_cols + a.eps);
    if (!(s <= 3.0e38f)) {  // the squares left fp32's range (or a value is no number): all values 2^80 smaller
        float s2 = 0.f;
        each(false, [&](int, const float (&u)[8], const Raw8<kWBf16>&) { s2 = squares(u, 0x1p-80f, s2); });
        s2 = sum_over_waves<kWaves>(s2, part[1]);
        rstd = 0x1p-80f / sqrtf(s2 * a.inv_cols);  // eps is nothing beside such squares
    }
    if (a.rstd && t == 0) a.rstd[row] = rstd;
    uint32_t m = 0;
    const bool keeps = kChunks > 0;
    if (keeps || a.q) {
        each(false, [&](int c, float (&u)[8], const Raw8<kWBf16>& ww) {
            normed<kWBf16>(ww, c, a.cols, rstd, u);
            if (a.q) m = max_bits(u, m);
            if (a.y) store8<kBf16>(a.y, (size_t)row * a.ldy + 8 * c, a.cols - 8 * c, u);
        });
    } else {
        each(false, [&](int c, float (&u)[8], const Raw8<kWBf16>& ww) {
            normed<kWBf16>(ww, c, a.cols, rstd, u);
            store8<kBf16>(a.y, (size_t)row * a.ldy + 8 * c, a.cols - 8 * c, u);
        });
    }
    if (!a.q) return;
    m = max_over_waves<kWaves>(m, reinterpret_cast<uint32_t*>(part[2]));
    const float top = __uint_as_float(m);
    const bool finite = m < 0x7f800000u;
    // 127 / top leaves fp32's range below 3.7e-37: the values of such a row are lifted first
    const bool low = top < 0x1p-100f;
    const float inv = finite && m ? 1.f / (low ? top * 0x1p+64f : top) * 127.f : 0.f;
    if (t == 0) a.scale[row] = finite ? top / 127.f : __uint_as_float(0x7fc00000u);
    each(false, [&](int c, float (&u)[8], const Raw8<kWBf16>& ww) {
        if (!keeps) normed<kWBf16>(ww, c, a.cols, rstd, u);
        if (!finite || low)
#pragma unroll
            for (int k = 0; k < 8; ++k) u[k] = finite ? u[k] * 0x1p+64f : 0.f;
        store_q(a.q + (size_t)row * a.ldq + 8 * c, a.cols - 8 * c, u, inv);
    });
}

struct GradArgs {
    const void *dy, *r, *w, *dr;
    const float* rstd;
    void* dx;
    float* parts;  // [gridDim.x][ldp], or NULL
    size_t lddy, ldr, lddr, lddx, ldp;
    int rows, cols;
    float inv_cols;
};

template <bool kBf16, bool kWBf16, int kWaves, int kChunks>
__global__ __launch_bounds__(NT) void norm_grad_kernel(const GradArgs a) {
    constexpr int kLanes = 64 * kWaves, kRows = NT / kLanes, kKept = kChunks ? kChunks : 1;
    constexpr bool kAhead = kChunks <= (kBf16 ? 4 : 2);
    __shared__ float part[2][NT / 64];
    __shared__ float joined[kWaves == 1 ? 512 * kKept : 1];  // a row of dw, for the waves of a workgroup
    const int t = threadIdx.x % kLanes, chunks = (a.cols + 7) / 8;
    const int slot = blockIdx.x * kRows + (kWaves == 1 ? (int)threadIdx.x / 64 : 0), step = gridDim.x * kRows;
    float dw[kKept][8] = {};
    struct Row {
        Raw8<kBf16> dy[kKept], r[kKept], dr[kKept];
        float rstd;
    };
    Raw8<kWBf16> w[kKept];
    auto ask = [&](Row& q, int i, int c, int row) {
        q.dy[i] = request<kBf16>(a.dy, (size_t)row * a.lddy, c, a.cols);
        q.r[i] = request<kBf16>(a.r, (size_t)row * a.ldr, c, a.cols);
        q.dr[i] = request<kBf16>(a.dr ? a.dr : a.dy, (size_t)row * (a.dr ? a.lddr : a.lddy), c, a.cols);
    };
    auto ask_row = [&](Row& q, int row) {
        q.rstd = a.rstd[row];
#pragma unroll
        for (int i = 0; i < kKept; ++i) ask(q, i, t + i * kLanes, row);
        __builtin_amdgcn_sched_barrier(0);
    };
    // n and g = dy w of a chunk
    auto read = [&](const Row& q, int i, int c, float (&n)[8], float (&dy)[8], float (&g)[8]) {
        float ww[8];
        arrived<kBf16>(q.dy[i], c, a.cols, dy);
        arrived<kBf16>(q.r[i], c, a.cols, n);
        arrived<kWBf16>(w[i], c, a.cols, ww);
#pragma unroll
        for (int k = 0; k < 8; ++k) n[k] *= q.rstd, g[k] = dy[k] * ww[k];
    };
    auto write = [&](const Row& q, int i, int c, int row, const float (&n)[8], const float (&g)[8], float mean) {
        float o[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) o[k] = q.rstd * (g[k] - n[k] * mean);
        if (a.dr) {
            float u[8];
            arrived<kBf16>(q.dr[i], c, a.cols, u);
#pragma unroll
            for (int k = 0; k < 8; ++k) o[k] += u[k];
        }
        store8<kBf16>(a.dx, (size_t)row * a.lddx + 8 * c, a.cols - 8 * c, o);
    };
    Row now, next;
    if constexpr (kChunks > 0) {
#pragma unroll
        for (int i = 0; i < kChunks; ++i) w[i] = request<kWBf16>(a.w, 0, t + i * kLanes, a.cols);
        if (slot < a.rows) ask_row(now, slot);
    }
    int turn = 0;
    for (int row = slot; row < a.rows; row += step, turn ^= 1) {  // the same rows in all waves that meet at a barrier
        float dot = 0.f, n[8], dy[8], g[8];
        if constexpr (kChunks > 0) {
            if constexpr (kAhead) ask_row(next, min(row + step, a.rows - 1));
#pragma unroll
            for (int i = 0; i < kChunks; ++i)
                if (t + i * kLanes < chunks) {
                    read(now, i, t + i * kLanes, n, dy, g);
#pragma unroll
                    for (int k = 0; k < 8; ++k) dot = fmaf(g[k], n[k], dot), dw[i][k] = fmaf(dy[k], n[k], dw[i][k]);
                }
        } else {
            now.rstd = a.rstd[row];
            for (int c = t; c < chunks; c += kLanes) {
                ask(now, 0, c, row);
                w[0] = request<kWBf16>(a.w, 0, c, a.cols);
                read(now, 0, c, n, dy, g);
#pragma unroll
                for (int k = 0; k < 8; ++k) dot = fmaf(g[k], n[k], dot);
            }
        }
        const float mean = sum_over_waves<kWaves>(dot, part[turn]) * a.inv_cols;
        if constexpr (kChunks > 0) {
#pragma unroll
            for (int i = 0; i < kChunks; ++i)
                if (t + i * kLanes < chunks) {
                    read(now, i, t + i * kLanes, n, dy, g);
                    write(now, i, t + i * kLanes, row, n, g, mean);
                }
            if constexpr (kAhead) now = next;
            else if (row + step < a.rows) ask_row(now, row + step);
        } else {
            // the part of dw lies in memory, each value in one thread's hands
            for (int c = t; c < chunks; c += kLanes) {
                ask(now, 0, c, row);
                w[0] = request<kWBf16>(a.w, 0, c, a.cols);
                read(now, 0, c, n, dy, g);
                if (a.parts) {
                    float* const p = a.parts + blockIdx.x * a.ldp;
                    float u[8] = {};
                    if (row != slot) load8<false>(p, 8 * c, 8, u);
#pragma unroll
                    for (int k = 0; k < 8; ++k) u[k] = fmaf(dy[k], n[k], u[k]);
                    store8<false>(p, 8 * c, 8, u);
                }
                write(now, 0, c, row, n, g, mean);
            }
        }
    }
    if (kChunks == 0 || !a.parts) return;
    float* const p = a.parts + blockIdx.x * a.ldp;
    if constexpr (kWaves == 1) {
        for (int turn_of = 0; turn_of < kRows; ++turn_of) {
            if ((int)threadIdx.x / 64 == turn_of)
#pragma unroll
                for (int i = 0; i < kKept; ++i)
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        float* const at = &joined[(i * 64 + t) * 8 + k];
                        *at = turn_of ? *at + dw[i][k] : dw[i][k];
                    }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < chunks; c += NT) {
            float u[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) u[k] = joined[c * 8 + k];
            store8<false>(p, 8 * c, 8, u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kKept; ++i)
            if (t + i * kLanes < chunks) store8<false>(p, 8 * (t + i * kLanes), 8, dw[i]);
    }
}

// dw = (accumulate ? dw : 0) + the parts in order: 64 columns a workgroup, 16 waves a part of the parts each.
__global__ __launch_bounds__(1024) void norm_join_kernel(const float* parts, size_t ldp, int count, float* dw, int cols, int accumulate) {
    __shared__ float sums[16][64];
    const int wave = threadIdx.x / 64, lane = threadIdx.x & 63, c = blockIdx.x * 64 + lane;
    const int per = (count + 15) / 16, p0 = wave * per, p1 = min(count, p0 + per);
    float s = 0.f;
    if (c < cols)
#pragma unroll 8
        for (int p = p0; p < p1; ++p) s += parts[p * ldp + c];
    sums[wave][lane] = s;
    __syncthreads();
    if (wave || c >= cols) return;
    s = accumulate ? dw[c] : 0.f;
#pragma unroll
    for (int w = 0; w < 16; ++w) s += sums[w][lane];
    dw[c] = s;
}

// A wave for each row needs no barrier, but its lanes hold more: 16384 x 1024 bf16 22.5 us (8 bits 21.3, backward
// 28.4), with a workgroup each 24.9 (28.8, 40.8); 16 x 1024 2.6 us (5.4), with a workgroup 2.4 (4.6); 16384 x 512
// 11.6 (16.3), 15.2 (31.4); 4133 x 2048 12.1 (19.5), with a workgroup 11.8 (17.3).
bool wave_per_row(int rows, int cols) { return cols <= 512 || (rows >= kManyRows && cols <= 1024); }

template <bool kBf16, bool kWBf16>
hipError_t launch_norm(const NormArgs& a, hipStream_t s) {
    const int by4 = (a.rows + 3) / 4;
    if (a.cols <= 512) norm_kernel<kBf16, kWBf16, 1, 1><<<by4, NT, 0, s>>>(a);
    else if (wave_per_row(a.rows, a.cols)) norm_kernel<kBf16, kWBf16, 1, 2><<<by4, NT, 0, s>>>(a);
    else if (a.cols <= 2048) norm_kernel<kBf16, kWBf16, 4, 1><<<a.rows, NT, 0, s>>>(a);
    else if (a.cols <= 4096) norm_kernel<kBf16, kWBf16, 4, 2><<<a.rows, NT, 0, s>>>(a);
    else if (a.cols <= 8192) norm_kernel<kBf16, kWBf16, 4, 4><<<a.rows, NT, 0, s>>>(a);
    else if (a.cols <= kInRegisters) norm_kernel<kBf16, kWBf16, 4, 8><<<a.rows, NT, 0, s>>>(a);
    else norm_kernel<kBf16, kWBf16, 4, 0><<<a.rows, NT, 0, s>>>(a);
    return hipGetLastError();
}

template <bool kBf16, bool kWBf16>
hipError_t launch_grad(const GradArgs& a, int grid, hipStream_t s) {
    if (a.cols <= 512) norm_grad_kernel<kBf16, kWBf16, 1, 1><<<grid, NT, 0, s>>>(a);
    else if (wave_per_row(a.rows, a.cols)) norm_grad_kernel<kBf16, kWBf16, 1, 2><<<grid, NT, 0, s>>>(a);
    else if (a.cols <= 2048) norm_grad_kernel<kBf16, kWBf16, 4, 1><<<grid, NT, 0, s>>>(a);
    else if (a.cols <= 4096) norm_grad_kernel<kBf16, kWBf16, 4, 2><<<grid, NT, 0, s>>>(a);
    else if (a.cols <= 8192) norm_grad_kernel<kBf16, kWBf16, 4, 4><<<grid, NT, 0, s>>>(a);
    else if (a.cols <= kInRegisters) norm_grad_kernel<kBf16, kWBf16, 4, 8><<<grid, NT, 0, s>>>(a);
    else norm_grad_kernel<kBf16, kWBf16, 4, 0><<<grid, NT, 0, s>>>(a);
    return hipGetLastError();
}

// Workgroups of the backward.
int grad_grid(int rows, int cols) {
    const int per = wave_per_row(rows, cols) ? 4 : 1;
    return (int)std::min<long long>(((long long)rows + per - 1) / per, kParts);
}

size_t part_stride(int cols) { return ((size_t)cols + 63) / 64 * 64; }

bool misaligned(const void* p, uintptr_t mask) { return ((uintptr_t)p & mask) != 0; }

constexpr long long kMaxStride = 1 << 21;

struct NormStrides {
    long long x, res, r, y, q;
};

int check_norm(const flexmoe_norm_desc* D, int rows, const char* who, NormStrides* st) {
    if (!D) return fail(FLEXMOE_EINVAL, "%s: desc is NULL", who);
    for (int dt : {D->dtype, D->w_dtype})
        if (dt != FLEXMOE_F32 && dt != FLEXMOE_BF16)
            return fail(FLEXMOE_EDTYPE, "%s: dtype %d is neither FLEXMOE_F32 nor FLEXMOE_BF16", who, dt);
    if (D->cols < 1 || D->cols > kMaxStride) return fail(FLEXMOE_ESHAPE, "%s: cols = %d outside [1, 2^21]", who, D->cols);
    if (D->max_rows < 0 || D->max_rows > (1 << 30)) return fail(FLEXMOE_ESHAPE, "%s: max_rows = %d outside [0, 2^30]", who, D->max_rows);
    if (!(D->eps >= 1e-30f && D->eps <= 1.f)) return fail(FLEXMOE_EINVAL, "%s: eps = %g outside [1e-30, 1]", who, (double)D->eps);
    const int unit = D->dtype == FLEXMOE_BF16 ? 8 : 4;
    *st = NormStrides{D->ldx ? D->ldx : D->cols, D->ldres ? D->ldres : D->cols, D->ldr ? D->ldr : D->cols, D->ldy ? D->ldy : D->cols,
                      D->ldq ? D->ldq : D->cols};
    const struct { long long ld; const char* name; } all[] = {{st->x, "ldx"}, {st->res, "ldres"}, {st->r, "ldr"}, {st->y, "ldy"}};
    for (const auto& s : all)
        if (s.ld < D->cols || s.ld > kMaxStride || s.ld % unit)
            return fail(FLEXMOE_ESHAPE, "%s: %s = %lld must be a multiple of %d in [%d, 2^21]", who, s.name, s.ld, unit, D->cols);
    if (rows < 0) return fail(FLEXMOE_EINVAL, "%s: rows = %d is negative", who, rows);
    if (rows > D->max_rows) return fail(FLEXMOE_ESHAPE, "%s: rows = %d above max_rows = %d", who, rows, D->max_rows);
    return FLEXMOE_OK;
}

size_t grad_bytes(int rows, int cols) {
    // a wave for each row starts at kManyRows rows: fewer workgroups there than for a few rows less
    const int grid = std::max(grad_grid(rows, cols), grad_grid(std::min(rows, kManyRows - 1), cols));
    return std::max<size_t>(256, (size_t)grid * part_stride(cols) * sizeof(float));
}

}  // namespace

extern "C" {

int flexmoe_rms_norm(const flexmoe_norm_desc* desc, int32_t rows, const void* x, const void* residual, const void* w, void* r, void* y,
                     void* q, float* scale, float* rstd, void* stream) {
    const char* who = "rms_norm";
    NormStrides st;
    const int rc = check_norm(desc, rows, who, &st);
    if (rc) return rc;
    if (q && (st.q < desc->cols || st.q > kMaxStride || st.q % 16))
        return fail(FLEXMOE_ESHAPE, "%s: ldq = %lld must be a multiple of 16 in [%d, 2^21]", who, st.q, desc->cols);
    if (rows == 0) return FLEXMOE_OK;
    if (!x || !w || (!y && !q)) return fail(FLEXMOE_EINVAL, "%s: a pointer is NULL", who);
    if (!q != !scale) return fail(FLEXMOE_EINVAL, "%s: q and scale go together", who);
    if (!residual != !r) return fail(FLEXMOE_EINVAL, "%s: residual and r go together", who);
    if (y && (y == x || y == residual || y == r)) return fail(FLEXMOE_EINVAL, "%s: y must be a buffer of its own", who);
    for (const void* p : {x, residual, w, (const void*)r, (const void*)y, (const void*)q})
        if (misaligned(p, 15)) return fail(FLEXMOE_EINVAL, "%s: rows and weights must be 16-byte aligned", who);
    if (misaligned(scale, 3) || misaligned(rstd, 3)) return fail(FLEXMOE_EINVAL, "%s: scale and rstd must be 4-byte aligned", who);
    const bool bf16 = desc->dtype == FLEXMOE_BF16, wbf16 = desc->w_dtype == FLEXMOE_BF16;
    const size_t es = bf16 ? 2 : 4;
    constexpr int kSlice = 1 << 22;  // a launch's threads are fewer than 2^32
    for (long long at = 0; at < rows; at += kSlice) {
        NormArgs a;
        auto rows_at = [&](const void* p, long long ld, size_t size) {
            return p ? (void*)(reinterpret_cast<const char*>(p) + (size_t)at * ld * size) : nullptr;
        };
        a.x = rows_at(x, st.x, es), a.res = rows_at(residual, st.res, es), a.r = rows_at(r, st.r, es), a.y = rows_at(y, st.y, es);
        a.q = (int8_t*)rows_at(q, st.q, 1), a.scale = scale ? scale + at : nullptr, a.rstd = rstd ? rstd + at : nullptr, a.w = w;
        a.ldx = st.x, a.ldres = st.res, a.ldr = st.r, a.ldy = st.y, a.ldq = st.q;
        a.rows = (int)std::min<long long>(kSlice, rows - at), a.cols = desc->cols, a.eps = desc->eps, a.inv_cols = 1.f / desc->cols;
        const hipStream_t s = (hipStream_t)stream;
        const hipError_t err = bf16 ? (wbf16 ? launch_norm<true, true>(a, s) : launch_norm<true, false>(a, s))
                                    : (wbf16 ? launch_norm<false, true>(a, s) : launch_norm<false, false>(a, s));
        if (err != hipSuccess) return hip_fail(err, who);
    }
    return FLEXMOE_OK;
}

size_t flexmoe_rms_norm_workspace_bytes(const flexmoe_norm_desc* desc, int32_t rows) {
    NormStrides st;
    if (check_norm(desc, rows, "rms_norm_workspace_bytes", &st)) return 0;
    return grad_bytes(rows, desc->cols);
}

int flexmoe_rms_norm_backward(const flexmoe_norm_desc* desc, int32_t rows, const void* dy, const void* r, const void* w, const float* rstd,
                              const void* dr, void* dx, float* dw, int32_t accumulate, void* workspace, size_t workspace_bytes,
                              void* stream) {
    const char* who = "rms_norm_backward";
    NormStrides st;
    const int rc = check_norm(desc, rows, who, &st);
    if (rc) return rc;
    if (accumulate != 0 && accumulate != 1) return fail(FLEXMOE_EINVAL, "%s: accumulate must be 0 or 1 (got %d)", who, accumulate);
    if (rows > 0 && (!dy || !r || !w || !rstd || !dx)) return fail(FLEXMOE_EINVAL, "%s: a pointer is NULL", who);
    for (const void* p : {dy, r, w, dr, (const void*)dx})
        if (misaligned(p, 15)) return fail(FLEXMOE_EINVAL, "%s: rows and weights must be 16-byte aligned", who);
    if (misaligned(dw, 3) || misaligned(rstd, 3)) return fail(FLEXMOE_EINVAL, "%s: dw and rstd must be 4-byte aligned", who);
    const size_t need = grad_bytes(rows, desc->cols);
    if (dw && rows > 0) {
        if (!workspace || workspace_bytes < need)
            return fail(FLEXMOE_EWORKSPACE, "%s: workspace of %zu bytes, %zu needed", who, workspace ? workspace_bytes : 0, need);
        if (misaligned(workspace, 255)) return fail(FLEXMOE_EWORKSPACE, "%s: workspace must be 256-byte aligned", who);
    }
    const hipStream_t s = (hipStream_t)stream;
    const int grid = grad_grid(rows, desc->cols);
    if (rows > 0) {
        GradArgs a;
        a.dy = dy, a.r = r, a.w = w, a.dr = dr, a.rstd = rstd, a.dx = dx, a.parts = dw ? (float*)workspace : nullptr;
        a.lddy = st.y, a.ldr = st.r, a.lddr = st.res, a.lddx = st.x, a.ldp = part_stride(desc->cols);
        a.rows = rows, a.cols = desc->cols, a.inv_cols = 1.f / desc->cols;
        const bool bf16 = desc->dtype == FLEXMOE_BF16, wbf16 = desc->w_dtype == FLEXMOE_BF16;
        const hipError_t err = bf16 ? (wbf16 ? launch_grad<true, true>(a, grid, s) : launch_grad<true, false>(a, grid, s))
                                    : (wbf16 ? launch_grad<false, true>(a, grid, s) : launch_grad<false, false>(a, grid, s));
        if (err != hipSuccess) return hip_fail(err, who);
    }
    if (dw && !(rows == 0 && accumulate)) {
        norm_join_kernel<<<(desc->cols + 63) / 64, 1024, 0, s>>>((const float*)workspace, part_stride(desc->cols), rows > 0 ? grid : 0, dw,
                                                                 desc->cols, accumulate);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return hip_fail(err, who);
    }
    return FLEXMOE_OK;
}

}  // extern "C"
