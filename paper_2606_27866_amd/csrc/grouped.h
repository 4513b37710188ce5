// Matrix products over the experts' ragged row groups: what one launch is
// given, how a workgroup finds its tile, and how operands reach LDS and the
// matrix cores (gfx950).
//
// Every form is C[r][c] = sum_d A(r, d) B(c, d) for one group at a time:
//   form          r         c   d         A                 B
//   kForward      row       n   k         x [row][k]        W [n][k]
//   kInputGrad    row       k   n         dy [row][n]       W [n][k]
//   kWeightGrad   n         k   row       dy [row][n]       x [row][k]
// An operand is contiguous in d ("along": x and W in the forward, dy in the
// input gradient) or in its own index ("across": W in the input gradient, both
// in the weight gradient).
#pragma once

#include "mfma_tile.h"

namespace flexmoe {

enum GroupedForm : int { kForward = 0, kInputGrad = 1, kWeightGrad = 2 };
enum GroupedElem : int { kElemBf16 = 0, kElemF32 = 1, kElemI8 = 2 };

struct GroupedParams {
    const void *a, *b;
    void* c;
    const int32_t* offsets;   // [E + 1] row ranges of the groups
    const int32_t* keep;      // [E] widths, or NULL
    const float *sa, *sb;     // int8: a scale for each row of x and of W
    void* partial;            // splits > 1: the partial sums of every split
    size_t lda, ldb, ldc;     // row strides in elements (of the buffers, not of A and B)
    int E, R, N, K;           // groups, rows of x, W_e is [N][K]
    int keep_axis;            // 0: none, 1: keep limits N, 2: keep limits K
    int tiles_c;              // column tiles of C
    int tiles_r;              // weight gradient: row tiles of C
    int splits;               // parts of the reduction, each a workgroup's
    int out_bf16;             // C is bf16 (else fp32)
    int accumulate;           // weight gradient: C += instead of C =
};

// One workgroup's part: C rows [r0, r0 + nr) and columns [c0, ...) of group e,
// reduction over [d0, d1).
struct GroupedTile {
    int e, row0, rows;        // the group and its rows of x
    int r0, r1;               // C rows of the tile, inside the group
    int c0;                   // first C column of the tile
    int rlim, clim;           // C rows and columns that exist; the rest are zeros
    int d0, d1;               // the part of the reduction
    int split;
};

__device__ __forceinline__ int group_begin(const GroupedParams& p, int e) { return min(max(p.offsets[e], 0), p.R); }
__device__ __forceinline__ int group_width(const GroupedParams& p, int e, int full) {
    return p.keep ? min(max(p.keep[e], 0), full) : full;
}

// Row tiles of `bm` rows of every group, counted before a wave's eyes: lane l
// holds groups 4l .. 4l + 3.  Finds the group whose tiles hold number q.
// Returns false past the last tile.  All 64 lanes must be active and q uniform.
__device__ __forceinline__ bool find_group(const GroupedParams& p, int bm, int q, int& e, int& row0, int& rows, int& first,
                                           int& tiles) {
    static_assert(kMaxExperts <= 4 * kWave, "four groups per lane");
    const int lane = threadIdx.x & 63;
    int b[5], t[4], sum = 0;
#pragma unroll
    for (int j = 0; j < 5; ++j) b[j] = group_begin(p, min(4 * lane + j, p.E));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        t[j] = (max(b[j + 1] - b[j], 0) + bm - 1) / bm;
        sum += t[j];
    }
    const int incl = wave_incl_scan(sum);
    const unsigned long long owner = __ballot(incl - sum <= q && q < incl);
    if (!owner) return false;
    int base = incl - sum, f = 0, my = 0;
    bool found = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (!found && q < base + t[j]) {
            found = true;
            my = j;
            f = base;
        }
        if (!found) base += t[j];
    }
    const int lb = my == 0 ? b[0] : my == 1 ? b[1] : my == 2 ? b[2] : b[3];
    const int le = my == 0 ? b[1] : my == 1 ? b[2] : my == 2 ? b[3] : b[4];
    const int lt = my == 0 ? t[0] : my == 1 ? t[1] : my == 2 ? t[2] : t[3];
    const int src = __builtin_ctzll(owner);
    e = 4 * src + __builtin_amdgcn_readlane(my, src);
    row0 = __builtin_amdgcn_readlane(lb, src);
    rows = __builtin_amdgcn_readlane(le, src) - row0;
    first = __builtin_amdgcn_readlane(f, src);
    tiles = __builtin_amdgcn_readlane(lt, src);
    return true;
}

// Tile number L (row tiles of a group fastest, then column tiles, then parts
// of the reduction: neighbours share a weight tile).  kD is the depth of a K
// tile: parts of the reduction are whole K tiles.
template <int kForm>
__device__ __forceinline__ bool grouped_tile(const GroupedParams& p, int L, int bm, int bn, int kd, GroupedTile& t) {
    int mt, ct, depth;
    if constexpr (kForm == kWeightGrad) {
        const int per = p.tiles_r * p.tiles_c * p.splits;
        t.e = L / per;
        if (t.e >= p.E) return false;
        const int local = L - t.e * per;
        mt = local % p.tiles_r;
        ct = local / p.tiles_r % p.tiles_c;
        t.split = local / (p.tiles_r * p.tiles_c);
        t.row0 = group_begin(p, t.e);
        t.rows = max(group_begin(p, t.e + 1) - t.row0, 0);
        t.r0 = mt * bm;
        t.r1 = min(t.r0 + bm, p.N);
        depth = t.rows;
    } else {
        const int per = p.tiles_c * p.splits;
        int first, tiles;
        if (!find_group(p, bm, L / per, t.e, t.row0, t.rows, first, tiles)) return false;
        const int local = L - first * per;
        mt = local % tiles;
        ct = local / tiles % p.tiles_c;
        t.split = local / (tiles * p.tiles_c);
        // equal shares of the rows, in steps of 16
        const int step = ceil_div(ceil_div(t.rows, tiles), 16) * 16;
        t.r0 = mt * step;
        t.r1 = min(t.r0 + step, t.rows);
        depth = kForm == kForward ? p.K : p.N;
    }
    t.c0 = ct * bn;
    const int wn = p.keep_axis == 1 ? group_width(p, t.e, p.N) : p.N;
    const int wk = p.keep_axis == 2 ? group_width(p, t.e, p.K) : p.K;
    t.rlim = kForm == kWeightGrad ? wn : t.rows;
    t.clim = kForm == kForward ? wn : wk;
    if constexpr (kForm != kWeightGrad) depth = kForm == kForward ? wk : wn;
    t.d0 = 0;
    t.d1 = depth;
    if (p.splits > 1) {
        const int step = ceil_div(ceil_div(depth, p.splits), kd) * kd;
        t.d0 = min(t.split * step, depth);
        t.d1 = min(t.d0 + step, depth);
    }
    if (t.r0 >= t.rlim || t.c0 >= t.clim) t.d1 = t.d0;  // zeros only
    return t.r0 < t.r1;
}

// Tile number of a workgroup: runs of `run` consecutive tiles per XCD (the
// hardware hands consecutive workgroups to the 8 XCDs in turn), so that tiles
// which share operands meet in one L2.  The grid is a multiple of 8 * run.
__device__ __forceinline__ int xcd_tile(int run) {
    const int b = blockIdx.x, x = b & 7, i = b >> 3;
    return ((i / run) * 8 + x) * run + i % run;
}

namespace mfma {

typedef int32_t intx4 __attribute__((ext_vector_type(4)));

// Element types.  Whatever the type, a K tile is 128 bytes of an operand row
// and a fragment is 16 bytes of it (kPer elements), so that the LDS layout and
// the requests are the same.  mma multiplies a fragment pair: 4 lanes groups
// times 16 bytes of depth.
struct Bf16 {
    typedef bf16_t T;
    typedef bf16x8 Frag;
    typedef floatx4 Acc;
    static constexpr int kBytes = 2, kPer = 8, kDepth = 64;
    static __device__ __forceinline__ Acc mma(Frag a, Frag b, Acc c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
};
struct F32 {
    typedef float T;
    typedef floatx4 Frag;
    typedef floatx4 Acc;
    static constexpr int kBytes = 4, kPer = 4, kDepth = 32;
    // lane group g holds depths 4g .. 4g + 3; product j takes the j-th of each
    static __device__ __forceinline__ Acc mma(Frag a, Frag b, Acc c) {
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
        return c;
    }
};
struct I8 {
    typedef int8_t T;
    typedef intx4 Frag;
    typedef intx4 Acc;
    static constexpr int kBytes = 1, kPer = 16, kDepth = 128;
    static __device__ __forceinline__ Acc mma(Frag a, Frag b, Acc c) {
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
    }
};

// The elements of a fragment from the `valid`-th on set to zero.
template <typename E>
__device__ __forceinline__ typename E::Frag head(typename E::Frag f, int valid) {
    u32x4 v = __builtin_bit_cast(u32x4, f);
    const int bytes = valid * E::kBytes;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const int n = bytes - 4 * w;
        v[w] &= n >= 4 ? 0xffffffffu : n <= 0 ? 0u : (1u << (8 * n)) - 1u;
    }
    return __builtin_bit_cast(typename E::Frag, v);
}

// "Across" tiles: LDS rows are depths, each W own-index values long (kBytes *
// W bytes).  The 16-byte chunks of a row are XOR-ed with depth bits so that a
// fragment read spreads over all 64 banks.  bf16: a transposing read takes 32
// bytes of each of 16 depths 8g + i (g = lane / 16, i < 4): the 32-byte unit is
// XOR-ed with (i, g & 1).  fp32: plain reads take 64 bytes of depths 4g + j:
// the 64-byte unit is XOR-ed with g.
template <typename E>
__device__ __forceinline__ int across_chunk(int depth, int chunk) {
    if constexpr (E::kBytes == 2) return chunk ^ (((depth & 3) | ((depth >> 3) & 1) << 2) << 1);
    else return chunk ^ (((depth >> 2) & 3) << 2);
}

// LDS address of fragment `col` .. col + 15 of a bf16 across tile whose rows are
// W values: lane i of a group of 16 (group g = lane / 16) points at 4 values of
// depth 8g + i / 4; ds_read_b64_tr_b16 hands it the values of index i of the
// group's four depths.  Step s and half h (depths 8g + 4h ..) are offsets.
template <int W>
__device__ __forceinline__ uint32_t across_addr(const unsigned char* base, int col) {
    const int lane = threadIdx.x & 63, g = lane >> 4, i = lane & 15, depth = g * 8 + (i >> 2);
    const unsigned char* a = base + depth * (W * 2) + across_chunk<Bf16>(depth, (col >> 3) + ((i & 3) >> 1)) * 16 + (i & 1) * 8;
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) unsigned char*)a;
}

// Four bf16 fragments of K step `kStep` from their addresses: the same depths
// per lane as a fragment of an along tile (chunk kStep * 4 + lane / 16).  The
// reads and their wait are one block: with the builtin the compiler waits for
// every request in flight (vmcnt 0) before each of them.
template <int W, int kStep>
__device__ __forceinline__ void across_read4(const uint32_t (&a)[4], bf16x8 (&f)[4]) {
    typedef int int2_t __attribute__((ext_vector_type(2)));
    int2_t l[4], h[4];
    asm volatile(
        "ds_read_b64_tr_b16 %0, %8 offset:%12\n\t"
        "ds_read_b64_tr_b16 %4, %8 offset:%13\n\t"
        "ds_read_b64_tr_b16 %1, %9 offset:%12\n\t"
        "ds_read_b64_tr_b16 %5, %9 offset:%13\n\t"
        "ds_read_b64_tr_b16 %2, %10 offset:%12\n\t"
        "ds_read_b64_tr_b16 %6, %10 offset:%13\n\t"
        "ds_read_b64_tr_b16 %3, %11 offset:%12\n\t"
        "ds_read_b64_tr_b16 %7, %11 offset:%13\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(l[0]), "=&v"(l[1]), "=&v"(l[2]), "=&v"(l[3]), "=&v"(h[0]), "=&v"(h[1]), "=&v"(h[2]), "=&v"(h[3])
        : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "n"(kStep * 32 * W * 2), "n"(kStep * 32 * W * 2 + 4 * W * 2)
        : "memory");
#pragma unroll
    for (int j = 0; j < 4; ++j)
        f[j] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(l[j], h[j], 0, 1, 2, 3));
}

// One fp32 fragment of an across tile, at K step s: lane group g takes depths
// 16s + 4g + j, index lane % 16.
template <int W>
__device__ __forceinline__ floatx4 across_frag_f32(const unsigned char* base, int col, int s) {
    const int lane = threadIdx.x & 63, g = lane >> 4, c = col + (lane & 15);
    floatx4 v;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int depth = (s * 4 + g) * 4 + j;
        v[j] = *reinterpret_cast<const float*>(base + depth * (W * 4) + across_chunk<F32>(depth, c >> 2) * 16 + (c & 3) * 4);
    }
    return v;
}

// Raw buffer descriptor over `bytes` bytes.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc_bytes(const void* base, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), (short)0, (int)bytes, 0x00020000);
}

// v as C's type; a lane's 4 consecutive columns col .. col + 3 of C row `c`
// (16-byte aligned rows), of which those below `cols` exist in C and those
// below `clim` are not zero.
template <bool kBf16>
__device__ __forceinline__ void store_run(void* crow, int col, int cols, int clim, floatx4 v, int accumulate) {
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = col + k < clim ? v[k] : 0.f;
    if constexpr (kBf16) {
        bf16_t* o = reinterpret_cast<bf16_t*>(crow) + col;
        if (col + 3 < cols) {
            if (accumulate) {
                const uint2 w = *reinterpret_cast<const uint2*>(o);
                v[0] += __uint_as_float(w.x << 16), v[1] += __uint_as_float(w.x & 0xffff0000u);
                v[2] += __uint_as_float(w.y << 16), v[3] += __uint_as_float(w.y & 0xffff0000u);
            }
            *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (col + k < cols) o[k] = f32_to_bf16(accumulate ? v[k] + bf16_to_f32(o[k]) : v[k]);
        }
    } else {
        float* o = reinterpret_cast<float*>(crow) + col;
        if (col + 3 < cols) {
            if (accumulate) v += *reinterpret_cast<const floatx4*>(o);
            *reinterpret_cast<floatx4*>(o) = v;
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (col + k < cols) o[k] = accumulate ? v[k] + o[k] : v[k];
        }
    }
}

}  // namespace mfma

hipError_t launch_grouped_mid(const GroupedParams& p, GroupedForm form, GroupedElem elem, long long grid, hipStream_t s);
hipError_t launch_grouped_join(const GroupedParams& p, GroupedForm form, GroupedElem elem, hipStream_t s);
// rows [rows][cols] of x (or silu(x) * x2) as whole numbers up to 127 and a scale each
hipError_t launch_quantize_rows(const void* x, const void* x2, size_t ldx, int8_t* q, size_t ldq, float* scale, int rows, int cols,
                                bool bf16, hipStream_t s);

constexpr int kGroupTile = 128;  // rows and columns of a launch_grouped_mid tile

}  // namespace flexmoe
