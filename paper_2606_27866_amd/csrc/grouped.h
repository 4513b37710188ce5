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
    int slim;                 // 128 x 128 tiles: one LDS stage, four workgroups per compute unit
    int once;                 // weights of groups with one row tile carry the non-temporal hint
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
    int row_tiles;            // row tiles of the group (weight gradient: of C)
};

__device__ __forceinline__ int group_begin(const GroupedParams& p, int e) { return min(max(p.offsets[e], 0), p.R); }
__device__ __forceinline__ int group_width(const GroupedParams& p, int e, int full) {
    return p.keep ? min(max(p.keep[e], 0), full) : full;
}

// The group whose row tiles (of bm rows) hold number q, its rows, the number of
// its first row tile and how many it has; false past the last tile.  Lane l
// counts groups 4l .. 4l + 3.  Groups are taken in their order, or, where their
// widths set the length of the reduction, in four classes of width, the widest
// first, so that a launch ends on short tiles (60 groups of 1408 x 2048, 16384
// rows with widths, input gradient 94 -> 85 us; 8 of 4096 x 14336, forward: no
// difference).  All 64 lanes must be active and q uniform.
__device__ __forceinline__ bool find_group(const GroupedParams& p, int bm, int q, bool by_width, int full, int& e, int& row0,
                                           int& rows, int& first, int& tiles) {
    static_assert(kMaxExperts <= 4 * kWave, "four groups per lane");
    const int lane = threadIdx.x & 63;
    int b[5], t[4], cls[4] = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 5; ++j) b[j] = group_begin(p, min(4 * lane + j, p.E));
    if (by_width)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int w = group_width(p, min(4 * lane + j, p.E - 1), full);
            cls[j] = w >= full - full / 4 ? 0 : w >= full / 2 ? 1 : w >= full / 4 ? 2 : 3;
        }
#pragma unroll
    for (int j = 0; j < 4; ++j) t[j] = (max(b[j + 1] - b[j], 0) + bm - 1) / bm;
    int before = 0;  // tiles of the classes done
    for (int k = 0; k < (by_width ? 4 : 1); ++k) {
        int u[4], sum = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            u[j] = cls[j] == k ? t[j] : 0;
            sum += u[j];
        }
        const int incl = before + wave_incl_scan(sum);
        const unsigned long long owner = __ballot(incl - sum <= q && q < incl);
        if (!owner) {
            before = lane63(incl);
            continue;
        }
        int f = incl - sum, my = 0;
#pragma unroll
        for (int j = 0; j < 3; ++j)
            if (my == j && q >= f + u[j]) {
                f += u[j];
                my = j + 1;
            }
        const int lb = my == 0 ? b[0] : my == 1 ? b[1] : my == 2 ? b[2] : b[3];
        const int le = my == 0 ? b[1] : my == 1 ? b[2] : my == 2 ? b[3] : b[4];
        const int lt = my == 0 ? u[0] : my == 1 ? u[1] : my == 2 ? u[2] : u[3];
        const int src = __builtin_ctzll(owner);
        e = 4 * src + __builtin_amdgcn_readlane(my, src);
        row0 = __builtin_amdgcn_readlane(lb, src);
        rows = __builtin_amdgcn_readlane(le, src) - row0;
        first = __builtin_amdgcn_readlane(f, src);
        tiles = __builtin_amdgcn_readlane(lt, src);
        return true;
    }
    return false;
}

// Tile number L (row tiles of a group fastest, then column tiles, then parts
// of the reduction: neighbours share a weight tile).  A group's row tiles take
// equal shares of its rows, in steps of `unit`; kd is the depth of a K tile:
// parts of the reduction are whole K tiles.
template <int kForm>
__device__ __forceinline__ bool grouped_tile(const GroupedParams& p, int L, int bm, int bn, int unit, int kd, GroupedTile& t) {
    int mt, ct, depth;
    if constexpr (kForm == kWeightGrad) {
        const int per = p.tiles_r * p.tiles_c * p.splits;
        t.e = L / per;
        if (t.e >= p.E) return false;
        const int local = L - t.e * per;
        t.row_tiles = p.tiles_r;
        ct = local % p.tiles_c;
        mt = local / p.tiles_c % p.tiles_r;
        t.split = local / (p.tiles_r * p.tiles_c);
        t.row0 = group_begin(p, t.e);
        t.rows = max(group_begin(p, t.e + 1) - t.row0, 0);
        t.r0 = mt * bm;
        t.r1 = min(t.r0 + bm, p.N);
        depth = t.rows;
    } else {
        const int per = p.tiles_c * p.splits;
        int first, tiles;
        const bool by_width = p.keep_axis == (kForm == kForward ? 2 : 1);
        if (!find_group(p, bm, L / per, by_width, kForm == kForward ? p.K : p.N, t.e, t.row0, t.rows, first, tiles)) return false;
        t.row_tiles = tiles;
        const int local = L - first * per;
        mt = local % tiles;
        ct = local / tiles % p.tiles_c;
        t.split = local / (tiles * p.tiles_c);
        const int step = ceil_div(ceil_div(t.rows, tiles), unit) * unit;
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

// Two bf16 fragments at both K steps: f[2 * step + fragment].
template <int W>
__device__ __forceinline__ void across_read2x2(uint32_t a0, uint32_t a1, bf16x8 (&f)[4]) {
    typedef int int2_t __attribute__((ext_vector_type(2)));
    int2_t l[4], h[4];
    asm volatile(
        "ds_read_b64_tr_b16 %0, %8 offset:%10\n\t"
        "ds_read_b64_tr_b16 %4, %8 offset:%11\n\t"
        "ds_read_b64_tr_b16 %1, %9 offset:%10\n\t"
        "ds_read_b64_tr_b16 %5, %9 offset:%11\n\t"
        "ds_read_b64_tr_b16 %2, %8 offset:%12\n\t"
        "ds_read_b64_tr_b16 %6, %8 offset:%13\n\t"
        "ds_read_b64_tr_b16 %3, %9 offset:%12\n\t"
        "ds_read_b64_tr_b16 %7, %9 offset:%13\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(l[0]), "=&v"(l[1]), "=&v"(l[2]), "=&v"(l[3]), "=&v"(h[0]), "=&v"(h[1]), "=&v"(h[2]), "=&v"(h[3])
        : "v"(a0), "v"(a1), "n"(0), "n"(4 * W * 2), "n"(32 * W * 2), "n"(36 * W * 2)
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

// F fragments from own index `first` on, at K step s.
template <typename E, bool kAcross, int F>
__device__ __forceinline__ void read_step(const unsigned char* tile, int first, int s, typename E::Frag (&f)[F]) {
    const int lane = threadIdx.x & 63;
    if constexpr (kAcross && E::kBytes == 2) {
        uint32_t addr[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) addr[i] = across_addr<128>(tile, first + i * 16) + s * (32 * 256);
        across_read4<128, 0>(addr, f);
    } else {
#pragma unroll
        for (int i = 0; i < F; ++i) {
            if constexpr (kAcross) f[i] = across_frag_f32<128>(tile, first + i * 16, s);
            else f[i] = __builtin_bit_cast(typename E::Frag, lds_frag(tile, first + i * 16 + (lane & 15), s * 4 + (lane >> 4)));
        }
    }
}

// F fragments from own index `first` on, at both K steps.
template <typename E, bool kAcross, int F>
__device__ __forceinline__ void read_frags(const unsigned char* tile, int first, typename E::Frag (&f)[2][F]) {
    const int lane = threadIdx.x & 63;
    if constexpr (kAcross && E::kBytes == 2) {
        static_assert(F == 4, "read four at a time (two: read_pair)");
        uint32_t addr[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) addr[i] = across_addr<128>(tile, first + i * 16);
        across_read4<128, 0>(addr, f[0]);
        across_read4<128, 1>(addr, f[1]);
    } else {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int i = 0; i < F; ++i) {
                if constexpr (kAcross) f[s][i] = across_frag_f32<128>(tile, first + i * 16, s);
                else f[s][i] = __builtin_bit_cast(typename E::Frag, lds_frag(tile, first + i * 16 + (lane & 15), s * 4 + (lane >> 4)));
            }
    }
}

// Two fragments from own index `first` on, at both K steps.
template <typename E, bool kAcross>
__device__ __forceinline__ void read_pair(const unsigned char* tile, int first, typename E::Frag (&f)[2][2]) {
    if constexpr (kAcross && E::kBytes == 2) {
        bf16x8 v[4];
        across_read2x2<128>(across_addr<128>(tile, first), across_addr<128>(tile, first + 16), v);
        f[0][0] = v[0], f[0][1] = v[1], f[1][0] = v[2], f[1][1] = v[3];
    } else {
        read_frags<E, kAcross, 2>(tile, first, f);
    }
}

// Raw buffer descriptor over `bytes` bytes.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc_bytes(const void* base, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), (short)0, (int)bytes, 0x00020000);
}

constexpr int STAGE = 16384;  // bytes of 128 rows' K tile

// Requests of N instructions of 1 KB for 128 own indices of an operand:
// instruction i fills the tile's LDS bytes (wave0 + i) * 1024 + lane * 16.
// kOnce: nothing else reads these bytes (non-temporal).
template <typename E, bool kAcross, int N, bool kOnce = false>
struct Loader {
    static __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t rsrc, uint32_t voff, uint32_t soff, unsigned char* lds) {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_ptr_t*)lds, 16, voff, soff, 0, kOnce ? 2 : 0);
    }
    const char* base;       // first element of the operand's part
    size_t step;            // bytes a K tile advances (across: 0 in the lane offsets)
    uint32_t off[N];        // lane offset, kOOB if its row or column does not exist
    int col[N];             // along: the chunk's first depth inside a K tile
    size_t ldb;             // across: bytes per depth
    uint32_t tail;          // across: bytes of the last depth that may be read
    __amdgpu_buffer_rsrc_t r;
    int depth;

    // `own`: rows (along) or columns (across) that exist from the tile's first
    // on; `wave0`: this wave's first instruction
    __device__ __forceinline__ void init(const void* p, size_t ld, int own, int d, int wave0) {
        const int lane = threadIdx.x & 63;
        base = reinterpret_cast<const char*>(p);
        depth = d;
        if constexpr (!kAcross) {
            r = make_rsrc_bytes(base, 0x7ffffff0u);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int row = (wave0 + i) * 8 + lane / CHUNKS, c = swz(row, lane % CHUNKS);
                col[i] = c * E::kPer;
                off[i] = row < own ? (uint32_t)((size_t)row * ld * E::kBytes) + c * 16 : kOOB;
            }
        } else {
            constexpr int kChunks = 128 * E::kBytes / 16;  // of an LDS row
            ldb = ld * E::kBytes;
            step = ldb * E::kDepth;
            tail = (uint32_t)((min(own, 128) * E::kBytes + 15) & ~15);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int dep = (wave0 + i) * (64 / kChunks) + lane / kChunks;
                const int c = across_chunk<E>(dep, lane % kChunks);
                col[i] = 0;
                off[i] = c * E::kPer < own ? (uint32_t)(dep * ldb) + c * 16 : kOOB;
            }
        }
    }
    // K tile kt to `lds` (this wave's first instruction's place); past the end zeros
    __device__ __forceinline__ void request(int kt, unsigned char* lds) {
        const int lim = depth - kt * E::kDepth;
        if constexpr (!kAcross) {
#pragma unroll
            for (int i = 0; i < N; ++i) load(r, col[i] < lim ? off[i] : kOOB, (uint32_t)kt * ROWB, lds + i * 1024);
        } else {
            // the descriptor covers the depths that exist
            const int n = max(min(lim, E::kDepth), 0);
            r = make_rsrc_bytes(base + (size_t)kt * step, max((n - 1) * (int)ldb + (int)tail, 0) & -(int)(n > 0));
#pragma unroll
            for (int i = 0; i < N; ++i) load(r, off[i], 0, lds + i * 1024);
        }
    }
};

// A lane's 4 consecutive columns col .. col + 3 of C row `crow` (16-byte
// aligned rows), of which those below `cols` exist: what is there, and v as C's
// type.
template <bool kBf16>
__device__ __forceinline__ floatx4 load_run(const void* crow, int col, int cols) {
    floatx4 v{0.f, 0.f, 0.f, 0.f};
    if constexpr (kBf16) {
        const bf16_t* o = reinterpret_cast<const bf16_t*>(crow) + col;
        if (col + 3 < cols) {
            const uint2 w = *reinterpret_cast<const uint2*>(o);
            v = floatx4{__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16),
                        __uint_as_float(w.y & 0xffff0000u)};
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (col + k < cols) v[k] = bf16_to_f32(o[k]);
        }
    } else {
        const float* o = reinterpret_cast<const float*>(crow) + col;
        if (col + 3 < cols) {
            v = *reinterpret_cast<const floatx4*>(o);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (col + k < cols) v[k] = o[k];
        }
    }
    return v;
}
template <bool kBf16>
__device__ __forceinline__ void store_run(void* crow, int col, int cols, floatx4 v) {
    if constexpr (kBf16) {
        bf16_t* o = reinterpret_cast<bf16_t*>(crow) + col;
        if (col + 3 < cols) {
            *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (col + k < cols) o[k] = f32_to_bf16(v[k]);
        }
    } else {
        float* o = reinterpret_cast<float*>(crow) + col;
        if (col + 3 < cols) {
            *reinterpret_cast<floatx4*>(o) = v;
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (col + k < cols) o[k] = v[k];
        }
    }
}

// First elements of a tile's operands, and how many of their own indices exist
// from there on.
template <typename E, int kForm>
struct Operands {
    const typename E::T *a, *b;
    int own_a, own_b;
    __device__ __forceinline__ Operands(const GroupedParams& p, const GroupedTile& t)
        : a(reinterpret_cast<const typename E::T*>(p.a)), b(reinterpret_cast<const typename E::T*>(p.b)), own_a(t.r1 - t.r0) {
        if constexpr (kForm == kWeightGrad) {
            a += (size_t)(t.row0 + t.d0) * p.lda + t.r0;
            b += (size_t)(t.row0 + t.d0) * p.ldb + t.c0;
        } else {
            a += (size_t)(t.row0 + t.r0) * p.lda + t.d0;
            b += (size_t)t.e * p.N * p.ldb;
            b += kForm == kForward ? (size_t)t.c0 * p.ldb + t.d0 : (size_t)t.d0 * p.ldb + t.c0;
        }
        own_b = (kForm == kForward ? p.N : p.K) - t.c0;
    }
};

// C's part of a tile that a wave holds, where C is bf16 and the accumulators hold
// all of it: rounded before it goes through LDS (2 KB of the wave's own), so that a store
// takes 8 columns of a lane and 16-byte accesses cover 8 rows of 64 columns.
// Arguments as below; runs 2q and 2q + 1 are neighbours.
template <typename E, int kForm, int kRows, int kCols, typename Column, typename Value>
__device__ __forceinline__ void store_tile_bf16(const GroupedParams& p, const GroupedTile& t, int first, unsigned char* scratch,
                                                Column&& column, Value&& value) {
    constexpr int kChunks = 2 * kCols, kSteps = kCols / 2;  // 16-byte chunks of a row; stores per fragment
    const int lane = threadIdx.x & 63, lr = lane & 15, lc = lane >> 4;
    const int cols = kForm == kForward ? p.N : p.K;
    auto crow_of = [&](int r) { return kForm == kWeightGrad ? (size_t)t.e * p.N + r : (size_t)t.row0 + r; };
    // int8: the scales of this lane's columns and rows, before any store: the
    // compiler keeps a read behind the stores before it
    float sb[kCols][4], sa[kRows];
    if constexpr (E::kBytes == 1) {
#pragma unroll
        for (int j = 0; j < kCols; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int c = column(4 * j + lc) + k;
                sb[j][k] = c < cols ? p.sb[(size_t)t.e * p.N + c] : 0.f;
            }
#pragma unroll
        for (int i = 0; i < kRows; ++i) sa[i] = p.sa[crow_of(min(first + i * 16 + lr, t.r1 - 1))];
    }
    const int chunk = lane % kChunks, c8 = column(2 * chunk);
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const int clim = first + i * 16 + lr < t.rlim ? t.clim : 0;
#pragma unroll
        for (int j = 0; j < kCols; ++j) {
            const int c = column(4 * j + lc);
            const typename E::Acc v = value(i, j);
            float f[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if constexpr (E::kBytes == 1) f[k] = (float)v[k] * (sa[i] * sb[j][k]);
                else f[k] = v[k];
                f[k] = c + k < clim ? f[k] : 0.f;
            }
            const int at = ((2 * j + (lc >> 1)) ^ (lr % kChunks)) * 16 + (lc & 1) * 8;
            *reinterpret_cast<uint2*>(scratch + lr * (kChunks * 16) + at) = make_uint2(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]));
        }
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int row = s * (64 / kChunks) + lane / kChunks, r = first + i * 16 + row;
            const u32x4 v = *reinterpret_cast<const u32x4*>(scratch + row * (kChunks * 16) + (chunk ^ (row % kChunks)) * 16);
            // what lies past a width is left as it is when C is added to
            const int end = kForm == kWeightGrad && p.accumulate ? (r < t.rlim ? min(t.clim, cols) : 0) : cols;
            if (r >= t.r1 || c8 >= end) continue;
            bf16_t* o = reinterpret_cast<bf16_t*>(p.c) + crow_of(r) * p.ldc + c8;
            if (c8 + 7 < end) {
                *reinterpret_cast<u32x4*>(o) = v;
            } else {
#pragma unroll
                for (int k = 0; k < 7; ++k)
                    if (c8 + k < end) o[k] = (bf16_t)(v[k >> 1] >> (16 * (k & 1)));
            }
        }
    }
}

// C's part of a tile that a wave holds: kRows fragments of 16 rows from C row
// `first` on and 4 * kCols runs (kCols 2 or 4) of 4 columns, run q at column(q),
// to C or to this part's place among the partial sums.  value(i, j) is the
// accumulator of row fragment i and runs 4j .. 4j + 3 (lane -> row lane % 16, run
// 4j + lane / 16).
// Each row fragment goes through 4 KB of LDS that are the wave's own, so that a
// store covers 4 rows of 16 (8 of 8) consecutive runs, whole cache lines, where straight
// from the accumulators it covers 16 rows of 4 runs (stores alone of 692 MB of
// fp32 with four 128 x 128 tiles per compute unit: 190 -> 123 us).
// kWhole: the accumulators hold all of C (no parts, and what it is added to is in
// them already).
template <typename E, int kForm, bool kBf16Out, int kRows, int kCols, bool kWhole, typename Column, typename Value>
__device__ __forceinline__ void store_tile(const GroupedParams& p, const GroupedTile& t, int first, unsigned char* scratch,
                                           Column&& column, Value&& value) {
    if constexpr (kBf16Out && kWhole) {
        store_tile_bf16<E, kForm, kRows, kCols>(p, t, first, scratch, column, value);
        return;
    } else {
        if constexpr (kBf16Out)
            if (p.splits == 1 && (kForm != kWeightGrad || !p.accumulate)) {
                store_tile_bf16<E, kForm, kRows, kCols>(p, t, first, scratch, column, value);
                return;
            }
        const int lane = threadIdx.x & 63, lr = lane & 15, lc = lane >> 4;
        const int cols = kForm == kForward ? p.N : p.K;
        const bool add = kForm == kWeightGrad && !kWhole && p.accumulate && p.splits == 1;
        constexpr int kRuns = 4 * kCols, kSteps = kCols;  // runs of a row; stores per fragment
        const int run = lane % kRuns, sub = lane / kRuns;  // a store's run and row (of 64 / kRuns) for this lane
        auto row_of = [&](int s) { return s * (64 / kRuns) + sub; };
        const int c = column(run);
        auto crow_of = [&](int r) { return kForm == kWeightGrad ? (size_t)t.e * p.N + r : (size_t)t.row0 + r; };
        auto address = [&](int r) { return reinterpret_cast<char*>(p.c) + crow_of(r) * p.ldc * (kBf16Out ? 2 : 4); };
        // old values are read a fragment ahead: the compiler keeps a read behind
        // the stores before it
        floatx4 old[kForm == kWeightGrad ? 2 : 1][kSteps];
        auto load_old = [&](int i) {
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                const int r = first + i * 16 + row_of(s);
                if (r < t.r1 && c < cols) old[i & 1][s] = load_run<kBf16Out>(address(r), c, cols);
            }
        };
        if constexpr (kForm == kWeightGrad)
            if (add) load_old(0);
        // int8: this lane's columns' and rows' scales, read before any store for
        // the same reason
        float sb[4], sa[kRows][kSteps];
        if constexpr (E::kBytes == 1)
            if (p.splits == 1) {
#pragma unroll
                for (int k = 0; k < 4; ++k) sb[k] = c + k < cols ? p.sb[(size_t)t.e * p.N + c + k] : 0.f;
#pragma unroll
                for (int i = 0; i < kRows; ++i)
#pragma unroll
                    for (int s = 0; s < kSteps; ++s) sa[i][s] = p.sa[crow_of(min(first + i * 16 + row_of(s), t.r1 - 1))];
            }
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            if constexpr (kForm == kWeightGrad)
                if (add && i + 1 < kRows) load_old(i + 1);
#pragma unroll
            for (int j = 0; j < kCols; ++j)
                *reinterpret_cast<typename E::Acc*>(scratch + lr * (kRuns * 16) + ((4 * j + lc) ^ (lr % kRuns)) * 16) = value(i, j);
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                const int row = row_of(s), r = first + i * 16 + row;
                typename E::Acc v = *reinterpret_cast<const typename E::Acc*>(scratch + row * (kRuns * 16) + (run ^ (row % kRuns)) * 16);
                const int clim = r < t.rlim ? t.clim : 0;
                // what lies past a width is left as it is when C is added to
                const int end = kForm == kWeightGrad && p.accumulate && p.splits == 1 ? min(clim, cols) : cols;
                if (r >= t.r1 || c >= end) continue;
                const size_t crow = crow_of(r);
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = c + k < clim ? v[k] : 0;
                if (!kWhole && p.splits > 1) {
                    const size_t rows = kForm == kWeightGrad ? (size_t)p.E * p.N : (size_t)p.R;
                    const size_t ldp = (cols + 3) & ~3;
                    *reinterpret_cast<typename E::Acc*>(reinterpret_cast<char*>(p.partial) + ((t.split * rows + crow) * ldp + c) * 4) = v;
                    continue;
                }
                floatx4 f;
                if constexpr (E::kBytes == 1) {
                    // past the width the factor may be anything: not multiplied
#pragma unroll
                    for (int k = 0; k < 4; ++k) f[k] = c + k < clim ? (float)v[k] * (sa[i][s] * sb[k]) : 0.f;
                } else {
                    f = v;
                }
                if constexpr (kForm == kWeightGrad)
                    if (add) f += old[i & 1][s];
                store_run<kBf16Out>(address(r), c, end, f);
            }
        }
    }
}

}  // namespace mfma

// 128 x 128 tiles: every form and type
hipError_t launch_grouped_mid(const GroupedParams& p, GroupedForm form, GroupedElem elem, long long grid, hipStream_t s);
// 32 x 128 tiles: x W^T and dy W with few rows, every type
hipError_t launch_grouped_few(const GroupedParams& p, GroupedForm form, GroupedElem elem, long long grid, hipStream_t s);
// 256 x 256 tiles: bf16 (every form) and int8
hipError_t launch_grouped_big(const GroupedParams& p, GroupedForm form, GroupedElem elem, long long grid, hipStream_t s);
hipError_t launch_grouped_join(const GroupedParams& p, GroupedForm form, GroupedElem elem, hipStream_t s);
// rows [rows][cols] of x (or silu(x) * x2) as whole numbers up to 127 and a scale each
hipError_t launch_quantize_rows(const void* x, const void* x2, size_t ldx, int8_t* q, size_t ldq, float* scale, int rows, int cols,
                                bool bf16, hipStream_t s);

constexpr int kGroupTile = 128;     // rows and columns of a launch_grouped_mid tile
constexpr int kGroupBigTile = 256;  // of a launch_grouped_big tile
constexpr int kGroupFewRows = 32;   // rows of a launch_grouped_few tile (128 columns)

}  // namespace flexmoe
