// Grouped products on 128 x 128 tiles (gfx950): every form and element type.
//
// A workgroup of 4 waves (2 x 2, each up to 64 x 64 of C as 16 x 16 MFMA
// accumulators) multiplies K tiles of 128 bytes depth.  Operands go from
// memory to LDS by buffer_load ... lds, 16 KB per operand and K tile, A one K
// tile ahead in two stages and B two ahead in three: 80 KB, so that two
// workgroups share a compute unit and one's MFMAs cover the other's waits.  An
// operand that is contiguous in the reduction is laid out as 128 rows of 128
// bytes, one that is not as K-tile rows of 128 values, which the fragment
// reads transpose (across_frag).
//
// Between the other two kinds of tiles: 60 groups of 1408 x 2048, bf16 x W^T, at
// 4096 rows 84 us (256 x 256 tiles: 100), at 16384 148 (147).  A small form with
// one stage (40 KB, four workgroups) takes short weight gradients.
//
// What lies outside a group, a width or a matrix reads as zeros: whole rows
// and 16-byte chunks by offsets past the descriptor, the elements of a chunk
// that straddles the end of the reduction by clearing both fragments, C's
// rows and columns past the width at the store.
#include <algorithm>

#include "grouped.h"

namespace flexmoe {

namespace {
using namespace mfma;

constexpr int GT = 256;                   // threads
constexpr int SMEM = 5 * STAGE;           // A0 A1 B0 B1 B2
constexpr int NI = STAGE / 1024 / 4;      // requests per wave and operand: 4
constexpr int SCRATCH = 2048;             // a wave's, beside the stages of the small weight gradient

// The accumulators of a wave's 64 x 64 of C from what is there, for columns and
// rows within the widths.  bf16: read as store_tile_bf16 writes (16 bytes of 8
// rows), through LDS.  `meanwhile` runs after the reads are under way.
template <typename E, bool kBf16Out, typename F>
__device__ __forceinline__ void old_tile(const GroupedParams& p, const GroupedTile& t, int wm, int wn, unsigned char* scratch,
                                         typename E::Acc (&acc)[4][4], F&& meanwhile) {
    const int lane = threadIdx.x & 63, lr = lane & 15, lc = lane >> 4;
    const int rend = min(t.r1, t.rlim), cend = min(t.clim, p.K);
    if constexpr (kBf16Out) {
        const int chunk = lane & 7, c = t.c0 + wn * 64 + chunk * 8;
        u32x4 raw[4][2];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int r = t.r0 + wm * 64 + i * 16 + s * 8 + (lane >> 3);
                const bf16_t* o = reinterpret_cast<const bf16_t*>(p.c) + ((size_t)t.e * p.N + r) * p.ldc + c;
                raw[i][s] = u32x4{0, 0, 0, 0};
                if (r >= rend || c >= cend) continue;
                if (c + 7 < cend) {
                    raw[i][s] = *reinterpret_cast<const u32x4*>(o);
                } else {
#pragma unroll
                    for (int k = 0; k < 7; ++k)
                        if (c + k < cend) raw[i][s][k >> 1] |= (uint32_t)o[k] << (16 * (k & 1));
                }
            }
        meanwhile();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int row = s * 8 + (lane >> 3);
                *reinterpret_cast<u32x4*>(scratch + row * 128 + (chunk ^ (row & 7)) * 16) = raw[i][s];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint2 w = *reinterpret_cast<const uint2*>(scratch + lr * 128 + ((2 * j + (lc >> 1)) ^ (lr & 7)) * 16 + (lc & 1) * 8);
                acc[j][i] = typename E::Acc{__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16),
                                            __uint_as_float(w.y & 0xffff0000u)};
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = t.r0 + wm * 64 + i * 16 + lr, c = t.c0 + wn * 64 + j * 16 + lc * 4;
                if (r < rend && c < cend)
                    acc[j][i] = load_run<false>(reinterpret_cast<const float*>(p.c) + ((size_t)t.e * p.N + r) * p.ldc, c, cend);
            }
        meanwhile();
    }
}

template <typename E, int kForm, bool kBf16Out, bool kSlim>
__global__ __launch_bounds__(GT, kSlim ? 4 : 2) void grouped_mid_kernel(GroupedParams p) {
    constexpr bool kAcrossA = kForm == kWeightGrad, kAcrossB = kForm != kForward;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[kSlim ? 2 * STAGE + 4 * SCRATCH : SMEM];
    GroupedTile t;
    if (!grouped_tile<kForm>(p, xcd_tile(8), kGroupTile, kGroupTile, 16, E::kDepth, t)) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int wm = wave >> 1, wn = wave & 1, lc = lane >> 4;
    const int nr = t.r1 - t.r0, depth = t.d1 - t.d0;
    const Operands<E, kForm> op(p, t);
    const int nk = ceil_div(depth, E::kDepth);

    auto run = [&](auto mf_c, auto once_c) {
        constexpr int MF = decltype(mf_c)::value;
        constexpr bool kOnce = decltype(once_c)::value;
        constexpr int NA = kAcrossA ? NI : MF;  // along: 32 * MF rows of A
        Loader<E, kAcrossA, NA> la;
        Loader<E, kAcrossB, NI, kOnce> lb;
        la.init(op.a, p.lda, op.own_a, depth, wave * NA);
        lb.init(op.b, p.ldb, op.own_b, depth, wave * NI);
        unsigned char* const sa = smem;
        unsigned char* const sb = smem + 2 * STAGE;
        auto request_a = [&](int kt, int stage) { la.request(kt, sa + stage * STAGE + wave * (NA * 1024)); };
        auto request_b = [&](int kt, int stage) { lb.request(kt, sb + stage * STAGE + wave * (NI * 1024)); };
        typename E::Acc acc[4][MF];
        // fp32: sums of 256 products are added to a second set, so that an
        // error grows with the number of those sums, not of products
        constexpr bool kTwoLevels = E::kBytes == 4 && !kSlim;
        constexpr int kFlush = 8;
        typename E::Acc total[kTwoLevels ? 4 : 1][kTwoLevels ? MF : 1];
        if constexpr (kTwoLevels)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < MF; ++i) total[j][i] = typename E::Acc{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < MF; ++i) acc[j][i] = typename E::Acc{0, 0, 0, 0};
        if constexpr (kSlim) {
            // one stage: four workgroups share a compute unit and cover each
            // other's waits
            unsigned char* const sb1 = smem + STAGE;
            auto request = [&](int kt) {
                la.request(kt, smem + wave * (NA * 1024));
                lb.request(kt, sb1 + wave * (NI * 1024));
            };
            // what C is added to starts the accumulators, read beside the first
            // K tile
            if (p.accumulate) old_tile<E, kBf16Out>(p, t, wm, wn, smem + 2 * STAGE + wave * SCRATCH, acc, [&] { request(0); });
            else request(0);
            for (int kt = 0; kt < nk; ++kt) {
                if (kt > 0) request(kt);
                __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
                barrier_no_fence();
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    typename E::Frag fa[MF], fb[4];
                    read_step<E, kAcrossB, 4>(sb1, wn * 64, s, fb);
                    read_step<E, kAcrossA, MF>(smem, wm * 16 * MF, s, fa);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int i = 0; i < MF; ++i) acc[j][i] = E::mma(fb[j], fa[i], acc[j][i]);
                }
                __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
                if (kt + 1 < nk) barrier_no_fence();
            }
        } else {
            request_a(0, 0);
            request_b(0, 0);
            request_b(1, 1);
            int st_b = 0;
            for (int kt = 0; kt < nk; ++kt) {
                // tile kt is in when only B of tile kt + 1 is outstanding; this
                // wave's LDS reads of tile kt - 1 are done, so that its stages may
                // be refilled after the barrier
                __builtin_amdgcn_s_waitcnt(waitcnt_vm(NI) & kWaitLgkm0);
                barrier_no_fence();
                request_a(kt + 1, (kt + 1) & 1);
                request_b(kt + 2, st_b == 0 ? 2 : st_b - 1);
                const unsigned char* at = sa + (kt & 1) * STAGE;
                const unsigned char* bt = sb + st_b * STAGE;
                st_b = st_b == 2 ? 0 : st_b + 1;
                if constexpr (kTwoLevels) {
                    // one K step at a time: the fragments of both would not fit
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        typename E::Frag fa[MF], fb[4];
                        read_step<E, kAcrossB, 4>(bt, wn * 64, s, fb);
                        read_step<E, kAcrossA, MF>(at, wm * 16 * MF, s, fa);
                        if constexpr (!kAcrossA)
                            if (kt == nk - 1 && depth % E::kPer) {
                                const int valid = depth - kt * E::kDepth - (s * 4 + lc) * E::kPer;
#pragma unroll
                                for (int i = 0; i < MF; ++i) fa[i] = head<E>(fa[i], valid);
                                if constexpr (!kAcrossB)
#pragma unroll
                                    for (int j = 0; j < 4; ++j) fb[j] = head<E>(fb[j], valid);
                            }
#pragma unroll
                        for (int j = 0; j < 4; ++j)
#pragma unroll
                            for (int i = 0; i < MF; ++i) acc[j][i] = E::mma(fb[j], fa[i], acc[j][i]);
                    }
                    if (kt % kFlush == kFlush - 1)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
#pragma unroll
                            for (int i = 0; i < MF; ++i) {
                                total[j][i] += acc[j][i];
                                acc[j][i] = typename E::Acc{0, 0, 0, 0};
                            }
                    continue;
                } else {
                    typename E::Frag fa[2][MF], fb[2][4];
                    read_frags<E, kAcrossB, 4>(bt, wn * 64, fb);
                    read_frags<E, kAcrossA, MF>(at, wm * 16 * MF, fa);
                    if constexpr (!kAcrossA)
                        if (kt == nk - 1 && depth % E::kPer) {
#pragma unroll
                            for (int s = 0; s < 2; ++s) {
                                const int valid = depth - kt * E::kDepth - (s * 4 + lc) * E::kPer;
#pragma unroll
                                for (int i = 0; i < MF; ++i) fa[s][i] = head<E>(fa[s][i], valid);
                                if constexpr (!kAcrossB)
#pragma unroll
                                    for (int j = 0; j < 4; ++j) fb[s][j] = head<E>(fb[s][j], valid);
                            }
                        }
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int s = 0; s < 2; ++s)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
#pragma unroll
                            for (int i = 0; i < MF; ++i) acc[j][i] = E::mma(fb[s][j], fa[s][i], acc[j][i]);
                }
            }
        }
        __builtin_amdgcn_s_waitcnt(waitcnt_vm(0) & kWaitLgkm0);  // no request may outlive the loop

        if constexpr (kTwoLevels)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < MF; ++i) acc[j][i] += total[j][i];
        barrier_no_fence();  // every wave has read its fragments: LDS becomes the stores' scratch
        store_tile<E, kForm, kBf16Out, MF, 4, kSlim>(
            p, t, t.r0 + wm * 16 * MF, smem + wave * 4096, [&](int q) { return t.c0 + wn * 64 + q * 4; },
            [&](int i, int j) { return acc[j][i]; });
    };
    auto by_rows = [&](auto once_c) {
        if (nr > 96) run(std::integral_constant<int, 4>{}, once_c);
        else if (nr > 64) run(std::integral_constant<int, 3>{}, once_c);
        else if (nr > 32) run(std::integral_constant<int, 2>{}, once_c);
        else run(std::integral_constant<int, 1>{}, once_c);
    };
    // a group with one row tile reads its weights once
    if constexpr (kAcrossA) run(std::integral_constant<int, 4>{}, std::false_type{});
    else if (p.once && t.row_tiles == 1) by_rows(std::true_type{});
    else by_rows(std::false_type{});
}

// The parts of a split reduction added in their order: one thread per run of 4
// columns of C.
template <bool kI8, bool kBf16Out, bool kRowGroups>
__global__ __launch_bounds__(256) void grouped_join_kernel(GroupedParams p, int cols, size_t rows) {
    const size_t runs = (cols + 3) / 4, ldp = runs * 4;
    const int first = kRowGroups ? group_begin(p, 0) : 0, end = kRowGroups ? group_begin(p, p.E) : 0;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < rows * runs; i += (size_t)gridDim.x * 256) {
        const size_t r = i / runs;
        const int c = (int)(i - r * runs) * 4;
        if (kRowGroups && ((int)r < first || (int)r >= end)) continue;
        int stop = cols;
        if (!kRowGroups && p.accumulate && p.keep) {
            // what lies past a width is left as it is, to the sign of a zero
            const int e = (int)(r / p.N), w = group_width(p, e, p.keep_axis == 1 ? p.N : p.K);
            if (p.keep_axis == 1 && (int)(r - (size_t)e * p.N) >= w) continue;
            if (p.keep_axis == 2) stop = min(cols, w);
            if (c >= stop) continue;
        }
        const char* src = reinterpret_cast<const char*>(p.partial) + (r * ldp + c) * 4;
        floatx4 v{0.f, 0.f, 0.f, 0.f};
        if constexpr (kI8) {
            mfma::intx4 s{0, 0, 0, 0};
            for (int k = 0; k < p.splits; ++k) s += *reinterpret_cast<const mfma::intx4*>(src + (size_t)k * rows * ldp * 4);
            int e = 0;  // the group of row r
            for (int lo = 0, hi = p.E; lo < hi;) {
                const int m = (lo + hi) / 2;
                if (group_begin(p, m + 1) <= (int)r) lo = m + 1;
                else hi = m;
                e = lo;
            }
            e = min(e, p.E - 1);
            const float sr = p.sa[r];
            const int clim = p.keep_axis == 1 ? group_width(p, e, p.N) : p.N;
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = c + k < clim ? (float)s[k] * (sr * p.sb[(size_t)e * p.N + c + k]) : 0.f;
        } else {
            for (int k = 0; k < p.splits; ++k) v += *reinterpret_cast<const floatx4*>(src + (size_t)k * rows * ldp * 4);
        }
        char* const crow = reinterpret_cast<char*>(p.c) + r * p.ldc * (kBf16Out ? 2 : 4);
        if (!kRowGroups && p.accumulate) v += load_run<kBf16Out>(crow, c, stop);
        store_run<kBf16Out>(crow, c, stop, v);
    }
}

template <typename E, int kForm>
void launch_mid(const GroupedParams& p, unsigned grid, hipStream_t s) {
    if constexpr (kForm == kWeightGrad)
        if (p.slim) {
            if (p.out_bf16) grouped_mid_kernel<E, kForm, true, true><<<grid, GT, 0, s>>>(p);
            else grouped_mid_kernel<E, kForm, false, true><<<grid, GT, 0, s>>>(p);
            return;
        }
    if (p.out_bf16) grouped_mid_kernel<E, kForm, true, false><<<grid, GT, 0, s>>>(p);
    else grouped_mid_kernel<E, kForm, false, false><<<grid, GT, 0, s>>>(p);
}

}  // namespace

hipError_t launch_grouped_mid(const GroupedParams& p, GroupedForm form, GroupedElem elem, long long tiles, hipStream_t s) {
    if (tiles <= 0) return hipSuccess;
    const unsigned grid = (unsigned)((tiles + 63) / 64 * 64);
    if (elem == kElemI8) launch_mid<I8, kForward>(p, grid, s);
    else if (elem == kElemBf16 && form == kForward) launch_mid<Bf16, kForward>(p, grid, s);
    else if (elem == kElemBf16 && form == kInputGrad) launch_mid<Bf16, kInputGrad>(p, grid, s);
    else if (elem == kElemBf16) launch_mid<Bf16, kWeightGrad>(p, grid, s);
    else if (form == kForward) launch_mid<F32, kForward>(p, grid, s);
    else if (form == kInputGrad) launch_mid<F32, kInputGrad>(p, grid, s);
    else launch_mid<F32, kWeightGrad>(p, grid, s);
    return hipGetLastError();
}

hipError_t launch_grouped_join(const GroupedParams& p, GroupedForm form, GroupedElem elem, hipStream_t s) {
    const int cols = form == kForward ? p.N : p.K;
    const size_t rows = form == kWeightGrad ? (size_t)p.E * p.N : (size_t)p.R;
    const size_t runs = rows * ((cols + 3) / 4);
    if (!runs) return hipSuccess;
    const unsigned grid = (unsigned)std::min<size_t>((runs + 255) / 256, 4096);
    if (elem == kElemI8) {
        if (p.out_bf16) grouped_join_kernel<true, true, true><<<grid, 256, 0, s>>>(p, cols, rows);
        else grouped_join_kernel<true, false, true><<<grid, 256, 0, s>>>(p, cols, rows);
    } else if (form == kWeightGrad) {
        if (p.out_bf16) grouped_join_kernel<false, true, false><<<grid, 256, 0, s>>>(p, cols, rows);
        else grouped_join_kernel<false, false, false><<<grid, 256, 0, s>>>(p, cols, rows);
    } else {
        if (p.out_bf16) grouped_join_kernel<false, true, true><<<grid, 256, 0, s>>>(p, cols, rows);
        else grouped_join_kernel<false, false, true><<<grid, 256, 0, s>>>(p, cols, rows);
    }
    return hipGetLastError();
}

}  // namespace flexmoe
