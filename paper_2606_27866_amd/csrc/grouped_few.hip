// Grouped products of few rows (gfx950): x W^T and dy W on tiles of 32 rows and
// 128 columns, every element type.
//
// Bound by the weights, which stream from memory once.  A workgroup of 4 waves,
// wave w owning columns 32w .. 32w + 31 and up to 32 rows (16 or 32 by the
// tile's rows), keeps one K tile of 128 bytes depth in LDS and one on its way:
// 40 KB, so that four workgroups share a compute unit (two of the 128 x 128
// tiles).  What is in flight is the same, the rounds of tiles are half as long: 60
// groups of 1408 x 2048, 1024 rows, int8 with the rounding 44.4 us on 128 x 128
// tiles, 36.0 on these, bf16 89 and 62; 8 of 512 x 256, 128 rows, fp32 12.6 and 9.1;
// but 64 of 2560 x 3584, 192 rows, bf16, widths on rows 108 and 116.
#include "grouped.h"

namespace flexmoe {

namespace {
using namespace mfma;

constexpr int FT = 256;
constexpr int A_STAGE = kGroupFewRows * ROWB;            // 4 KB
constexpr int FEW_SMEM = 2 * (STAGE + A_STAGE);
constexpr int NB = STAGE / 1024 / 4;                     // requests per wave: 4 of B, 1 of A

template <typename E, int kForm, bool kBf16Out>
__global__ __launch_bounds__(FT, 4) void grouped_few_kernel(GroupedParams p) {
    constexpr bool kAcrossB = kForm != kForward;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[FEW_SMEM];
    GroupedTile t;
    if (!grouped_tile<kForm>(p, xcd_tile(8), kGroupFewRows, kGroupTile, 16, E::kDepth, t)) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lc = (threadIdx.x & 63) >> 4;
    const int nr = t.r1 - t.r0, depth = t.d1 - t.d0;
    const Operands<E, kForm> op(p, t);
    const int nk = ceil_div(depth, E::kDepth);

    auto run = [&](auto mr_c, auto once_c) {
        constexpr int MR = decltype(mr_c)::value;
        Loader<E, false, 1> la;
        Loader<E, kAcrossB, NB, decltype(once_c)::value> lb;
        la.init(op.a, p.lda, op.own_a, depth, wave);
        lb.init(op.b, p.ldb, op.own_b, depth, wave * NB);
        auto request = [&](int kt) {
            unsigned char* const st = smem + (kt & 1) * (STAGE + A_STAGE);
            lb.request(kt, st + wave * (NB * 1024));
            la.request(kt, st + STAGE + wave * 1024);
        };
        typename E::Acc acc[2][MR];
        constexpr bool kTwoLevels = E::kBytes == 4;  // as in the 128 x 128 tiles
        typename E::Acc total[kTwoLevels ? 2 : 1][kTwoLevels ? MR : 1];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < MR; ++i) {
                acc[j][i] = typename E::Acc{0, 0, 0, 0};
                if constexpr (kTwoLevels) total[j][i] = typename E::Acc{0, 0, 0, 0};
            }
        request(0);
        for (int kt = 0; kt < nk; ++kt) {
            // tile kt is in, and this wave's reads of the other stage are done
            __builtin_amdgcn_s_waitcnt(waitcnt_vm(0) & kWaitLgkm0);
            barrier_no_fence();
            if (kt + 1 < nk) request(kt + 1);
            const unsigned char* const st = smem + (kt & 1) * (STAGE + A_STAGE);
            typename E::Frag fa[2][MR], fb[2][2];
            read_pair<E, kAcrossB>(st, wave * 32, fb);
            read_frags<E, false, MR>(st + STAGE, 0, fa);
            if (kt == nk - 1 && depth % E::kPer) {
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const int valid = depth - kt * E::kDepth - (s * 4 + lc) * E::kPer;
#pragma unroll
                    for (int i = 0; i < MR; ++i) fa[s][i] = head<E>(fa[s][i], valid);
                    if constexpr (!kAcrossB)
#pragma unroll
                        for (int j = 0; j < 2; ++j) fb[s][j] = head<E>(fb[s][j], valid);
                }
            }
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int i = 0; i < MR; ++i) acc[j][i] = E::mma(fb[s][j], fa[s][i], acc[j][i]);
            if constexpr (kTwoLevels)
                if (kt % 8 == 7)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int i = 0; i < MR; ++i) {
                            total[j][i] += acc[j][i];
                            acc[j][i] = typename E::Acc{0, 0, 0, 0};
                        }
        }
        if constexpr (kTwoLevels)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < MR; ++i) acc[j][i] += total[j][i];
        __builtin_amdgcn_s_waitcnt(waitcnt_vm(0) & kWaitLgkm0);  // no request may outlive the loop
        barrier_no_fence();  // LDS becomes the stores' scratch
        store_tile<E, kForm, kBf16Out, MR, 2, false>(
            p, t, t.r0, smem + wave * 4096, [&](int q) { return t.c0 + wave * 32 + q * 4; }, [&](int i, int j) { return acc[j][i]; });
    };
    auto by_rows = [&](auto once_c) {
        if (nr > 16) run(std::integral_constant<int, 2>{}, once_c);
        else run(std::integral_constant<int, 1>{}, once_c);
    };
    if (p.once && t.row_tiles == 1) by_rows(std::true_type{});
    else by_rows(std::false_type{});
}

template <typename E, int kForm>
void launch_few(const GroupedParams& p, unsigned grid, hipStream_t s) {
    if (p.out_bf16) grouped_few_kernel<E, kForm, true><<<grid, FT, 0, s>>>(p);
    else grouped_few_kernel<E, kForm, false><<<grid, FT, 0, s>>>(p);
}

}  // namespace

hipError_t launch_grouped_few(const GroupedParams& p, GroupedForm form, GroupedElem elem, long long tiles, hipStream_t s) {
    if (form == kWeightGrad) return hipErrorInvalidValue;
    if (tiles <= 0) return hipSuccess;
    const unsigned grid = (unsigned)((tiles + 63) / 64 * 64);
    if (elem == kElemI8) launch_few<I8, kForward>(p, grid, s);
    else if (elem == kElemBf16 && form == kForward) launch_few<Bf16, kForward>(p, grid, s);
    else if (elem == kElemBf16) launch_few<Bf16, kInputGrad>(p, grid, s);
    else if (form == kForward) launch_few<F32, kForward>(p, grid, s);
    else launch_few<F32, kInputGrad>(p, grid, s);
    return hipGetLastError();
}

}  // namespace flexmoe
