// Grouped products on 256 x 256 tiles (gfx950): bf16 in every form, int8.
//
// A workgroup of 8 waves; wave (wm, wn) = (wave / 4, wave % 4) owns, in each of
// the four 128 x 128 quadrants (A half, B half), 16 * MF rows and 32 columns of
// C (128 accumulator registers at MF = 4).  K tiles are 128 bytes deep, LDS
// holds two of them as halves A0 A1 B0 B1 of 16 KB (128 KB).
//
// The two waves of a SIMD (w and w + 4) run half a phase apart: while one
// multiplies a quadrant, the other reads fragments and requests operands, and
// an s_barrier after each part swaps them.  A K tile takes four phases; each
// reads one half from LDS and requests one:
//   phase   LDS reads            requests from memory   multiplies
//     0     A half 0 (tile kt)   A half 1 (kt + 1)      A0 x B0
//     1     B half 1 (kt)        B half 0 (kt + 2)      A0 x B1
//     2     A half 1 (kt)        A half 0 (kt + 2)      A1 x B1
//     3     B half 0 (kt + 1)    B half 1 (kt + 2)      A1 x B0
// A half read in phase i is refilled from phase i + 2 on, one barrier after its
// last reader; a request leaves six phases before its data is read, and the
// wait at the end of a phase leaves the last five phases' requests in flight.
// Across halves are read through the transposing LDS reads, whose wait is part
// of the read: there the requests go out first.
//
// The order of all waves' accesses to LDS is that of mfma_pingpong.h's loop; both
// are checked on the host from their own text.
//
// Bound by the matrix cores at the card's power limit: 8192^3 in bf16 1519 (x
// W^T), 1454 (dy W at 2048 columns), 1345 TFLOP/s (dy^T x), where the vendor's
// library reaches 1574 to 1600 (x W^T) in the same run; 8192^3 in int8, with the
// rounding of the rows, 2555 TOP/s.  Another card, 1377 (x W^T), with runs of 32
// tiles per XCD instead of 8: 1150.
#include "grouped.h"

namespace flexmoe {

namespace {
using namespace mfma;

constexpr int BT = 512;                  // threads
constexpr int NR = STAGE / 1024 / 8;     // requests per wave and half: 2
constexpr int BIG_SMEM = 8 * STAGE;

// The depths from `valid` on set to zero.
template <typename E, int N>
__device__ __forceinline__ void clear_tail(typename E::Frag (&f)[2][N], int valid) {
    const int lc = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < N; ++i) f[s][i] = head<E>(f[s][i], valid - (s * 4 + lc) * E::kPer);
}
template <typename E, int kForm, bool kBf16Out>
__global__ __launch_bounds__(BT, 2) void grouped_big_kernel(GroupedParams p) {
    constexpr bool kAcrossA = kForm == kWeightGrad, kAcrossB = kForm != kForward;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[BIG_SMEM];
    GroupedTile t;
    if (!grouped_tile<kForm>(p, xcd_tile(8), kGroupBigTile, kGroupBigTile, 64, E::kDepth, t)) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 2, wn = wave & 3;
    const int nr = t.r1 - t.r0, depth = t.d1 - t.d0;
    const Operands<E, kForm> op(p, t);
    const int nk = ceil_div(depth, E::kDepth);

    // kTail: the reduction ends inside a 16-byte unit of an along operand (a
    // loop of its own: the test and the clearing cost registers)
    auto run = [&](auto mf_c, auto tail_c) {
        constexpr int MF = decltype(mf_c)::value;
        constexpr bool kTail = decltype(tail_c)::value;
        Loader<E, kAcrossA, NR> la[2];
        Loader<E, kAcrossB, NR> lb[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            // A half h starts at C row h * 32 * MF of the tile
            if constexpr (kAcrossA) la[h].init(op.a + h * 128, p.lda, op.own_a - h * 128, depth, wave * NR);
            else la[h].init(op.a + (size_t)(h * 32 * MF) * p.lda, p.lda, min(op.own_a - h * 32 * MF, 32 * MF), depth, wave * NR);
            if constexpr (kAcrossB) lb[h].init(op.b + h * 128, p.ldb, op.own_b - h * 128, depth, wave * NR);
            else lb[h].init(op.b + (size_t)(h * 128) * p.ldb, p.ldb, op.own_b - h * 128, depth, wave * NR);
        }
        typename E::Acc acc[2][2][2 * MF];
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int f = 0; f < 2 * MF; ++f) acc[q >> 1][q & 1][f] = typename E::Acc{0, 0, 0, 0};
        // halves: 0 A0, 1 A1, 2 B0, 3 B1
        auto half_of = [&](int half, int kt) { return smem + ((kt & 1) * 4 + half) * STAGE; };
        auto request = [&](int half, int kt) {
            unsigned char* dst = half_of(half, kt) + wave * (NR * 1024);
            if (half < 2) la[half].request(kt, dst);
            else lb[half & 1].request(kt, dst);
        };
        typename E::Frag fa[2][MF], fx[2][2], fy[2][2];  // [K step][fragment]
        auto read_a = [&](int half, int kt) {
            read_frags<E, kAcrossA, MF>(half_of(half, kt), wm * 16 * MF, fa);
            if constexpr (!kAcrossA) {
                if (kTail && kt == nk - 1) clear_tail<E, MF>(fa, depth - kt * E::kDepth);
            }
        };
        auto read_b = [&](int half, int kt, typename E::Frag (&f)[2][2]) {
            read_pair<E, kAcrossB>(half_of(2 + half, kt), wn * 32, f);
            if constexpr (!kAcrossB) {
                if (kTail && kt == nk - 1) clear_tail<E, 2>(f, depth - kt * E::kDepth);
            }
        };
        auto multiply = [&](typename E::Acc (&c)[2 * MF], const typename E::Frag (&f)[2][2]) {
            __builtin_amdgcn_s_waitcnt(waitcnt_vm(5 * NR));
            __builtin_amdgcn_sched_barrier(0);
            barrier_no_fence();
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
            __builtin_amdgcn_s_setprio(1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int i = 0; i < MF; ++i) c[j * MF + i] = E::mma(f[s][j], fa[s][i], c[j * MF + i]);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(0);
            barrier_no_fence();
            __builtin_amdgcn_sched_barrier(0);
        };
        // B half 0 of tile kt is in x at the start; x holds B half 0 and y B
        // half 1 of the tile, and y B half 0 of the next tile at the end
        auto tile = [&](int kt, typename E::Frag (&x)[2][2], typename E::Frag (&y)[2][2]) {
            if constexpr (!kAcrossA) read_a(0, kt);
            request(1, kt + 1);
            if constexpr (kAcrossA) read_a(0, kt);
            multiply(acc[0][0], x);
            if constexpr (!kAcrossB) read_b(1, kt, y);
            request(2, kt + 2);
            if constexpr (kAcrossB) read_b(1, kt, y);
            multiply(acc[0][1], y);
            if constexpr (!kAcrossA) read_a(1, kt);
            request(0, kt + 2);
            if constexpr (kAcrossA) read_a(1, kt);
            multiply(acc[1][1], y);
            if constexpr (!kAcrossB) read_b(0, kt + 1, y);
            request(3, kt + 2);
            if constexpr (kAcrossB) read_b(0, kt + 1, y);
            multiply(acc[1][0], x);
        };
        request(2, 0);
        request(0, 0);
        request(3, 0);
        request(1, 0);
        request(2, 1);
        request(0, 1);
        request(3, 1);
        __builtin_amdgcn_s_waitcnt(waitcnt_vm(5 * NR));  // B0 and A0 of tile 0 are in
        barrier_no_fence();
        if (wm == 1) barrier_no_fence();  // the lagging waves; the leading ones wait at the end
        __builtin_amdgcn_sched_barrier(0);
        read_b(0, 0, fx);
        // its half is refilled in phase 1 of the leading waves, a slot sooner after
        // this read than the loop's are after theirs
        __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
        int kt = 0;
        for (; kt + 1 < nk; kt += 2) {
            tile(kt, fx, fy);
            tile(kt + 1, fy, fx);
        }
        if (kt < nk) tile(kt, fx, fy);
        __builtin_amdgcn_s_waitcnt(waitcnt_vm(0) & kWaitLgkm0);
        if (wm == 0) barrier_no_fence();
        // the lagging waves meet that barrier with up to five phases' zero fills
        // in flight: one more, behind every wave's wait, before LDS becomes the
        // stores' scratch
        barrier_no_fence();
        __builtin_amdgcn_sched_barrier(0);

#pragma unroll
        for (int ah = 0; ah < 2; ++ah)
            store_tile<E, kForm, kBf16Out, MF, 4, false>(
                p, t, t.r0 + ah * 32 * MF + wm * 16 * MF, smem + wave * 4096,
                [&](int q) { return t.c0 + (q >> 3) * 128 + wn * 32 + (q & 7) * 4; },
                [&](int i, int j) { return acc[ah][j >> 1][(j & 1) * MF + i]; });
    };
    auto by_rows = [&](auto tail_c) {
        if (nr > 192) run(std::integral_constant<int, 4>{}, tail_c);
        else if (nr > 128) run(std::integral_constant<int, 3>{}, tail_c);
        else if (nr > 64) run(std::integral_constant<int, 2>{}, tail_c);
        else run(std::integral_constant<int, 1>{}, tail_c);
    };
    if constexpr (kAcrossA) run(std::integral_constant<int, 4>{}, std::false_type{});
    else if (depth % E::kPer) by_rows(std::true_type{});
    else by_rows(std::false_type{});
}

template <typename E, int kForm>
void launch_big(const GroupedParams& p, unsigned grid, hipStream_t s) {
    if (p.out_bf16) grouped_big_kernel<E, kForm, true><<<grid, BT, 0, s>>>(p);
    else grouped_big_kernel<E, kForm, false><<<grid, BT, 0, s>>>(p);
}

}  // namespace

hipError_t launch_grouped_big(const GroupedParams& p, GroupedForm form, GroupedElem elem, long long tiles, hipStream_t s) {
    if (elem == kElemF32) return hipErrorInvalidValue;
    if (tiles <= 0) return hipSuccess;
    const unsigned grid = (unsigned)((tiles + 63) / 64 * 64);
    if (elem == kElemI8) launch_big<I8, kForward>(p, grid, s);
    else if (form == kForward) grouped_big_kernel<Bf16, kForward, true><<<grid, BT, 0, s>>>(p);
    else if (form == kInputGrad) grouped_big_kernel<Bf16, kInputGrad, true><<<grid, BT, 0, s>>>(p);
    else launch_big<Bf16, kWeightGrad>(p, grid, s);
    return hipGetLastError();
}

}  // namespace flexmoe
