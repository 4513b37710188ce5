"""The K loops of the 256 x 256 tiles (grouped_big.hip with its stores, mfma_pingpong.h), compiled for the host with
requests, waits, barriers and LDS reads that write down when they happen: whatever two waves do to the same LDS bytes is
ordered by a wait and a barrier.

A wave's accesses carry the number of barriers it had passed when they began and when they were known to be done (a
request: the wait that drains it; a read: the wait for LDS, or at once where the wait is part of the read).  An access that
was done after b barriers is before another wave's that began after b + 1."""
import os
import re
import subprocess

import pytest

from paper_2606_27866_amd import flexmoe as fm

HALF, WAVES, REQUEST, SCRATCH = 16384, 8, 1024, 4096

COMMON = """
#include <cstdio>
#include <type_traits>
#include <cstddef>
#include <cstdint>
constexpr int STAGE = 16384, NR = 2;
static unsigned char memory[8 * STAGE];
static unsigned char* const smem = memory;
// bit 8 clear: waits for LDS; low 8 bits: requests left in flight
constexpr int waitcnt_vm(int n) { return 0x100 | n; }
constexpr int kWaitLgkm0 = 0xff;
inline void __builtin_amdgcn_s_waitcnt(int w) { std::printf("wait %d %d\\n", w & 0xff, !(w & 0x100)); }
inline void barrier_no_fence() { std::printf("barrier\\n"); }
inline void __builtin_amdgcn_sched_barrier(int) {}
inline void __builtin_amdgcn_s_setprio(int) {}
inline void requested(int kt, const unsigned char* dst) { std::printf("request %d %d\\n", kt, (int)(dst - smem)); }
"""

STUBS = COMMON + """
struct Tile { int r0, c0; };
struct E { struct Frag {}; struct Acc {}; static constexpr int kDepth = 64; static Acc mma(Frag, Frag, Acc c) { return c; } };
template <typename T, bool kAcross, int F> void read_frags(const unsigned char* at, int, typename T::Frag (&)[2][F]) {
    std::printf("read %d %d\\n", (int)(at - smem), kAcross);
}
template <typename T, bool kAcross> void read_pair(const unsigned char* at, int, typename T::Frag (&)[2][2]) {
    std::printf("read %d %d\\n", (int)(at - smem), kAcross);
}
template <typename T, int N> void clear_tail(typename T::Frag (&)[2][N], int) {}
template <typename T, int kForm, bool kBf16Out, int kRows, int kCols, bool kWhole, typename P, typename C, typename V>
void store_tile(P, const Tile&, int, unsigned char* scratch, C, V) { std::printf("store %d\\n", (int)(scratch - smem)); }

struct Loader { void request(int kt, unsigned char* dst) { for (int i = 0; i < NR; ++i) requested(kt, dst + i * 1024); } };
template <typename E, int MF, bool kAcrossA, bool kAcrossB>
void run(int wave, int depth) {
    constexpr bool kTail = false, kBf16Out = false;
    constexpr int kForm = 0;
    const int wm = wave >> 2, wn = wave & 3, nk = (depth + E::kDepth - 1) / E::kDepth, p = 0;
    const Tile t{0, 0};
    Loader la[2], lb[2];
    typename E::Acc acc[2][2][2 * MF];
"""

PINGPONG = COMMON + """
#define __device__
#define __forceinline__ inline
constexpr int BK = 64, PP_HALF = STAGE, PP_ND = 2, PP_RPI = 8, ROWB = 128;
constexpr uint32_t kOOB = 0x80000000u;
typedef int __amdgpu_buffer_rsrc_t;
struct floatx4 { float v[4]; };
struct bf16x8 {};
struct bf16_t {};
struct PPOperands { int ra, rb[2]; uint32_t aoff[2][PP_ND], boff[2][PP_ND]; int col[PP_ND]; int K; };
struct PPSecond { const bf16_t *a, *a2, *b, *b2; size_t aext, bext; };
struct PPNoSecond {};
struct PPZeroTail { void operator()(int, int, unsigned char*) const {} };
template <int MF> using PPAcc = floatx4[2][2][2 * MF];
inline int ceil_div(int a, int b) { return (a + b - 1) / b; }
inline int make_rsrc(const bf16_t*, size_t) { return 0; }
inline void load_lds16(int, uint32_t, uint32_t soff, unsigned char* dst) { requested(soff / (BK * 2), dst); }
inline bf16x8 lds_frag(const unsigned char* at, int, int) { std::printf("read %d 0\\n", (int)(at - smem)); return {}; }
inline floatx4 __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf16x8, bf16x8, floatx4 c, int, int, int) { return c; }
"""

MAIN = """
int main(int argc, char** argv) {
    int form, nk;
    std::sscanf(argv[1], "%d", &form), std::sscanf(argv[2], "%d", &nk);
    for (int w = 0; w < 8; ++w) std::printf("wave\\n"), trace(w, nk, form);
}
"""

GROUPED_TRACE = """
}
void trace(int wave, int nk, int form) {
    if (form == 2) run<E, 4, true, true>(wave, nk * E::kDepth);
    else if (form == 1) run<E, 1, false, true>(wave, nk * E::kDepth);
    else run<E, 3, false, false>(wave, nk * E::kDepth);
}
"""

# the loop's callers meet at a barrier before they use LDS for themselves
PINGPONG_TRACE = """
template <int MF>
void run(int wave, int nk) {
    PPAcc<MF> acc;
    PPOperands op{};
    op.K = nk * BK;
    pp_loop<MF, false>(smem, op, wave, 0, acc, PPZeroTail{});
    barrier_no_fence();
    for (int h = 0; h < 2; ++h) std::printf("store %d\\n", h * 8 * 4096 + wave * 4096);
}
void trace(int wave, int nk, int form) {
    if (form) run<4>(wave, nk);
    else run<1>(wave, nk);
}
"""


FORMS = [("grouped", 0), ("grouped", 1), ("grouped", 2), ("pingpong", 0), ("pingpong", 1)]


@pytest.fixture(scope="module")
def lines(tmp_path_factory):
    """lines(form, nk): what the eight waves of a tile of nk K tiles write down."""
    csrc = os.path.join(os.path.dirname(fm.__file__), "csrc")
    d = tmp_path_factory.mktemp("order")

    def part(name, pattern):
        return re.search(pattern, open(os.path.join(csrc, name)).read(), re.S | re.M).group(0)

    texts = dict(grouped=STUBS + part("grouped_big.hip", r"^        // halves: 0 A0.*?\* MF \+ i\]; \}\);$") + GROUPED_TRACE + MAIN,
                 pingpong=PINGPONG + part("mfma_pingpong.h", r"^template <int MF, bool kSwap, typename Tail.*?^}$") + PINGPONG_TRACE + MAIN)
    for name, text in texts.items():
        (d / (name + ".cpp")).write_text(text)
        subprocess.run(["g++", "-std=c++17", "-w", "-o", str(d / name), str(d / (name + ".cpp"))], check=True)

    def run(form, nk):
        out = subprocess.run([str(d / form[0]), str(form[1]), str(nk)], check=True, capture_output=True, text=True).stdout.splitlines()
        # a read of several fragments is one access
        return [x for i, x in enumerate(out) if not (x.startswith("read") and i and out[i - 1] == x)]

    return run


class Access:
    def __init__(self, wave, kind, at, size, slot, index, tag=None):
        self.wave, self.kind, self.at, self.end, self.began, self.index, self.tag = wave, kind, at, at + size, slot, index, tag
        self.done = self.done_index = None  # barriers passed, and place in the wave's own order

    def finish(self, slot, index):
        self.done, self.done_index = slot, index

    def before(self, other):
        if self.done is None:
            return False
        return self.done_index <= other.index if self.wave == other.wave else self.done < other.began


def accesses(lines):
    out, wave, barriers = [], -1, []
    for index, line in enumerate(lines):
        op, *args = line.split()
        args = [int(a) for a in args]
        if op == "wave":
            wave, slot, flying, reading = wave + 1, 0, [], []
            barriers.append(0)
        elif op == "barrier":
            slot += 1
            barriers[-1] = slot
        elif op == "request":
            a = Access(wave, "write", args[1], REQUEST, slot, index, args[0])
            out.append(a)
            flying.append(a)
        elif op == "wait":
            while len(flying) > args[0]:
                flying.pop(0).finish(slot, index)
            if args[1]:
                for a in reading:
                    a.finish(slot, index)
                reading = []
        elif op == "read":
            a = Access(wave, "read", args[0], HALF, slot, index)
            out.append(a)
            if args[1]:
                a.finish(slot, index)
            else:
                reading.append(a)
        elif op == "store":
            out.append(Access(wave, "store", args[0], SCRATCH, slot, index))
    return out, barriers


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("nk", range(8))
def test_accesses_to_the_same_bytes_are_ordered(lines, form, nk):
    acc, barriers = accesses(lines(form, nk))
    assert len(barriers) == WAVES and len(set(barriers)) == 1  # every wave meets the same barriers
    assert sum(a.kind == "store" for a in acc) == 2 * WAVES
    unordered = set()
    for i, a in enumerate(acc):
        for b in acc[i + 1:]:
            if a.at < b.end and b.at < a.end and (a.kind != "read" or b.kind != "read") and not a.before(b) and not b.before(a):
                if a.wave == b.wave and a.kind == b.kind == "store":
                    continue  # one wave's scratch, in its own order
                unordered.add((a.kind, a.wave, b.kind, b.wave))
    assert not unordered, sorted(unordered)


@pytest.mark.parametrize("form", FORMS)
def test_a_read_sees_its_own_tile(lines, form):
    """Of the requests for a half before a read of it, the last is the K tile that the phase multiplies: A0 B1 A1 of tile kt,
    then B0 of the next."""
    nk = 5
    acc, _ = accesses(lines(form, nk))
    for w in range(WAVES):
        reads = [a for a in acc if a.wave == w and a.kind == "read"]
        want = [(2, 0)] + [h for kt in range(nk) for h in ((0, kt), (3, kt), (1, kt), (2, kt + 1))]
        assert len(reads) == len(want)
        for a, (half, kt) in zip(reads, want):
            assert a.at == ((kt & 1) * 4 + half) * HALF
            for other in range(WAVES):
                past = [b.tag for b in acc if b.wave == other and b.kind == "write" and a.at <= b.at < a.end and b.before(a)]
                assert len(past) >= 2 and max(past) == kt
