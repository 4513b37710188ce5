"""The 256 x 256 tiles' K loop and stores, compiled for the host from grouped_big.hip with requests, waits, barriers and LDS
reads that write down when they happen: the stores' scratch is ordered behind whatever else uses its bytes, by a wait and a
barrier.

A wave's accesses carry the number of barriers it had passed when they began and when they were known to be done (a
request: the wait that drains it; a read: the wait for LDS, or at once where the wait is part of the read).  An access that
was done after b barriers is before another wave's that began after b + 1."""
import os
import re
import subprocess

import pytest

from paper_2606_27866_amd import flexmoe as fm

HALF, WAVES, REQUEST, SCRATCH = 16384, 8, 2048, 4096

STUBS = """
#include <cstdio>
#include <type_traits>
typedef unsigned int uint32_t_;
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
struct Loader { void request(int kt, unsigned char* dst) { std::printf("request %d %d\\n", kt, (int)(dst - smem)); } };
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

template <typename E, int MF, bool kAcrossA, bool kAcrossB>
void run(int wave, int depth) {
    constexpr bool kTail = false, kBf16Out = false;
    constexpr int kForm = 0;
    const int wm = wave >> 2, wn = wave & 3, nk = (depth + E::kDepth - 1) / E::kDepth, p = 0;
    const Tile t{0, 0};
    Loader la[2], lb[2];
    typename E::Acc acc[2][2][2 * MF];
"""

MAIN = """
}
extern "C" void trace(int wave, int depth, int across) {
    if (across == 2) run<E, 4, true, true>(wave, depth);
    else if (across == 1) run<E, 1, false, true>(wave, depth);
    else run<E, 3, false, false>(wave, depth);
    std::fflush(stdout);
}
int main(int argc, char** argv) {
    int across, nk;
    std::sscanf(argv[1], "%d", &across), std::sscanf(argv[2], "%d", &nk);
    for (int w = 0; w < 8; ++w) std::printf("wave\\n"), trace(w, nk * E::kDepth, across);
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    src = open(os.path.join(os.path.dirname(fm.__file__), "csrc", "grouped_big.hip")).read()
    body = re.search(r"^        // halves: 0 A0.*?\* MF \+ i\]; \}\);$", src, re.S | re.M).group(0)
    d = tmp_path_factory.mktemp("order")
    (d / "t.cpp").write_text(STUBS + body + MAIN)
    subprocess.run(["g++", "-std=c++17", "-w", "-o", str(d / "t"), str(d / "t.cpp")], check=True)
    return str(d / "t")


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
            flying += [a] * (REQUEST // 1024)  # instructions that the wait counts
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


@pytest.mark.parametrize("across", [0, 1, 2])
@pytest.mark.parametrize("nk", range(8))
def test_the_scratch_of_the_stores_is_free(program, across, nk):
    lines = subprocess.run([program, str(across), str(nk)], check=True, capture_output=True, text=True).stdout.splitlines()
    acc, barriers = accesses(lines)
    assert len(barriers) == WAVES and len(set(barriers)) == 1  # every wave meets the same barriers
    assert sum(a.kind == "store" for a in acc) == 2 * WAVES
    unordered = set()
    for i, a in enumerate(acc):
        for b in acc[i + 1:]:
            if "store" not in (a.kind, b.kind):
                continue
            if a.at < b.end and b.at < a.end and not a.before(b) and not b.before(a):
                if a.wave == b.wave and a.kind == b.kind == "store":
                    continue  # one wave's scratch, in its own order
                unordered.add((a.kind, a.wave, b.kind, b.wave))
    assert not unordered, sorted(unordered)


@pytest.mark.parametrize("across", [0, 1, 2])
def test_a_read_sees_its_own_tile(program, across):
    """Of the requests for a half before a read of it, the last is the K tile that the phase multiplies: A0 B1 A1 of tile kt,
    then B0 of the next."""
    nk = 5
    lines = subprocess.run([program, str(across), str(nk)], check=True, capture_output=True, text=True).stdout.splitlines()
    acc, _ = accesses(lines)
    for w in range(WAVES):
        reads = [a for a in acc if a.wave == w and a.kind == "read"]
        want = [(2, 0)] + [h for kt in range(nk) for h in ((0, kt), (3, kt), (1, kt), (2, kt + 1))]
        assert len(reads) == len(want)
        for a, (half, kt) in zip(reads, want):
            assert a.at == ((kt & 1) * 4 + half) * HALF
            for other in range(WAVES):
                past = [b.tag for b in acc if b.wave == other and b.kind == "write" and a.at <= b.at < a.end and b.before(a)]
                assert past and max(past) == kt
