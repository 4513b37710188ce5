"""Which tiles and how many parts a product takes, from the rule in grouped_api.hip compiled for the host, and sizes that
take each of them."""
import ctypes
import os
import re
import subprocess

from paper_2606_27866_amd import flexmoe as fm

KINDS = ("mid", "slim", "big", "few")
FORMS = ("forward", "input_grad", "weight_grad")


def compile_rule(directory):
    """plan(form, type of the operands, type of the result, groups, N, K, R) -> (kind, parts)."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(fm.__file__)))
    csrc = os.path.join(os.path.dirname(fm.__file__), "csrc")

    def read(name):
        return open(os.path.join(csrc, name)).read()

    api, grouped = read("grouped_api.hip"), read("grouped.h")
    enums = "\n".join(re.findall(r"^enum Grouped.*?;$", grouped, re.M))
    consts = "\n".join(re.findall(r"^constexpr int kGroup.*?;.*?$", grouped, re.M))
    consts += "\n" + re.search(r"^constexpr size_t kMostPartial.*?$", api, re.M).group(0)
    rule = api[api.index("// How a product is cut into workgroups."):api.index("int launch(const flexmoe_grouped_desc* D")]
    src = os.path.join(str(directory), "plan.cpp")
    with open(src, "w") as f:
        f.write('#include <algorithm>\n#include <cmath>\n#include <cstdint>\n#include "flexmoe.h"\n'
                "static int ceil_div(int a, int b) { return (a + b - 1) / b; }\n" + enums + "\n" + consts + "\n" + rule + """
extern "C" int plan_of(int form, int int8, int dtype, int dw_dtype, int groups, int N, int K, int R) {
    flexmoe_grouped_desc D{groups, N, K, dtype, dw_dtype, FLEXMOE_KEEP_NONE, R, 0, 0, 0, 0};
    const Plan p = plan(D, (GroupedForm)form, int8 != 0, R, kMostPartial);
    return p.tiles * 1000 + p.splits;
}
""")
    out = os.path.join(str(directory), "plan.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", os.path.join(root, "include"), "-o", out, src], check=True)
    lib = ctypes.CDLL(out)

    def plan(form, elem, result, groups, N, K, R):
        int8 = elem == "i8"
        code = lib.plan_of(FORMS.index(form), int(int8), int((result if int8 else elem) == "bf16"), int(result == "bf16"), groups, N, K, R)
        return KINDS[code // 1000], code % 1000

    return plan


# (form, type of the operands, of the result, tiles, parts of the reduction, groups, N, K, R): every pair of tiles and parts
# that the rule has for a form and its types
SIZES = [
    ("forward", "bf16", "bf16", "big", "one", 5, 2313, 131, 3178),
    ("forward", "bf16", "bf16", "big", "several", 9, 143, 6969, 1527),
    ("forward", "bf16", "bf16", "few", "one", 1, 148, 204, 69),
    ("forward", "bf16", "bf16", "few", "several", 1, 157, 617, 135),
    ("forward", "bf16", "bf16", "mid", "one", 1, 169, 132, 5),
    ("forward", "bf16", "bf16", "mid", "several", 1, 143, 903, 1),
    ("forward", "f32", "f32", "few", "one", 1, 139, 162, 1),
    ("forward", "f32", "f32", "few", "several", 1, 141, 260, 41),
    ("forward", "f32", "f32", "mid", "one", 1, 142, 143, 1),
    ("forward", "f32", "f32", "mid", "several", 1, 137, 272, 1),
    ("forward", "i8", "bf16", "big", "one", 5, 389, 133, 18081),
    ("forward", "i8", "bf16", "big", "several", 10, 135, 8160, 3667),
    ("forward", "i8", "bf16", "few", "one", 1, 156, 145, 103),
    ("forward", "i8", "bf16", "few", "several", 1, 157, 1344, 97),
    ("forward", "i8", "bf16", "mid", "one", 1, 148, 137, 4),
    ("forward", "i8", "bf16", "mid", "several", 1, 147, 1717, 8),
    ("forward", "i8", "f32", "big", "one", 64, 389, 133, 12875),
    ("forward", "i8", "f32", "big", "several", 26, 138, 6682, 3539),
    ("forward", "i8", "f32", "few", "one", 1, 144, 138, 148),
    ("forward", "i8", "f32", "few", "several", 1, 150, 1632, 114),
    ("forward", "i8", "f32", "mid", "one", 1, 148, 135, 2),
    ("forward", "i8", "f32", "mid", "several", 1, 136, 1346, 33),
    ("input_grad", "bf16", "bf16", "big", "one", 9, 142, 402, 16580),
    ("input_grad", "bf16", "bf16", "big", "several", 8, 8087, 137, 1413),
    ("input_grad", "bf16", "bf16", "few", "one", 1, 138, 137, 116),
    ("input_grad", "bf16", "bf16", "few", "several", 1, 579, 230, 121),
    ("input_grad", "bf16", "bf16", "mid", "one", 1, 141, 135, 2),
    ("input_grad", "bf16", "bf16", "mid", "several", 1, 929, 134, 5),
    ("input_grad", "f32", "f32", "few", "one", 1, 168, 164, 1),
    ("input_grad", "f32", "f32", "few", "several", 1, 368, 158, 38),
    ("input_grad", "f32", "f32", "mid", "one", 1, 151, 135, 1),
    ("input_grad", "f32", "f32", "mid", "several", 1, 269, 154, 2),
    ("weight_grad", "bf16", "bf16", "big", "one", 11, 151, 1480, 6662),
    ("weight_grad", "bf16", "bf16", "big", "several", 3, 153, 542, 17039),
    ("weight_grad", "bf16", "bf16", "mid", "one", 1, 337, 1058, 536),
    ("weight_grad", "bf16", "bf16", "mid", "several", 1, 141, 131, 493),
    ("weight_grad", "bf16", "bf16", "slim", "one", 1, 137, 139, 2),
    ("weight_grad", "bf16", "f32", "big", "one", 12, 145, 1488, 6646),
    ("weight_grad", "bf16", "f32", "big", "several", 3, 137, 523, 15053),
    ("weight_grad", "bf16", "f32", "mid", "one", 1, 424, 893, 525),
    ("weight_grad", "bf16", "f32", "mid", "several", 1, 143, 131, 453),
    ("weight_grad", "bf16", "f32", "slim", "one", 1, 132, 141, 1),
    ("weight_grad", "f32", "bf16", "mid", "one", 15, 167, 137, 1367),
    ("weight_grad", "f32", "bf16", "mid", "several", 1, 142, 185, 145),
    ("weight_grad", "f32", "bf16", "slim", "one", 1, 139, 155, 1),
    ("weight_grad", "f32", "f32", "mid", "one", 20, 135, 158, 1183),
    ("weight_grad", "f32", "f32", "mid", "several", 1, 137, 188, 129),
    ("weight_grad", "f32", "f32", "slim", "one", 1, 132, 133, 6),
]


def rows_of(groups, R):
    """Uneven rows of every group, the second with none."""
    if groups == 1:
        return [R]
    share = [0 if e == 1 else 1 + e % 3 for e in range(groups)]
    rows = [R * s // sum(share) for s in share]
    rows[0] += R - sum(rows)
    return rows


# depths of 2 to 5 K tiles and rows of the last 256 x 256 tile of a group (each number of its 64-row steps)
BIG_DEPTHS, BIG_LAST = (104, 128, 192, 256, 320), (1, 65, 129, 193, 256)


def big_sizes(last):
    """(groups, N, R) of bf16 products x W^T on 256 x 256 tiles at those depths: groups of equal rows."""
    return 4, 2304, 4 * (1280 + last)
