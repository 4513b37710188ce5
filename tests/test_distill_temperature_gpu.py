"""Distillation at temperatures below 1 and far below it: formulas and bounds of test_distill_gpu.py, the temperature rounded to fp32 as the
descriptor holds it; and a listed token's logarithm, which is in 64 bits: a KL that is one long logarithm is off by its own rounding alone."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
from paper_2606_27866_amd import flexmoe as fm  # noqa: E402
from tests.test_distill_gpu import BF16, F32, U, check, make  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("t", [0.7, 0.1, 1e-6])
@pytest.mark.parametrize("rows,V", [(4, 1000), (3, 50001), (600, 3000), (1700, 30001), (510, 65001)])
def test_rows(dtype, tail, t, rows, V):
    """Two sums with the sharper one at t; the last sizes are held whole (the last in fp32). At 1e-6 the logits span 10 t all the same."""
    t = float(np.float32(t))
    g, x, ids, lp, labels = make(rows, V, 16, dtype)
    if t < 1e-3:
        x *= t
    teacher = x.float() / t + torch.empty(rows, V, device="cuda").normal_(0, 1, generator=g)
    lp, ids = torch.log_softmax(teacher, 1).topk(16, 1)
    ids, lp = ids.int().contiguous(), lp.contiguous()
    scale = torch.linspace(0.5, 2.0, rows, device="cuda")
    check(x, ids, lp, None, scale, t, tail)
    check(x, ids, lp, labels, scale, t, tail, 0.4, 1.5)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("t", [0.7, 0.1, 0.3, 1.1, 3.0, 1e-3, 1e-6, 7e5])
def test_one_long_logarithm(tail, t):
    """The teacher is on one token far below another: KL = (largest - x) / t, whose sums (S = 1) are off by (1 / 256 + 30) u at most."""
    t = float(np.float32(t))
    rows, V = 64, 300
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    x = fm._padded((rows, V), F32, "cuda").fill_(-math.inf)
    gap = torch.empty(rows, device="cuda").uniform_(1e3, 1e4, generator=g) * t
    x[:, 1], x[:, 2] = gap / 3, gap / 3 - gap
    ids = torch.full((rows, 1), 2, dtype=torch.int32, device="cuda")
    kl = fm.Distillation(V, 1, rows, temperature=t, tail=tail).forward(x, ids, torch.zeros(rows, 1, device="cuda"))[0].double()
    want = (x[:, 1].double() - x[:, 2].double()) / t
    assert bool(((kl - want).abs() <= U * want + 32 * U).all()), float(((kl - want).abs() / want).max() / U)
