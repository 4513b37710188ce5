"""Distillation with a tail where listed and other tokens lie far apart: the rest's share q_rest may be far below what fp32 holds, its
logarithm and the others' shares of it are not.

Reference in 64 bits from logarithms.  Bounds, u = 2^-24: a sum over the vocabulary is off by err = (range / 256 + 30) u of itself (positive terms, 20
joins, each term within 4 u + 2 u d where e^-d d < 0.4).  KL carries two such sums, each at most (sum p + p_rest) = 1 times, and terms whose
sizes add up to KL and the entropies (below 10), each with the rounding of 1 / t and of the result: 4 err + 3 u (|KL| + 10).  A gradient's terms are
p, q and p_rest q / q_rest, each off by 3 err + (10 + 4 d) u of itself, terms below 2^-126 are 0; then half a step of its type."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
from paper_2606_27866_amd import flexmoe as fm  # noqa: E402

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
NEG = -math.inf
BF16, F32 = torch.bfloat16, torch.float32
K = 12
KINDS = 9


def make(rows, V, dtype, t, seed):
    """Row r is of kind r % KINDS; logits spread over a few t."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 101 + rows + V)
    x = torch.empty(rows, V, device="cuda").normal_(0, 1, generator=g)
    ids = torch.stack([torch.randperm(V, generator=g, device="cuda")[:K] for _ in range(rows)])
    p = torch.empty(rows, K + 1, device="cuda").exponential_(1.0, generator=g)
    p[:, 0] += 4
    lp = torch.log(p / p.sum(1, keepdim=True))[:, :K].contiguous()  # what is left: about 6 %
    labels = torch.randint(0, V, (rows,), generator=g, device="cuda")
    kind = torch.arange(rows, device="cuda") % KINDS
    first = torch.zeros(rows, V, device="cuda").scatter_(1, ids[:, :1], 1.0)
    listed = torch.zeros(rows, V, device="cuda").scatter_(1, ids, 1.0)
    for k, gap in ((0, 90.0), (1, 110.0), (2, 1000.0)):  # one listed token above all others
        x += (kind == k).unsqueeze(1) * first * gap
    x += (kind == 3).unsqueeze(1) * listed * 95.0         # all listed tokens above the others
    x -= (kind == 4).unsqueeze(1) * listed * 200.0        # and below them
    alone = torch.rand(rows, V, generator=g, device="cuda") < 0.999
    alone &= torch.arange(V, device="cuda") != (listed == 0).long().argmax(1, keepdim=True)
    x = torch.where((kind == 5).unsqueeze(1) & (listed == 0) & alone, NEG, x + (kind == 5).unsqueeze(1) * listed * 300.0)  # few others, far below
    low = torch.rand(rows, V, generator=g, device="cuda") < 0.5
    x -= (kind == 6).unsqueeze(1) * (listed == 0) * torch.where(low, 70.0, 101.0)  # in reach of fp32, but for some
    at = torch.where(kind == 7, ids[:, 3], labels)        # the label is listed, else hardly ever
    x = fm._padded((rows, V), dtype, "cuda").copy_(x * t)
    return x, ids.int().contiguous(), lp, at.int().contiguous()


def reference(x, ids, lp, labels, scale, t, klw, cew):
    """(kl, ce, gradient, size of its terms, distance (largest - x) / t of each)"""
    x, lp, ids = x.double(), lp.double(), ids.long()
    z = x / t
    is_listed = torch.zeros_like(z, dtype=torch.bool).scatter_(1, ids, True)
    logq = z - torch.logsumexp(z, 1, keepdim=True)
    p = lp.exp()
    rest = (1 - p.sum(1, keepdim=True)).clamp(min=0)
    others = torch.where(is_listed, NEG, z)
    log_share = others - torch.logsumexp(others, 1, keepdim=True)  # of q_rest
    log_rest = torch.logsumexp(others, 1, keepdim=True) - torch.logsumexp(z, 1, keepdim=True)
    kl = (p * (lp - logq.gather(1, ids))).sum(1) + (rest * (rest.log() - log_rest)).squeeze(1)
    total = p.sum(1, keepdim=True) + rest
    target = torch.zeros_like(z).scatter_(1, ids, p)
    pull = torch.where(is_listed, target, rest * log_share.exp())
    grad, size = klw * t * (total * logq.exp() - pull), klw * t * (total * logq.exp() + pull)
    ce = torch.zeros_like(kl)
    if labels is not None:
        log1 = torch.log_softmax(x, 1)
        y = labels.long().unsqueeze(1)
        ce = -log1.gather(1, y).squeeze(1)
        one = torch.zeros_like(z).scatter_(1, y, 1.0)
        grad, size = grad + cew * (log1.exp() - one), size + cew * (log1.exp() + one)
    s = scale.double().unsqueeze(1)
    top = torch.where(is_listed, z.amax(1, keepdim=True), others.amax(1, keepdim=True))
    return kl, ce, s * grad, s * size, torch.nan_to_num(top - z, posinf=0.0).clamp(0, 100)


def check(x, ids, lp, labels, scale, t, klw, cew, got):
    err = (min(x.shape[1], 131072) / 256 + 30) * U
    kl, ce, grad, size, d = reference(x, ids, lp, labels, scale, t, klw, cew)
    for name, a, b, bound in (("kl", got[0], kl, 4 * err + 3 * U * (kl.abs() + 10)), ("ce", got[1], ce, err + 2 * U * (ce.abs() + 1))):
        a = a.double()
        inf = torch.isinf(b)
        assert bool(torch.isfinite(kl).all()) and torch.equal(a[inf], b[inf]), name
        off = (a - b).abs()[~inf] / bound[~inf]
        assert bool((off <= 1).all()), (name, off.tolist())
    if got[2] is not None:
        floor = 2.0 ** -120 * (1 + klw * t + cew) * scale.double().unsqueeze(1)
        bound = (3 * err + (10 + 4 * d) * U * max(1.0, t)) * size + torch.finfo(x.dtype).eps / 2 * grad.abs() + 2 * U * grad.abs() + floor
        off = ((got[2].double() - grad).abs() / bound).amax(1)
        assert bool((off <= 1).all()), off.tolist()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("t", [1.0, 0.1, 2.0, 1e-3])
@pytest.mark.parametrize("rows,V", [(9, 400), (18, 9001), (9, 140000), (600, 3000)])
def test_rows_in_parts(dtype, t, rows, V):
    t = float(np.float32(t))
    x, ids, lp, labels = make(rows, V, dtype, t, 1)
    scale = torch.linspace(0.5, 2.0, rows, device="cuda")
    for lab in (None, labels):
        h = fm.Distillation(V, K, rows, temperature=t, tail=True, kl_weight=0.8, ce_weight=0.6)
        kl, ce = h.forward(x, ids, lp, lab, scale)
        check(x, ids, lp, lab, scale, t, 0.8, 0.6, (kl, ce, None))
        check(x, ids, lp, lab, scale, t, 0.8, 0.6, h.gradient(x, ids, lp, lab, scale))


# as test_distill_gpu.py's: these are held whole
@pytest.mark.parametrize("dtype,rows,V", [(BF16, 1700, 30001), (BF16, 1500, 50003), (BF16, 500, 131072), (F32, 1600, 16001), (F32, 1000, 32003),
                                          (F32, 510, 65001)])
@pytest.mark.parametrize("t", [1.0, 0.1])
def test_whole_rows(dtype, rows, V, t):
    t = float(np.float32(t))
    few = 5 * KINDS
    part = make(few, V, dtype, t, 2)
    turn = torch.arange(rows, device="cuda") % few
    x = fm._padded((rows, V), dtype, "cuda").copy_(part[0][turn])
    ids, lp, labels = (a[turn].contiguous() for a in part[1:])
    scale = torch.ones(rows, device="cuda")
    for lab in (None, labels):
        h = fm.Distillation(V, K, rows, temperature=t, tail=True, kl_weight=0.8, ce_weight=0.6)
        kl, ce, d = h.gradient(x, ids, lp, lab, scale)
        check(part[0], part[1], part[2], None if lab is None else part[3], scale[:few], t, 0.8, 0.6, (kl[:few], ce[:few], d[:few]))
        for a in (kl, ce, d.view(torch.int16 if dtype == BF16 else torch.int32)):  # the same row: the same bits
            assert all(torch.equal(a[i:i + few], a[:len(a[i:i + few])]) for i in range(few, rows, few))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,V", [(3, 700), (1700, 30001)])
def test_largest_gap(dtype, rows, V):
    """The type's largest value on a listed token, its lowest on all others: the gap itself is past fp32's range."""
    top = torch.finfo(dtype).max
    x = fm._padded((rows, V), dtype, "cuda").fill_(-top)
    x[:, 5] = top
    ids = torch.full((rows, 2), -1, dtype=torch.int32, device="cuda")
    ids[:, 0] = 5
    lp = torch.full((rows, 2), math.log(0.9), device="cuda")
    kl, _, d = fm.Distillation(V, 2, rows, tail=True).gradient(x, ids, lp)
    rest = 1 - math.exp(float(lp[0, 0].double()))
    assert bool(((kl.double() - rest * 2 * top).abs() <= 4 * U * rest * 2 * top).all())
    share = rest / (V - 1)  # all others alike
    err = (V / 256 + 40) * U
    near = torch.full((V,), -share, dtype=torch.float64, device="cuda")
    near[5] = 1 - math.exp(float(lp[0, 0].double()))
    assert bool(((d.double() - near).abs() <= (3 * err + torch.finfo(dtype).eps / 2) * near.abs() + 2 * U * (torch.arange(V, device="cuda") == 5)).all())


def test_nothing_but_masks_beside_the_list():
    """Where no other token is left, what the teacher leaves makes KL infinite; labels and the list keep their gradients."""
    V, rows = 500, 4
    x = torch.full((rows, 504), NEG, device="cuda")[:, :V]
    ids = torch.arange(6, dtype=torch.int32, device="cuda").repeat(rows, 1).contiguous()
    x[:, :6] = torch.arange(6.0, device="cuda")
    lp = torch.log_softmax(torch.arange(6.0, device="cuda"), 0).repeat(rows, 1).contiguous()
    lp[1] -= 0.5
    labels = torch.tensor([2, 3, 77, -100], dtype=torch.int32, device="cuda")
    kl, ce, d = fm.Distillation(V, 6, rows, tail=True, ce_weight=1.0).gradient(x, ids, lp, labels)
    bound = 4 * (V / 256 + 30) * U
    q = torch.softmax(torch.arange(6.0, dtype=torch.float64), 0)
    assert float(kl[1]) == math.inf and bool((kl[[0, 2, 3]].abs() < bound).all())
    assert float(ce[2]) == math.inf and float(ce[3]) == 0 and abs(float(ce[0]) + math.log(q[2])) < bound
    want = q.clone()
    want[2] -= 1
    assert bool(((d[0, :6].double().cpu() - want).abs() < bound).all()) and not bool(d[:2, 6:].any()) and not bool(d[3, 6:].any())
    assert float(d[2, 77]) == -1 and bool(torch.isfinite(d).all())


def test_gradient_against_differences():
    """Central differences of KL over a gap of 100 t in fp32 logits, t = 0.5: the loss in units of u (|KL| + 10), step 2^-5."""
    t, V = 0.5, 40
    x, ids, lp, _ = make(1, V, F32, t, 3)
    ids = ids[:, :K].contiguous()
    x[0, int(ids[0, 0])] = 50.0
    h = fm.Distillation(V, K, 1, temperature=t, tail=True)
    d = h.gradient(x, ids, lp)[2]
    step = 2.0 ** -5
    others = [v for v in range(V) if v not in ids[0].tolist()]
    for v in (others[0], others[7], int(ids[0, 0]), int(ids[0, 4])):
        loss = []
        for sign in (1, -1):
            y = fm._padded((1, V), F32, "cuda").copy_(x)
            y[0, v] += sign * step
            loss.append(float(h.forward(y, ids, lp)[0].double()) * t * t)
        # third derivative of t^2 KL: below 1 / t; roundings of the loss over 2 step
        assert abs((loss[0] - loss[1]) / (2 * step) - float(d[0, v])) <= step ** 2 / 6 / t + 2 * t * t * 40 * U * 30 / (2 * step)


@pytest.mark.parametrize("t", [0.7, 1.0, 2.0, 0.03])
def test_the_join_across_a_gap_keeps_small_divergences(t):
    """All others are 0, so that their sum is exact, and one listed token has about as much as they together: KL, a few hundredths at most, is off by
    the rounding of S (u), the logarithms of S and s (half a step of up to 0.35 each, u / 2 together) and its own, within 3 u."""
    t, rows, V = float(np.float32(t)), 48, 1 << 20
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    x = torch.zeros(rows, V, device="cuda")
    x[:, 77] = (math.log(V) + torch.empty(rows, device="cuda").uniform_(-0.3, 0.3, generator=g)) * t
    ids = torch.full((rows, 1), 77, dtype=torch.int32, device="cuda")
    lp = torch.log(torch.empty(rows, 1, device="cuda").uniform_(0.45, 0.55, generator=g))
    h = fm.Distillation(V, 1, rows, temperature=t, tail=True)
    p, others = lp.double().exp(), math.log(V - 1)
    top = x[:, 77:78].double() / t
    log_s = torch.logaddexp(top, torch.full_like(top, others))
    want = (p * (lp.double() - (top - log_s)) + (1 - p) * (torch.log1p(-p) - (others - log_s))).squeeze(1)
    for kl in (h.forward(x, ids, lp)[0], h.gradient(x, ids, lp)[0]):
        assert bool((want < 0.1).all())
        off = (kl.double() - want).abs() / U
        assert bool((off <= 3).all()), float(off.max())
