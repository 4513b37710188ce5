"""Distillation and cross entropy of each row and the logits' gradient against their formulas in 64 bits.

Bounds, u = 2^-24, d = (largest - x) / t.  A sum over the vocabulary is off by err = (range / 256 + 30) u of itself (positive terms, 20 joins,
each term within 4 u + 2 u d where e^-d d < 0.4).  The listed tokens' logarithms add the rounding of 1 / t, u d.  So KL is off by twice err + u d (q and
q_rest), CE by err + u, each rounded once more; a gradient's term q by err + (8 + 4 d) u of itself, with a tail times 1 + p_rest / q_rest, whose
quotient carries twice err; then half a step of its type.  Terms below 2^-126 of their factor are 0."""
import math

import pytest

torch = pytest.importorskip("torch")
from paper_2606_27866_amd import flexmoe as fm  # noqa: E402

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
NEG = -math.inf
BF16, F32 = torch.bfloat16, torch.float32


def make(rows, V, K, dtype, seed=0, t=1.0, extra=8):
    """Student, and a teacher's list that partly agrees with it."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 31 + rows * 7 + V + K)
    wide = torch.full((rows, -(-V // 8) * 8 + extra), float("nan"), dtype=dtype, device="cuda")
    x = wide[:, :V]
    x.copy_(torch.empty(rows, V, device="cuda").normal_(0, 2, generator=g))
    teacher = (x.float() + torch.empty(rows, V, device="cuda").normal_(0, 1, generator=g)) / t
    lp, ids = torch.log_softmax(teacher, 1).topk(K, 1)
    labels = torch.randint(0, V, (rows,), generator=g, device="cuda").int()
    return g, x, ids.int().contiguous(), lp.contiguous(), labels


def reference(x, ids, lp, labels, scale, t, tail, klw, cew):
    """(kl, ce, gradient, size of the gradient's terms) row by row; a token's first place in its list counts."""
    x, lp = x.double(), lp.double()
    R, V = x.shape
    first = (ids.unsqueeze(2) == ids.unsqueeze(1)).long().argmax(2) == torch.arange(ids.shape[1], device=ids.device)
    ok = (ids >= 0) & (ids < V) & first
    at = torch.where(ok, ids, 0).long()
    top = x.amax(1, keepdim=True)
    z = (x - top) / t
    S = z.exp().sum(1, keepdim=True)
    logq = z - S.log()
    q = logq.exp()
    listed = torch.zeros(R, V + 1, dtype=torch.bool, device=x.device).scatter_(1, torch.where(ok, at, V), True)[:, :V]
    if tail:
        p = torch.where(ok, lp.exp(), 0.0)
        rest = (1 - p.sum(1, keepdim=True)).clamp(min=0)
        logp = lp
    else:
        masked = torch.where(ok, lp, NEG)
        logp = masked - torch.logsumexp(masked, 1, keepdim=True)
        p = torch.where(ok & (masked > NEG), logp.exp(), 0.0)
        rest = torch.zeros(R, 1, dtype=torch.float64, device=x.device)
    mass = p.sum(1, keepdim=True)
    kl = torch.where(p > 0, p * (logp - logq.gather(1, at)), 0.0).sum(1)
    q_rest = torch.where(listed, 0.0, q).sum(1, keepdim=True)
    ratio = torch.zeros_like(rest)
    if tail:
        none = q_rest == 0
        part = rest * (rest.log() - q_rest.log())
        kl = kl + torch.where(rest == 0, 0.0, torch.where(none, torch.where(rest <= 1e-5, 0.0, math.inf), part)).squeeze(1)
        ratio = torch.where(none, 0.0, rest / q_rest)
    total = mass + rest
    target = torch.zeros(R, V + 1, dtype=torch.float64, device=x.device).scatter_add_(1, torch.where(ok, at, V), p)[:, :V]
    grad = klw * t * torch.where(listed, total * q - target, (total - ratio) * q)
    size = klw * t * q * (1 + ratio)
    ce = torch.zeros(R, dtype=torch.float64, device=x.device)
    if labels is not None:
        inside = (labels >= 0) & (labels < V)
        y = labels.clamp(0, V - 1).long().unsqueeze(1)
        z1 = x - top
        log1 = z1 - z1.exp().sum(1, keepdim=True).log()
        ce = torch.where(inside, -log1.gather(1, y).squeeze(1), 0.0)
        g1 = log1.exp().scatter_add(1, y, torch.full((R, 1), -1.0, dtype=torch.float64, device=x.device))
        grad = grad + torch.where(inside.unsqueeze(1), cew * g1, 0.0)
        size = size + abs(cew) * log1.exp()
    if scale is not None:
        s = scale.double().unsqueeze(1)
        off = (scale == 0)
        kl, ce = kl.masked_fill(off, 0), ce.masked_fill(off, 0)
        grad, size = torch.where(off.unsqueeze(1), 0.0, s * grad), torch.where(off.unsqueeze(1), 0.0, s.abs() * size)
    return kl, ce, grad, size


def near(a, b, bound):
    a = a.double()
    assert torch.equal(torch.isnan(a), torch.isnan(b))
    whole = torch.isfinite(b)
    assert torch.equal(a[torch.isinf(b)], b[torch.isinf(b)])
    off = (a - b).abs()[whole] - bound[whole]
    assert bool((off <= 0).all()), (float(off.max()), float(((a - b).abs() / bound)[whole].max()))


def check(x, ids, lp, labels=None, scale=None, t=1.0, tail=False, klw=1.0, cew=0.0, holder=None):
    R, V = x.shape
    K = ids.shape[1]
    h = holder or fm.Distillation(V, K, R, temperature=t, tail=tail, kl_weight=klw, ce_weight=cew)
    kl0, ce0 = h.forward(x, ids, lp, labels, scale)
    ref = reference(x, ids, lp, labels, scale, t, tail, klw, cew)
    kl, ce, d = h.gradient(x, ids, lp, labels, scale)
    err = (min(V, 131072) / 256 + 30) * U
    z = x.double() / t
    fin = torch.where(torch.isfinite(z), z, 0.0)
    deep = (fin.amax(1) - fin.amin(1))
    # the losses alone may be summed in another order than with the gradient: both within the bounds
    near(kl0, ref[0], 2 * (err + 2 * U * deep) * (2 if tail else 1) + 2 * U * torch.nan_to_num(ref[0].abs(), posinf=0.0))
    near(ce0, ref[1], err + 2 * U * torch.nan_to_num(ref[1].abs(), posinf=0.0) + 2 * U)
    near(kl, ref[0], 2 * (err + 2 * U * deep) * (2 if tail else 1) + 2 * U * torch.nan_to_num(ref[0].abs(), posinf=0.0))
    near(ce, ref[1], err + 2 * U * torch.nan_to_num(ref[1].abs(), posinf=0.0) + 2 * U)
    assert d.dtype == x.dtype
    d_each = torch.where(torch.isfinite(z), z.amax(1, keepdim=True) - z, 0.0).clamp(max=100)
    rel = 3 * err + (10 + 4 * d_each) * U * max(1.0, t)
    bound = rel * ref[3] + torch.finfo(x.dtype).eps / 2 * ref[2].abs() + 2 * U * ref[2].abs() + 2.0 ** -120 * (1 + abs(klw) * t + abs(cew))
    near(d, ref[2], bound)
    return kl, ce, d


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("rows,V,K", [(1, 2, 1), (3, 7, 2), (2, 8, 4), (5, 9, 8), (1, 300, 128), (4, 1000, 100), (1, 2049, 20), (30, 4097, 5),
                                      (600, 3000, 16), (2, 50001, 65), (1, 131072, 64), (2, 131073, 40), (1, 300007, 100)])
def test_rows(dtype, tail, rows, V, K):
    _, x, ids, lp, labels = make(rows, V, K, dtype)
    check(x, ids, lp, tail=tail)
    check(x, ids, lp, labels, tail=tail, klw=0.7, cew=0.3)
    _, x, ids, lp, labels = make(rows, V, K, dtype, t=2.0)
    scale = torch.linspace(0.5, 2.0, rows, device="cuda")
    check(x, ids, lp, None, scale, 2.0, tail)
    check(x, ids, lp, labels, scale, 2.0, tail, 0.4, 1.5)


# from 96 MB of logits on, and where the last round of workgroups is full enough, rows are held whole: three sizes of workgroups
WHOLE = [(BF16, 1700, 30001), (BF16, 1500, 50003), (BF16, 500, 131072), (F32, 1600, 16001), (F32, 1000, 32003), (F32, 510, 65001)]


@pytest.mark.parametrize("dtype,rows,V", WHOLE)
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("t", [1.0, 2.0])
def test_whole_rows(dtype, rows, V, tail, t):
    """The rows of test_masks_... and padding among ordinary ones: a workgroup takes several, one after another."""
    low = torch.finfo(dtype).min
    g, x, ids, lp, labels = make(rows, V, 40, dtype, t=t)
    at = torch.randperm(rows, generator=g, device="cuda")
    x[at[0], torch.rand(V, generator=g, device="cuda") < 0.5] = NEG
    x[at[1], ids[at[1], 3].long()] = NEG
    x[at[2], labels[at[2]].long()] = NEG
    x[at[3]] = low
    x[at[4], ids[at[4], 0].long()] = float("nan")
    x[at[5]] = torch.finfo(dtype).max
    ids[at[6], 5] = ids[at[6], 2]
    ids[at[7], 4:] = -1
    labels[at[8]], labels[at[9]] = ids[at[8], 1], -100
    ids[at[10]] = -1
    ids[at[11], 0], ids[at[12], 0] = 0, V - 1
    scale = torch.linspace(0.5, 2.0, rows, device="cuda")
    scale[at[20:rows // 3]] = 0
    x[at[20]] = float("nan")
    keep = x.clone() if dtype == F32 else None
    _, _, d = check(x, ids, lp, labels if t == 2.0 else None, scale, t, tail, 0.8, 0.6)
    if keep is not None:
        assert torch.equal(torch.nan_to_num(keep, nan=1.5), torch.nan_to_num(x, nan=1.5))
    h = fm.Distillation(V, 40, rows, temperature=t, tail=tail, kl_weight=0.8, ce_weight=0.6)
    into = fm._padded((rows, V), dtype, "cuda").copy_(x)  # in the place of the logits: the same bits
    h.gradient(into, ids, lp, labels if t == 2.0 else None, scale, dlogits=into)
    assert torch.equal(torch.nan_to_num(into.float(), nan=1.5), torch.nan_to_num(d.float(), nan=1.5))


@pytest.mark.parametrize("live", [[0], [1599], [255, 256, 1000], list(range(600, 900)), list(range(0, 1600, 3))])
def test_few_rows_with_a_loss_among_whole_rows(live):
    """Long runs of padding: whole groups of rows that hold nothing to do, and workgroups that get no row."""
    rows, V = 1600, 32000
    _, x, ids, lp, labels = make(rows, V, 20, BF16)
    scale = torch.zeros(rows, device="cuda")
    scale[live] = 0.5
    x[scale == 0] = float("nan")
    h = fm.Distillation(V, 20, rows, tail=True, ce_weight=0.5)
    out = fm._padded((rows, V), BF16, "cuda").fill_(3.0)
    kl, ce, d = h.gradient(x, ids, lp, labels, scale, dlogits=out)
    off = scale == 0
    assert not bool(kl[off].any()) and not bool(ce[off].any()) and not bool(d[off].any())
    on = torch.tensor(live, device="cuda")
    ref = reference(x[on], ids[on], lp[on], labels[on], scale[on], 1.0, True, 1.0, 0.5)
    err = (V / 256 + 30) * U
    near(ce[on], ref[1], err + 2 * U * ref[1].abs() + 2 * U)
    # as in check: the sums' relative error in each term, and one rounding to bf16
    near(d[on], ref[2], 2.0 ** -8 * ref[2].abs() + 4 * (err + 60 * U) * ref[3] + 2.0 ** -133)
    assert all(torch.equal(a, b) for a, b in zip((kl, ce, d), h.gradient(x, ids, lp, labels, scale)))


def test_nothing_but_padding_or_masks_in_whole_rows():
    rows, V = 1700, 30001
    _, x, ids, lp, labels = make(rows, V, 8, BF16)
    h = fm.Distillation(V, 8, rows, tail=True, ce_weight=1.0)
    kl, ce, d = h.gradient(x, ids, lp, labels, torch.zeros(rows, device="cuda"))
    assert not kl.any() and not ce.any() and not d.any()
    x[:] = NEG
    kl, ce, d = h.gradient(x, ids, lp, labels)
    assert bool((kl == math.inf).all()) and bool((ce == math.inf).all()) and not d.any()


def test_labels_alone_and_outside():
    """Weights of 0, labels that are ignored, labels on and off the list."""
    _, x, ids, lp, labels = make(8, 500, 20, F32)
    labels[0], labels[1], labels[2] = -100, 500, ids[2, 3]
    labels[3] = ids[3, 0]
    check(x, ids, lp, labels, klw=0.0, cew=1.0)
    kl, ce, _ = check(x, ids, lp, labels, cew=1.0, tail=True)
    assert float(ce[0]) == 0 and float(ce[1]) == 0 and bool((ce[2:] > 0).all())


@pytest.mark.parametrize("tail", [False, True])
def test_lists(tail):
    """Tokens named twice (the first place counts), ids outside, probabilities of 0, nothing listed, everything listed."""
    _, x, ids, lp, labels = make(8, 40, 12, F32)
    ids[0, 5], ids[0, 9] = ids[0, 2], ids[0, 2]
    ids[1, 4:] = -1
    ids[2, 0] = 40
    lp[3, 6:] = NEG
    ids[4] = -1
    ids[5] = ids[5, 0]
    ids[6, 11] = -5
    check(x, ids, lp, labels, tail=tail, cew=0.5)
    check(x, ids, lp, tail=tail)
    _, x, ids, lp, _ = make(4, 30, 30, F32)  # all of the vocabulary
    kl, _, d = check(x, ids, lp, tail=tail)
    assert bool(torch.isfinite(kl).all()) and bool(torch.isfinite(d).all())
    _, x, ids, lp, _ = make(3, 9, 12 - 3, F32)
    h = fm.Distillation(9, 12, 3, tail=tail)  # a list that is longer than the vocabulary
    more = torch.cat((ids, torch.full((3, 3), -1, dtype=torch.int32, device="cuda")), 1).contiguous()
    kl2, _, d2 = h.gradient(x, more, torch.cat((lp, torch.zeros(3, 3, device="cuda")), 1).contiguous())
    kl, _, d = check(x, ids, lp, tail=tail)
    assert torch.equal(kl, kl2) and torch.equal(d, d2)


def test_logits_over_the_temperature_do_as_well():
    """Without a tail a shift of a row's list changes nothing but roundings (of the shifted values: 2^-24 times their size)."""
    _, x, ids, lp, _ = make(5, 700, 30, F32)
    h = fm.Distillation(700, 30, 5)
    a, b = h.forward(x, ids, lp)[0], h.forward(x, ids, lp + 8.0)[0]
    assert bool(((a - b).abs() <= 64 * U * 8).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("V", [600, 9000])
def test_masks_and_values_that_are_no_numbers(dtype, tail, V):
    low = torch.finfo(dtype).min
    g, x, ids, lp, labels = make(9, V, 10, dtype)
    x[0, torch.rand(V, generator=g, device="cuda") < 0.5] = NEG
    x[0, ids[0].long()] = 1.0
    x[1, ids[1, 3].long()] = NEG          # the teacher is on a masked token
    x[2, labels[2].long()] = NEG          # the label is
    x[3] = NEG
    x[3, ids[3].long()] = 0.5             # nothing but the list is left
    x[4] = low
    x[5, ids[5, 0].long()] = float("nan")
    x[6] = torch.finfo(dtype).max
    lp[7] = torch.log_softmax(lp[7], 0)
    for lab in (None, labels):
        live = [0, 1, 2, 4, 5, 6, 7, 8] + ([3] if not tail else [])
        check(fm._padded((len(live), V), dtype, "cuda").copy_(x[live]), ids[live].contiguous(), lp[live].contiguous(),
              None if lab is None else lab[live].contiguous(), tail=tail, cew=0.5)
    if tail:  # the teacher leaves a tenth and more to masked tokens
        kl, _, _ = fm.Distillation(V, 10, 9, tail=True).gradient(x, ids, lp)
        assert float(kl[3]) == math.inf


def test_a_row_of_nothing_but_masks():
    for V in (100, 5000):
        for tail in (False, True):
            _, x, ids, lp, labels = make(3, V, 6, F32)
            x[1] = NEG
            kl, ce, d = fm.Distillation(V, 6, 3, tail=tail, ce_weight=1.0).gradient(x, ids, lp, labels)
            assert float(kl[1]) == math.inf and float(ce[1]) == math.inf and bool((d[1] == 0).all())
            assert bool(torch.isfinite(kl[[0, 2]]).all()) and bool(torch.isfinite(d[[0, 2]]).all())


@pytest.mark.parametrize("rows,V", [(6, 800), (6, 70000), (600, 900)])
def test_padding_is_not_read(rows, V):
    _, x, ids, lp, labels = make(rows, V, 9, BF16)
    scale = torch.full((rows,), 0.25, device="cuda")
    scale[rows // 2:] = 0
    x[rows // 2:] = float("nan")
    ids[rows // 2:] = 2 ** 31 - 1
    lp[rows // 2:] = float("nan")
    labels[rows // 2:] = -2 ** 31
    for tail in (False, True):
        h = fm.Distillation(V, 9, rows, tail=tail, ce_weight=0.5)
        out = fm._padded((rows, V), BF16, "cuda").fill_(3.0)
        kl, ce, d = h.gradient(x, ids, lp, labels, scale, dlogits=out)
        assert bool((kl[rows // 2:] == 0).all()) and bool((ce[rows // 2:] == 0).all()) and bool((d[rows // 2:] == 0).all())
        assert bool(torch.isfinite(d).all()) and bool((kl[: rows // 2] > 0).all())


@pytest.mark.parametrize("rows,V", [(3, 77), (600, 2000), (2, 40000), (300, 9000)])
def test_in_the_place_of_the_logits_and_nothing_past_a_row(rows, V):
    for dtype in (BF16, F32):
        _, x, ids, lp, labels = make(rows, V, 7, dtype)
        h = fm.Distillation(V, 7, rows, tail=True, ce_weight=0.5)
        want = h.gradient(x, ids, lp, labels)
        wide = torch.full((rows, -(-V // 8) * 8 + 16), 7.0, dtype=dtype, device="cuda")
        wide[:, :V] = x
        kl, ce, d = h.gradient(wide[:, :V], ids, lp, labels, dlogits=wide[:, :V])
        assert torch.equal(kl, want[0]) and torch.equal(ce, want[1]) and torch.equal(wide[:, :V], want[2]) and bool((wide[:, V:] == 7).all())


def test_gradient_against_differences():
    """Central differences of the loss in fp32 logits: step 1e-2, third-order terms below 1e-4 of the loss's size here."""
    for tail, t in ((False, 1.0), (True, 2.0)):
        _, x, ids, lp, labels = make(3, 25, 6, F32, t=t)
        scale = torch.tensor([1.0, 0.5, 2.0], device="cuda")
        h = fm.Distillation(25, 6, 3, temperature=t, tail=tail, kl_weight=0.8, ce_weight=0.6)
        d = h.gradient(x, ids, lp, labels, scale)[2]

        def loss(v):
            kl, ce = h.forward(v, ids, lp, labels, scale)
            return float((scale.double() * (0.8 * t * t * kl.double() + 0.6 * ce.double())).sum())

        for i, j in ((0, 0), (1, int(ids[1, 2])), (2, int(labels[2])), (2, 24)):
            up, down = fm._padded((3, 25), F32, "cuda").copy_(x), fm._padded((3, 25), F32, "cuda").copy_(x)
            up[i, j] += 1e-2
            down[i, j] -= 1e-2
            assert abs((loss(up) - loss(down)) / 2e-2 - float(d[i, j])) < 2e-3


def test_rows_of_the_gradient_sum_to_zero():
    """softmax gradients: each row sums to 0 (V roundings of at most 2^-24 of terms whose sizes add up to 2 at most)."""
    _, x, ids, lp, labels = make(20, 6000, 50, F32)
    for tail in (False, True):
        d = fm.Distillation(6000, 50, 20, tail=tail, ce_weight=1.0).gradient(x, ids, lp, labels)[2]
        assert bool((d.double().sum(1).abs() < 1e-4).all())


def test_a_teacher_of_its_own_has_no_divergence():
    """The student's own log probabilities: KL 0 within the sums' bound, with a tail even where the rest is small."""
    _, x, _, _, _ = make(50, 5000, 8, F32)
    x *= 3
    lp, ids = torch.log_softmax(x.double(), 1).topk(40, 1)
    kl, _, d = fm.Distillation(5000, 40, 50, tail=True).gradient(x, ids.int(), lp.float())
    err = (5000 / 256 + 60) * U * 3
    assert bool((kl.abs() < err).all()) and bool((d.abs() < 4 * err).all())


def test_deterministic_and_smaller_calls():
    _, x, ids, lp, labels = make(40, 30000, 30, BF16)
    a, b = (fm.Distillation(30000, 30, n, tail=True, ce_weight=0.1) for n in (40, 3000))
    first = a.gradient(x, ids, lp, labels)
    for h in (a, b):
        assert all(torch.equal(p, q) for p, q in zip(h.gradient(x, ids, lp, labels), first))


def test_offsets_past_32_bits():
    V, rows = 131080, 16500  # 2.16e9 values
    x = torch.zeros(rows, V, dtype=BF16, device="cuda")
    ids = torch.full((rows, 1), 77, dtype=torch.int32, device="cuda")
    scale = torch.zeros(rows, device="cuda")
    scale[-2:] = 1
    kl, _, d = fm.Distillation(V, 1, rows).gradient(x, ids, torch.zeros(rows, 1, device="cuda"), row_scale=scale, dlogits=x)
    assert bool(((kl[-2:].double() - math.log(V)).abs() < 1e-4).all())
    assert abs(float(d[-1, 77]) + 1) < 0.01 and abs(float(d[-1, 78]) * V - 1) < 0.01 and float(d[0].abs().max()) == 0


def test_no_rows():
    kl, ce, d = fm.Distillation(64, 4, 10).gradient(torch.empty(0, 64, device="cuda"), torch.empty(0, 4, dtype=torch.int32, device="cuda"),
                                                    torch.empty(0, 4, device="cuda"))
    assert kl.shape == (0,) and ce.shape == (0,) and d.shape == (0, 64)
