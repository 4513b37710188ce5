"""Routing with scores, a bias and groups, its tables and its gradient, against their definitions in 64 bits.

Choices are compared for equality: the reference decides on scores in 64 bits, from the same logits.  Weights, u = 2^-24: a log score
of size s carries 2 u s + 4 u (its exp, log1p and sum), the exponential of a difference the same as a relative error, a sum of up
to 256 positive terms 12 u more, quotient and scale 2 u."""
import math

import pytest

torch = pytest.importorskip("torch")
from paper_2606_27866_amd import flexmoe as fm  # noqa: E402

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
NEG = -math.inf


def reference(logits, bias, k, score, normalize, scale, groups, top_groups, best):
    """(ids, weights) token by token, in plain Python order: value descending, id ascending, NaN last, -inf never."""
    x = logits.double().cpu()
    T, E = x.shape
    s = torch.sigmoid(x) if score == "sigmoid" else torch.softmax(x, 1)
    by_logits = bias is None and (groups == 1 or best == 1)
    c = x if by_logits else s if bias is None else s + bias.double().cpu()
    masked = x == NEG
    if bias is not None:
        masked = masked | (bias.cpu() == NEG)
    ids, w = torch.full((T, k), -1, dtype=torch.int32), torch.zeros(T, k, dtype=torch.float64)
    size = E // groups

    def order(v):
        return (math.isnan(v), -v if not math.isnan(v) else 0.0)

    for t in range(T):
        row, m = c[t].tolist(), masked[t].tolist()
        ranked = []
        for g in range(groups):
            members = sorted((order(row[e]), row[e]) for e in range(g * size, (g + 1) * size) if not m[e])
            if members:
                total = members[0][1] if best == 1 or len(members) == 1 else members[0][1] + members[1][1]
                ranked.append((order(total), g))
        kept = {g for _, g in sorted(ranked)[:top_groups]}
        chosen = sorted((order(row[e]), e) for e in range(E) if not m[e] and e // size in kept)[:k]
        for j, (_, e) in enumerate(chosen):
            ids[t, j] = e
        if chosen:
            of = [e for _, e in chosen]
            if normalize:
                ls = torch.nn.functional.logsigmoid(x[t, of]) if score == "sigmoid" else x[t, of]
                ww = torch.softmax(ls, 0)
                if score == "softmax" and bool(torch.isnan(x[t]).any()):
                    ww = ww * math.nan
            else:
                ww = s[t, of]
            w[t, :len(of)] = scale * ww
    return ids, w


def check_tables(r, E):
    """counts, offsets, perm and pos against the ids."""
    idx = r.topk_idx.cpu().view(-1).long()
    live = idx >= 0
    counts = torch.bincount(idx[live], minlength=E)
    assert torch.equal(r.counts.cpu().long(), counts)
    offsets = torch.cat((torch.zeros(1, dtype=torch.long), counts.cumsum(0)))
    assert torch.equal(r.offsets.cpu().long(), offsets)
    order = torch.sort(torch.where(live, idx, E), stable=True).indices[:int(live.sum())]
    perm = torch.full_like(idx, -1)
    perm[:len(order)] = order
    assert torch.equal(r.perm.cpu().long(), perm)
    pos = torch.full_like(idx, -1)
    pos[order] = torch.arange(len(order))
    assert torch.equal(r.pos.cpu().long(), pos)


def make(T, E, seed=0, dtype=torch.float32, std=1.5, bias=False):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000 + T + E)
    x = torch.empty(T, E, device="cuda").normal_(0, std, generator=g).to(dtype)
    b = torch.empty(E, device="cuda").normal_(0, 0.2, generator=g) if bias else None
    return g, x, b


def check(x, b, k, score="softmax", normalize=True, scale=1.0, groups=1, top_groups=1, best=1, max_tokens=None):
    T, E = x.shape
    router = fm.Router(E, k, T if max_tokens is None else max_tokens, score, normalize, scale, groups, top_groups, best)
    r = router.route(x, b)
    ids, w = reference(x, b, k, score, normalize, scale, groups, top_groups, best)
    assert torch.equal(r.topk_idx.cpu(), ids)
    finite = x.double()[torch.isfinite(x)]
    big = float(finite.abs().max()) if finite.numel() else 0.0
    bound = (4 * min(big, 1e3) + 30) * U
    got, want = r.topk_w.cpu().double(), w
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    ok = ~torch.isnan(want)
    assert bool(((got - want).abs()[ok] <= (bound * want.abs() + 2.0 ** -126)[ok]).all())
    assert bool((got[ids < 0] == 0).all())
    check_tables(r, E)
    alone = router.route(x, b, tables=False)
    assert torch.equal(alone.topk_idx, r.topk_idx) and torch.equal(alone.topk_w.view(torch.int32), r.topk_w.view(torch.int32)) and alone.perm is None
    return router, r


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("normalize", [False, True])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 64, 8), (3, 2, 2), (16, 60, 4), (17, 63, 7), (33, 65, 16), (130, 256, 8), (200, 8, 2), (1, 256, 16)])
def test_choice_and_weights(score, normalize, T, E, k):
    _, x, _ = make(T, E)
    check(x, None, k, score, normalize, 2.5)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("T", [1, 15, 16, 17, 100])
@pytest.mark.parametrize("E,groups,top_groups,best,k", [(8, 1, 1, 1, 2), (8, 4, 2, 1, 4), (16, 8, 3, 2, 5), (60, 5, 2, 2, 6), (256, 8, 4, 2, 8),
                                                        (256, 64, 3, 2, 10), (64, 64, 9, 1, 9), (255, 3, 2, 2, 16)])
def test_bias_and_groups(score, T, E, groups, top_groups, best, k):
    _, x, b = make(T, E, bias=True)
    check(x, b, k, score, True, 1.0, groups, top_groups, best)
    check(x, None, k, score, False, 1.0, groups, top_groups, best)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_ties_go_to_the_lower_id(dtype):
    x = (torch.arange(40 * 64, device="cuda").view(40, 64) * 7 % 5).to(dtype)
    x[3] = 0.0
    x[3, 1::2] = -0.0
    for bias in (None, torch.zeros(64, device="cuda")):
        for score in ("softmax", "sigmoid"):
            check(x, bias, 9, score)
            check(x, bias, 9, score, groups=8, top_groups=3, best=2)


def test_scores_next_to_each_other():
    """Scores that differ by less than 32 bits hold: a bias of 1 leaves 24 bits of a score near 1e-3."""
    g, x, _ = make(300, 64)
    x = -7 + x * 1e-6
    check(x, torch.ones(64, device="cuda"), 8, "sigmoid")
    check(x, torch.ones(64, device="cuda"), 8, "softmax")
    check(x, torch.ones(64, device="cuda"), 4, "sigmoid", groups=8, top_groups=2, best=2)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("level", [20.0, 60.0, 86.0, 100.0])
def test_scores_far_down(score, level):
    """Small scores are less exact in 32 bits, and past e^-87 they are none: sums of a group's two best that depend on it."""
    g, x, _ = make(300, 64)
    x = -level + x * 1e-6 * level
    x[:, 63] = 0.0
    check(x, None, 8, score, groups=16, top_groups=4, best=2)
    check(x, torch.full((64,), 2.0 ** -80, device="cuda"), 8, score)
    x = torch.full((4, 16), -300.0, device="cuda")
    x[:, 14] = 0.0
    x[:, 0], x[:, 1], x[:, 6] = -86.5, -88.0, -86.4
    x[1, :2], x[1, 6] = -86.45, -86.4
    x[2, 1] = -89.5
    check(x, None, 4, score, groups=8, top_groups=2, best=2)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups,best", [(1, 1), (4, 1), (4, 2)])
def test_masks(score, groups, best):
    """-inf in some places, in all but a few, everywhere; the lowest finite value; a bias of -inf."""
    low = torch.finfo(torch.float32).min
    g, x, b = make(60, 32, bias=True)
    x[torch.rand(60, 32, generator=g, device="cuda") < 0.5] = NEG
    x[3], x[17], x[59] = NEG, NEG, NEG
    x[5, 1:] = NEG
    x[6, :] = NEG
    x[6, 30:] = -1.0
    x[7], x[8, 3:] = low, low
    b[4] = NEG
    for bias in (None, b):
        for normalize in (True, False):
            check(x, bias, 4, score, normalize, 1.0, groups, max(1, groups // 2), best)
    router = fm.Router(32, 4, 60, score)
    r = router.route(x)
    for t in (3, 17, 59):
        assert bool((r.topk_idx[t] == -1).all()) and bool((r.topk_w[t] == 0).all())


def test_not_a_number():
    g, x, b = make(40, 16, bias=True)
    x[2, 5], x[9], x[11, 0] = math.nan, math.nan, math.nan
    x[11, 1:] = NEG
    for score in ("softmax", "sigmoid"):
        check(x, None, 3, score)
        check(x, None, 3, score, normalize=False)
    r = fm.Router(16, 3, 40, "sigmoid").route(x, b)
    assert bool(torch.isfinite(r.topk_w[:2]).all()) and int(r.topk_idx[2, 0]) >= 0 and 5 not in r.topk_idx[2].tolist()


def test_rows_of_a_wider_buffer():
    g = torch.Generator(device="cuda")
    wide = torch.empty(50, 100, device="cuda").normal_(generator=g)
    x = wide[:, 3:40]
    check(x, None, 5)
    router = fm.Router(37, 5, 50)
    out = torch.full((50, 41), 9.0, device="cuda")
    r = router.route(x)
    dw = torch.ones(50, 5, device="cuda")
    d = router.backward(x, r.topk_idx, dw, dlogits=out[:, 2:39])
    assert bool((out[:, :2] == 9).all()) and bool((out[:, 39:] == 9).all())
    assert torch.equal(d, router.backward(x.contiguous(), r.topk_idx, dw))


def test_many_tokens():
    """Every chunk's length: one token more or less than whole chunks, and a batch that fills them all."""
    for T in (2047, 2048, 2049, 5000, 20011, 32768, 32769, 65537, 131075):
        _, x, _ = make(T, 24, seed=T)
        router = fm.Router(24, 3, max(T, 30000))
        r = router.route(x)
        assert torch.equal(r.topk_idx.long(), x.sort(dim=1, descending=True, stable=True).indices[:, :3])
        check_tables(r, 24)


def gradient(x, ids, dw, score, normalize, scale):
    """Autograd in 64 bits through the weights of the given ids."""
    with torch.enable_grad():
        v = x.double().clamp(min=-1e5).requires_grad_()
        live = ids >= 0
        at = ids.clamp(min=0).long()
        logs = torch.nn.functional.logsigmoid(v) if score == "sigmoid" else torch.log_softmax(v, 1)
        of = logs.gather(1, at).masked_fill(~live, -1e5)
        w = torch.softmax(of, 1) if normalize else of.exp()
        (scale * w * dw.double() * live).sum().backward()
    return v.grad


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("normalize", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 8, 2), (5, 60, 4), (130, 256, 16), (33, 65, 3)])
def test_backward(score, normalize, dtype, T, E, k):
    """Each factor is off by at most 40 u of itself, a difference g - mean by 40 u of the largest |g| of its row."""
    g, x, _ = make(T, E, dtype=dtype)
    if T > 4:
        x[2], x[4, 3:] = NEG, NEG
    router = fm.Router(E, k, T, score, normalize, 1.5)
    ids = router.route(x, tables=False).topk_idx
    dw = torch.empty(T, k, device="cuda").normal_(generator=g)
    dl = router.backward(x, ids, dw)
    ref = gradient(x, ids, dw, score, normalize, 1.5)
    size = 1.5 * dw.abs().amax(1, keepdim=True).double()
    assert dl.dtype == dtype
    assert bool(((dl.double() - ref).abs() <= 80 * U * size + torch.finfo(dtype).eps / 2 * ref.abs()).all())
    assert bool((dl[x == NEG] == 0).all())


def test_gradient_against_differences():
    g, x, _ = make(3, 10)
    c = torch.empty(3, 3, device="cuda").normal_(generator=g)
    for score in ("softmax", "sigmoid"):
        for normalize in (False, True):
            router = fm.Router(10, 3, 3, score, normalize, 2.0)
            ids = router.route(x).topk_idx
            dl = router.backward(x, ids, c)
            h = 1e-2  # the choice is the same on both sides: the chosen are further apart here
            for t, e in ((0, int(ids[0, 0])), (1, int(ids[1, 2])), (2, 4)):
                f = []
                for step in (h, -h):
                    v = x.clone()
                    v[t, e] += step
                    r = router.route(v)
                    if not torch.equal(r.topk_idx.sort(1).values, ids.sort(1).values):
                        break
                    at = (r.topk_idx.unsqueeze(2) == ids.unsqueeze(1)).double()
                    f.append(float((at * (r.topk_w.double().unsqueeze(2) * c.double().unsqueeze(1))).sum()))
                if len(f) == 2:
                    assert abs((f[0] - f[1]) / (2 * h) - float(dl[t, e])) < 1e-3


def test_no_tokens():
    router = fm.Router(8, 2, 10)
    r = router.route(torch.empty(0, 8, device="cuda"))
    assert r.topk_idx.shape == (0, 2) and bool((r.counts == 0).all()) and bool((r.offsets == 0).all())
    assert router.backward(torch.empty(0, 8, device="cuda"), r.topk_idx, r.topk_w).shape == (0, 8)


def test_routes_as_the_layer_does():
    """Softmax without bias or groups: the layer's own routing and tables."""
    T, E, k, d = 300, 24, 4, 64
    g, logits, _ = make(T, E)
    layer = fm.Layer(d, E, 64, k, max_tokens=T)
    layer.set_weights(*[torch.zeros(E, *s, dtype=torch.bfloat16, device="cuda") for s in ((64, d), (64, d), (d, 64))])
    i32 = dict(dtype=torch.int32, device="cuda")
    dbg = dict(topk_idx=torch.empty(T * k, **i32), topk_w=torch.empty(T * k, device="cuda"), counts=torch.empty(E, **i32),
               offsets=torch.empty(E + 1, **i32), perm=torch.empty(T * k, **i32), pos=torch.empty(T * k, **i32))
    layer.forward(torch.zeros(T, d, dtype=torch.bfloat16, device="cuda"), logits, dbg=dbg)
    r = fm.Router(E, k, T).route(logits)
    for name in ("topk_idx", "counts", "offsets", "perm", "pos"):
        assert torch.equal(getattr(r, name).view(-1), dbg[name]), name
    assert bool(((r.topk_w.view(-1) - dbg["topk_w"]).abs() <= 80 * U * dbg["topk_w"]).all())
