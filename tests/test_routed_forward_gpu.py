"""The layer's forward with a caller's routing: the bits of its own routing given back, slots that go nowhere, and the routers'
output taken as it is."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from paper_2606_27866_amd import flexmoe as fm  # noqa: E402
from paper_2606_27866_amd import synth  # noqa: E402
from tests.bruteforce import f64, silu  # noqa: E402
from tests.gpu_util import BF16_TOL, F32_TOL, check_y, mini_layer, say, y_to_f64  # noqa: E402

pytestmark = pytest.mark.gpu

# T, d, E, I, k, I_shared, dtype: one token, decode tiles, one workgroup's dispatch and more, 128 and 256 tiles, fp32
CASES = [(1, 256, 16, 200, 4, 128, synth.BF16), (16, 256, 60, 72, 4, 0, synth.BF16), (64, 128, 24, 72, 8, 64, synth.BF16),
         (65, 128, 24, 72, 8, 64, synth.BF16), (129, 128, 24, 72, 8, 0, synth.BF16), (300, 256, 8, 320, 2, 0, synth.BF16),
         (700, 136, 8, 264, 2, 256, synth.BF16), (90, 64, 6, 48, 2, 64, synth.F32), (600, 64, 16, 48, 3, 0, synth.F32)]


def layer_of(case):
    T, d, E, I, k, I_s, dtype = case
    cfg, x, lg, w, s = mini_layer("routed", T, d, E, I, k, I_s, dtype=dtype, norm=1, config_id=150 + CASES.index(case))
    layer = fm.Layer(d, E, I, k, I_s, dtype, 1, max_tokens=T)
    layer.set_weights(*[fm.to_device(a) if a is not None else None for a in (*w, *s)])
    rng = np.random.default_rng(T)
    keep = rng.integers(0, I + 1, E).astype(np.int32)
    keep[rng.integers(0, E)] = 0
    layer.set_budget(keep)
    return layer, x, lg, w, s, keep


def routing_of(ids, weights):
    return fm.Routing(fm.to_device(np.ascontiguousarray(ids, np.int32)), fm.to_device(np.ascontiguousarray(weights, np.float32)))


def reference(x, ids, weights, w, s, keep):
    """Slot by slot in 64 bits: ids outside [0, E), and those a token has already, add nothing."""
    X, (wg, wu, wd) = f64(x), [f64(a) for a in w]
    Y = np.zeros_like(X)
    if s[0] is not None:
        sg, su, sd = [f64(a) for a in s]
        Y += (silu(X @ sg.T) * (X @ su.T)) @ sd.T
    for t in range(len(X)):
        seen = set()
        for e, v in zip(ids[t], weights[t]):
            if 0 <= e < len(wg) and e not in seen:
                seen.add(e)
                n = keep[e]
                Y[t] += float(v) * ((silu(wg[e, :n] @ X[t]) * (wu[e, :n] @ X[t])) @ wd[e, :, :n].T)
    return Y


@pytest.mark.parametrize("case", CASES)
def test_own_routing_given_back(case):
    T, d, E, I, k = case[:5]
    say("routed", case)
    layer, x, lg, *_ = layer_of(case)
    xd, ld = fm.to_device(x), fm.to_device(lg)
    dbg = dict(topk_idx=torch.empty(T, k, dtype=torch.int32, device="cuda"), topk_w=torch.empty(T, k, device="cuda"))
    y = layer.forward(xd, ld, dbg=dbg)
    again = layer.forward(xd, routing=fm.Routing(dbg["topk_idx"], dbg["topk_w"]))
    assert torch.equal(y, again)


@pytest.mark.parametrize("case", CASES)
def test_slots_that_go_nowhere(case):
    T, d, E, I, k, I_s, dtype = case
    say("routed, holes", case)
    layer, x, _, w, s, keep = layer_of(case)
    rng = np.random.default_rng(5 * T)
    ids = np.stack([rng.permutation(E)[:k] for _ in range(T)]).astype(np.int32)
    ids[rng.random((T, k)) < 0.2] = -1
    bad = rng.random((T, k)) < 0.1
    ids[bad] = rng.choice(np.array([E, E + 7, -5, 2 ** 31 - 1, -2 ** 31], np.int64), bad.sum()).astype(np.int32)
    ids[:, -1] = np.where(rng.random(T) < 0.3, ids[:, 0], ids[:, -1])  # the same expert twice
    if T > 2:
        ids[T // 2] = -1
    weights = rng.normal(0.3, 0.3, (T, k)).astype(np.float32)
    xd, r = fm.to_device(x), routing_of(ids, weights)
    y = layer.forward(xd, routing=r)
    assert torch.equal(y, layer.forward(xd, routing=r))
    ref = reference(x, ids, weights, w, s, keep)
    got = y_to_f64(fm.to_host(y)).reshape(T, d)
    check_y(got, ref, BF16_TOL if dtype == synth.BF16 else F32_TOL)
    if T > 2 and not I_s:
        assert not got[T // 2].any()


@pytest.mark.parametrize("T", [3, 200])
def test_no_token_goes_anywhere(T):
    layer = fm.Layer(128, 16, 64, 2, 0, synth.BF16, 1, max_tokens=T)
    g = torch.Generator(device="cuda").manual_seed(1)
    layer.set_weights(*[torch.randn(16, a, b, generator=g, device="cuda").bfloat16() for a, b in ((64, 128), (64, 128), (128, 64))])
    x = torch.randn(T, 128, generator=g, device="cuda").bfloat16()
    y = layer.forward(x, routing=routing_of(np.full((T, 2), -1), np.ones((T, 2))), y=torch.full_like(x, 7.0))
    assert not bool(y.any())


@pytest.mark.parametrize("T", [8, 300])
def test_clipped_weights(T):
    d, E, I, k = 256, 8, 320, 2
    cfg, x, lg, w, s = mini_layer("routed", T, d, E, I, k, 0, dtype=synth.BF16, norm=1, config_id=170)
    layer = fm.Layer(d, E, I, k, 0, synth.BF16, 1, max_tokens=T)
    layer.set_weights(*[fm.to_device(a) for a in w])
    keep = np.array([40, 0, 320, 9, 16, 100, 7, 64], np.int32)
    layer.set_budget(keep)
    cw = layer.export_clipped(keep)
    r = fm.Router(E, k, T).route(fm.to_device(lg))
    r.topk_idx[0, 0] = -1
    xd = fm.to_device(x)
    assert torch.equal(layer.forward(xd, routing=r), layer.forward(xd, routing=r, clipped=cw))


@pytest.mark.parametrize("T", [1, 40, 500])
def test_a_router_with_groups_before_the_layer(T):
    d, E, I, k, dtype = 128, 32, 72, 4, synth.BF16
    cfg, x, lg, w, s = mini_layer("routed", T, d, E, I, k, 64, dtype=dtype, norm=1, config_id=171)
    layer = fm.Layer(d, E, I, k, 64, dtype, 1, max_tokens=T)
    layer.set_weights(*[fm.to_device(a) for a in (*w, *s)])
    bias = torch.linspace(-0.1, 0.1, E, device="cuda")
    bias[3] = float("-inf")
    logits = fm.to_device(lg)
    logits[T // 2] = float("-inf")  # padding
    router = fm.Router(E, k, T, score="sigmoid", scale=2.5, groups=8, top_groups=3, group_best=2)
    r = router.route(logits, bias, tables=False)
    assert not bool((r.topk_idx == 3).any()) and bool((r.topk_idx[T // 2] == -1).all())
    y = layer.forward(fm.to_device(x), routing=r)
    ref = reference(x, r.topk_idx.cpu().numpy(), r.topk_w.cpu().numpy(), w, s, np.full(E, I))
    check_y(y_to_f64(fm.to_host(y)).reshape(T, d), ref, BF16_TOL)


def test_captured():
    case = CASES[4]
    layer, x, lg, *_ = layer_of(case)
    T, E, k = case[0], case[2], case[4]
    xd, ld, router = fm.to_device(x), fm.to_device(lg), fm.Router(case[2], k, T)
    y = torch.empty(T, case[1], dtype=torch.bfloat16, device="cuda")

    def step():
        layer.forward(xd, routing=router.route(ld), y=y)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        ld.copy_(fm.to_device(np.roll(lg, i, 1)))
        y.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, y)
