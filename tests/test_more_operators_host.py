"""Refusals of routing, norms, log probabilities and distillation: every bad argument is reported on the host, before any
device work (no call here reaches a kernel launch)."""
import pytest

torch = pytest.importorskip("torch")
from paper_2606_27866_amd import flexmoe as fm  # noqa: E402

FAKE = 0x100000  # never dereferenced


def code_of(f, *args, **kw):
    with pytest.raises(fm.FlexMoEError) as ei:
        f(*args, **kw)
    assert fm.flexmoe_last_error()
    return ei.value.code


# ---- routing ----------------------------------------------------------------
def router(**kw):
    a = dict(E=16, top_k=2, max_tokens=100)
    a.update(kw)
    return fm.make_router_desc(**a)


OUT = dict(topk_idx=FAKE, topk_w=FAKE, counts=FAKE, offsets=FAKE, perm=FAKE, pos=FAKE)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=4), -5), (dict(E=0), -2), (dict(E=257), -2), (dict(top_k=0), -2), (dict(top_k=17), -2), (dict(E=1), -2),
    (dict(normalize=2), -1), (dict(groups=0), -2), (dict(groups=3), -2), (dict(E=130, groups=65), -2), (dict(groups=4, top_groups=0), -2),
    (dict(groups=4, top_groups=5), -2), (dict(top_k=5, groups=4, top_groups=1), -2), (dict(group_best=0), -2), (dict(group_best=3), -2),
    (dict(groups=16, top_groups=2, group_best=2), -2), (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1), (dict(max_tokens=-1), -2),
    (dict(max_tokens=1 << 29), -2), (dict(ldl=15), -2), (dict(ldl=(1 << 21) + 1), -2)])
def test_router_descriptor(kw, code):
    D = router(**kw)
    assert code_of(fm.flexmoe_route_workspace_bytes, D, 1) == -2
    assert code_of(fm.flexmoe_route, D, 1, FAKE, None, OUT, FAKE, 1 << 30, 0) == code
    assert code_of(fm.flexmoe_route_backward, D, 1, FAKE, FAKE, FAKE, FAKE, 0, 0) == code


def test_router_score_out_of_range():
    D = router()
    D.score = 2
    assert code_of(fm.flexmoe_route, D, 1, FAKE, None, OUT, FAKE, 1 << 30, 0) == -1
    with pytest.raises(ValueError, match="score"):
        fm.Router(16, 2, 10, score="relu", device="cpu")


def test_router_arguments():
    def call(T=50, logits=FAKE, bias=None, ws=FAKE, nbytes=1 << 30, **out):
        fm.flexmoe_route(router(), T, logits, bias, dict(OUT, **out), ws, nbytes, 0)

    for kw, code in [(dict(T=-1), -1), (dict(T=101), -2), (dict(logits=None), -1), (dict(topk_idx=None), -1), (dict(topk_w=None), -1),
                     (dict(counts=None), -1), (dict(offsets=None), -1), (dict(perm=None), -1), (dict(pos=None), -1), (dict(logits=FAKE + 2), -1),
                     (dict(bias=FAKE + 2), -1), (dict(topk_idx=FAKE + 1), -1), (dict(pos=FAKE + 2), -1), (dict(ws=None), -4), (dict(nbytes=100), -4),
                     (dict(ws=FAKE + 16), -4)]:
        assert code_of(call, **kw) == code, kw
    fm.flexmoe_route(router(), 0, None, None, {}, None, 0, 0)  # nothing to do

    def back(T=50, logits=FAKE, idx=FAKE, dw=FAKE, dl=FAKE, lddl=0):
        fm.flexmoe_route_backward(router(), T, logits, idx, dw, dl, lddl, 0)

    for kw, code in [(dict(T=-1), -1), (dict(T=101), -2), (dict(logits=None), -1), (dict(idx=None), -1), (dict(dw=None), -1), (dict(dl=None), -1),
                     (dict(lddl=15), -2), (dict(dl=FAKE + 2), -1), (dict(idx=FAKE + 2), -1)]:
        assert code_of(back, **kw) == code, kw
    back(T=0)


def test_router_tensors():
    r = fm.Router(16, 2, 10, device="cpu")
    ok = torch.zeros(4, 16)
    for bad in (ok[0], ok[:, :8], ok.half(), ok):  # the last is not on the GPU
        with pytest.raises(ValueError):
            r.route(bad)
    with pytest.raises(ValueError):
        r.backward(ok, torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2))


# ---- norm -------------------------------------------------------------------
def norm(**kw):
    a = dict(cols=64, max_rows=100)
    a.update(kw)
    return fm.make_norm_desc(**a)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=3), -5), (dict(w_dtype=-1), -5), (dict(cols=0), -2), (dict(cols=(1 << 21) + 8), -2), (dict(max_rows=-1), -2),
    (dict(max_rows=(1 << 30) + 1), -2), (dict(eps=0.0), -1), (dict(eps=1e-31), -1), (dict(eps=2.0), -1), (dict(eps=float("nan")), -1),
    (dict(cols=60), -2), (dict(ldx=56), -2), (dict(ldx=68), -2), (dict(ldres=70), -2), (dict(ldr=60), -2), (dict(ldy=(1 << 21) + 8), -2)])
def test_norm_descriptor(kw, code):
    D = norm(**kw)
    assert code_of(fm.flexmoe_rms_norm_workspace_bytes, D, 1) == -2
    assert code_of(fm.flexmoe_rms_norm, D, 1, FAKE, None, FAKE, None, FAKE, None, None, None, 0) == code
    assert code_of(fm.flexmoe_rms_norm_backward, D, 1, FAKE, FAKE, FAKE, FAKE, None, FAKE, FAKE, 0, FAKE, 1 << 30, 0) == code


def test_norm_arguments():
    at = dict(zip("x residual w r y q scale rstd".split(), [FAKE + 4096 * i for i in range(8)]))

    def call(rows=10, D=norm(), **kw):
        a = dict(at, **kw)
        fm.flexmoe_rms_norm(D, rows, a["x"], a["residual"], a["w"], a["r"], a["y"], a["q"], a["scale"], a["rstd"], 0)

    for kw, code in [(dict(rows=-1), -1), (dict(rows=101), -2), (dict(x=None), -1), (dict(w=None), -1), (dict(y=None, q=None, scale=None), -1),
                     (dict(scale=None), -1), (dict(q=None), -1), (dict(r=None), -1), (dict(residual=None), -1), (dict(x=FAKE + 8), -1),
                     (dict(r=FAKE + 2), -1), (dict(w=FAKE + 4), -1), (dict(scale=FAKE + 2), -1), (dict(rstd=FAKE + 1), -1),
                     (dict(D=norm(ldq=72)), -2), (dict(D=norm(ldq=48)), -2), (dict(y=at["x"]), -1), (dict(y=at["residual"]), -1),
                     (dict(y=at["r"]), -1)]:
        assert code_of(call, **kw) == code, kw
    call(rows=0, x=None)

    def back(rows=10, dy=FAKE, r=FAKE, w=FAKE, rstd=FAKE, dr=None, dx=FAKE, dw=FAKE, accumulate=0, ws=FAKE, nbytes=1 << 30):
        fm.flexmoe_rms_norm_backward(norm(), rows, dy, r, w, rstd, dr, dx, dw, accumulate, ws, nbytes, 0)

    for kw, code in [(dict(rows=-1), -1), (dict(rows=101), -2), (dict(dy=None), -1), (dict(r=None), -1), (dict(w=None), -1), (dict(rstd=None), -1),
                     (dict(dx=None), -1), (dict(accumulate=2), -1), (dict(dr=FAKE + 8), -1), (dict(dw=FAKE + 2), -1), (dict(ws=None), -4),
                     (dict(nbytes=255), -4), (dict(ws=FAKE + 128), -4)]:
        assert code_of(back, **kw) == code, kw
    back(rows=0, dw=None, ws=None, nbytes=0)


def test_norm_workspace_serves_fewer_rows():
    for cols in (8, 512, 2048, 2056, 40000):
        sizes = [fm.flexmoe_rms_norm_workspace_bytes(norm(cols=cols, max_rows=1 << 20), n) for n in (0, 1, 255, 1023, 1024, 1030, 5000, 1 << 20)]
        assert sizes == sorted(sizes) and sizes[0] >= 256


def test_norm_tensors():
    n = fm.RMSNorm(torch.ones(64), 10)
    x = torch.zeros(4, 64)
    for bad in (x[0], x[:, :32], x.half(), x):  # the last is not on the GPU
        with pytest.raises(ValueError):
            n.forward(bad)
    with pytest.raises(ValueError, match="residual"):
        n.forward(x, r=x)
    with pytest.raises(ValueError, match="accumulate"):
        n.backward(x, x, torch.zeros(4), accumulate=True)
    with pytest.raises(ValueError, match="weight_grad"):
        n.backward(x, x, torch.zeros(4), dw=torch.zeros(64), weight_grad=False)
    with pytest.raises(ValueError, match="dimension"):
        fm.RMSNorm(torch.ones(1, 64), 10)


# ---- log probabilities --------------------------------------------------------
def logprobs(**kw):
    a = dict(V=1000, top=8, max_rows=100)
    a.update(kw)
    return fm.make_logprob_desc(**a)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), -5), (dict(V=0), -2), (dict(V=(1 << 21) + 8), -2), (dict(top=-1), -2), (dict(top=129), -2), (dict(V=8, top=9), -2),
    (dict(max_rows=-1), -2), (dict(max_rows=(1 << 24) + 1), -2), (dict(V=1001), -2), (dict(ld=992), -2), (dict(ld=1004), -2), (dict(ld=(1 << 22) + 8), -2),
    (dict(temperature=0.0), -1), (dict(temperature=-1.0), -1), (dict(temperature=1e7), -1), (dict(temperature=float("nan")), -1)])
def test_logprobs_descriptor(kw, code):
    D = logprobs(**kw)
    assert code_of(fm.flexmoe_token_logprobs_workspace_bytes, D, 1) == -2
    assert code_of(fm.flexmoe_token_logprobs, D, 1, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 30, 0) == code


def test_logprobs_arguments():
    def call(rows=10, D=logprobs(V=20000), logits=FAKE, tokens=FAKE, logprob=FAKE, entropy=FAKE, lse=FAKE, ids=FAKE, top=FAKE, ws=FAKE, nbytes=1 << 30):
        fm.flexmoe_token_logprobs(D, rows, logits, tokens, logprob, entropy, lse, ids, top, ws, nbytes, 0)

    for kw, code in [(dict(rows=-1), -1), (dict(rows=101), -2), (dict(logits=None), -1), (dict(tokens=None), -1), (dict(logprob=None), -1),
                     (dict(entropy=None), -1), (dict(lse=None), -1), (dict(ids=None), -1), (dict(top=None), -1), (dict(D=logprobs(top=0)), -1),
                     (dict(logits=FAKE + 8), -1), (dict(tokens=FAKE + 2), -1), (dict(top=FAKE + 1), -1), (dict(ws=None), -4), (dict(nbytes=300), -4),
                     (dict(ws=FAKE + 64), -4)]:
        assert code_of(call, **kw) == code, kw
    call(rows=0, logits=None)


def test_logprobs_workspace_serves_fewer_rows():
    for V in (100, 5000, 131072, 300000):
        sizes = [fm.flexmoe_token_logprobs_workspace_bytes(logprobs(V=V, ld=1 << 21, max_rows=1 << 20), n) for n in (0, 1, 2, 9, 64, 511, 512, 513, 5000, 1 << 20)]
        assert sizes == sorted(sizes) and sizes[0] >= 256


def test_logprobs_tensors():
    h = fm.TokenLogprobs(64, 10, top=3, device="cpu")
    x = torch.zeros(4, 64)
    for bad in (x[0], x[:, :32], x.half(), x):  # the last is not on the GPU
        with pytest.raises(ValueError):
            h(bad)


# ---- distillation -------------------------------------------------------------
def distill(**kw):
    a = dict(V=1000, top=8, max_rows=100)
    a.update(kw)
    return fm.make_distill_desc(**a)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), -5), (dict(V=0), -2), (dict(V=(1 << 21) + 8), -2), (dict(top=0), -2), (dict(top=129), -2), (dict(max_rows=-1), -2),
    (dict(max_rows=(1 << 24) + 1), -2), (dict(V=1001), -2), (dict(ld=992), -2), (dict(ldd=1004), -2), (dict(ldd=(1 << 22) + 8), -2),
    (dict(temperature=0.0), -1), (dict(temperature=float("inf")), -1), (dict(tail=2), -1), (dict(kl_weight=float("nan")), -1),
    (dict(ce_weight=float("inf")), -1)])
def test_distill_descriptor(kw, code):
    D = distill(**kw)
    assert code_of(fm.flexmoe_distill_workspace_bytes, D, 1) == -2
    assert code_of(fm.flexmoe_distill, D, 1, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 40, 0) == code


def test_distill_arguments():
    def call(rows=10, D=distill(), logits=FAKE, ids=FAKE, lp=FAKE, labels=None, scale=None, kl=FAKE, ce=FAKE, d=None, ws=FAKE, nbytes=1 << 30):
        fm.flexmoe_distill(D, rows, logits, ids, lp, labels, scale, kl, ce, d, ws, nbytes, 0)

    for kw, code in [(dict(rows=-1), -1), (dict(rows=101), -2), (dict(logits=None), -1), (dict(ids=None), -1), (dict(lp=None), -1),
                     (dict(kl=None), -1), (dict(ce=None), -1), (dict(logits=FAKE + 8), -1), (dict(d=FAKE + 4), -1), (dict(ids=FAKE + 2), -1),
                     (dict(labels=FAKE + 2), -1), (dict(scale=FAKE + 1), -1), (dict(d=FAKE, D=distill(ldd=1008)), -1), (dict(ws=None), -4),
                     (dict(nbytes=300), -4), (dict(ws=FAKE + 64), -4)]:
        assert code_of(call, **kw) == code, kw
    call(rows=0, logits=None)


def test_distill_workspace_serves_fewer_rows():
    for V in (100, 5000, 131072, 300000):
        sizes = [fm.flexmoe_distill_workspace_bytes(distill(V=V, ld=1 << 21, ldd=1 << 21, max_rows=1 << 20), n)
                 for n in (0, 1, 2, 9, 64, 511, 512, 513, 5000, 1 << 20)]
        assert sizes == sorted(sizes) and sizes[0] >= 256


def test_distill_tensors():
    h = fm.Distillation(64, 3, 10, device="cpu")
    x, ids, lp = torch.zeros(4, 64), torch.zeros(4, 3, dtype=torch.int32), torch.zeros(4, 3)
    for bad in (x[0], x[:, :32], x.half(), x):  # the last is not on the GPU
        with pytest.raises(ValueError):
            h.forward(bad, ids, lp)


def test_outputs_made_together_and_apart():
    make, like = fm.tensors().make, torch.zeros(1)
    pieces = ((0, 5), (1, 3, 5, 8), (3, 0), (3, 0, 4, 4), (2, 3), (4, 7, 10, 16))
    for together in (True, False):
        made = make(like, pieces, together)
        assert [tuple(t.shape) for t in made] == [(5,), (3, 5), (0,), (0, 4), (3,), (7, 10)]
        assert [t.dtype for t in made] == [torch.float32, torch.bfloat16, torch.int32, torch.int32, torch.uint8, torch.int8]
        assert [t.stride() for t in made] == [(1,), (8, 1), (1,), (4, 1), (1,), (16, 1)]
        storages = {t.untyped_storage().data_ptr() for t in made if t.numel()}
        assert len(storages) == (1 if together else 4)
        for i, t in enumerate(made):
            t.fill_(i)
        assert all(bool((t == i).all()) for i, t in enumerate(made))
    assert make(like, (), True) == ()
    for together in (True, False):
        at = (fm.ctypes.c_void_p * 3)(7, 7, 7)
        made = make(like, ((3, 2, 4, 4), (0, 5)), together, fm.ctypes.addressof(at))
        assert [at[i] for i in range(3)] == [made[0].data_ptr(), made[1].data_ptr(), 7]
    for bad in [(like,), (like, ((5, 1),), 1), (like, ((0, 1, 3, 2),), 1), (like, ((0, 1, 3),), 1), (None, (), 1), (like, [], 1),
                (like, ((0, -1),), 1), (like, ((0, "1"),), 1), (like, ((0, 1 << 31, 1 << 31, 1 << 31),), 1), (like, ((0, 1),) * 17, 1)]:
        with pytest.raises(TypeError):
            make(*bad)


# ---- the forward with a caller's routing ---------------------------------------
def test_routed_forward_arguments():
    D = fm.make_desc(64, 8, 40, 2, 0, fm.FLEXMOE_BF16, 1, 100)

    def call(T=10, x=FAKE, ids=FAKE, w=FAKE, keep=FAKE, packed=-1, y=FAKE, ws=FAKE, nbytes=1 << 30, shared=None):
        fm.flexmoe_layer_forward_routed(D, T, x, ids, w, FAKE, FAKE, FAKE, keep, packed, shared, shared, shared, y, ws, nbytes, 0)

    for kw, code in [(dict(T=-1), -1), (dict(T=101), -2), (dict(x=None), -1), (dict(ids=None), -1), (dict(w=None), -1), (dict(keep=None), -1),
                     (dict(y=None), -1), (dict(packed=-2), -1), (dict(packed=8 * 40 + 8), -1), (dict(ids=FAKE + 2), -1), (dict(w=FAKE + 1), -1),
                     (dict(x=FAKE + 8), -1), (dict(keep=FAKE + 2), -1), (dict(ws=None), -4), (dict(nbytes=64), -4), (dict(ws=FAKE + 8), -4),
                     (dict(shared=FAKE), -1)]:
        assert code_of(call, **kw) == code, kw
    call(T=0, x=None, ids=None, w=None)  # nothing to do


def test_layer_takes_logits_or_routing():
    layer = fm.Layer(64, 8, 40, 2, device="cpu")
    x, logits, r = torch.zeros(1, 64, dtype=torch.bfloat16), torch.zeros(1, 8), fm.Routing(torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, 2))
    for kw in [dict(), dict(logits=logits, routing=r), dict(routing=r, dbg={}), dict(routing=r, bucketed=([40] * 8, 8)),
               dict(routing=r), dict(routing=r._replace(topk_idx=torch.zeros(1, 2, dtype=torch.int64)))]:
        with pytest.raises(ValueError):
            layer.forward(x, **kw)
