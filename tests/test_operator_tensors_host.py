"""What the holders of the experts' products, the 8-bit products and AdamW take from a tensor, without a GPU: CPU tensors
that say they are on one (no call here reaches a kernel launch)."""
import pytest

torch = pytest.importorskip("torch")
from paper_2606_27866_amd import flexmoe as fm  # noqa: E402

BF, F32, I8 = torch.bfloat16, torch.float32, torch.int8


class OnGpu(torch.Tensor):
    is_cuda = property(lambda self: True)


def on_gpu(t):
    return t.as_subclass(OnGpu)


@pytest.fixture
def no_launch(monkeypatch):
    """Any call of the library fails: what is refused must be refused before it."""
    class Library:
        def __getattr__(self, name):
            def called(*_):
                raise AssertionError("reached " + name)
            return called

    monkeypatch.setattr(fm, "lib", Library)


def expanded(*shape, dtype=BF, over=0):
    """A tensor that repeats one slice along dimension `over` with stride 0, as the gradient of a sum is."""
    one = [1 if i == over else n for i, n in enumerate(shape)]
    return on_gpu(torch.zeros(one, dtype=dtype).expand(shape))


def test_the_gradient_of_a_sum_is_an_expanded_tensor():
    y = torch.zeros(10, 64, requires_grad=True)
    z, seen = y * 1, []
    z.register_hook(seen.append)
    z.sum(0).backward(torch.ones(64))
    assert seen[0].stride() == (0, 1)


@pytest.mark.parametrize("t", [expanded(10, 64), expanded(10, 64, dtype=F32), expanded(10, 64, dtype=I8), expanded(10, 1),
                               expanded(3, 4, 64, over=1), expanded(3, 1, 64), on_gpu(torch.zeros(3, 1, 64).expand(3, 4, 64)),
                               on_gpu(torch.zeros(1, 1, 64).expand(3, 4, 64)),
                               on_gpu(torch.zeros(100).as_strided((10, 64), (4, 1)))])
def test_rows_that_overlap_are_refused(t):
    with pytest.raises(ValueError):
        fm._matrix(t, tuple(t.shape), t.dtype, "x")


def test_rows_that_do_not_overlap_are_taken():
    for t, ld in [(torch.zeros(10, 64), 64), (torch.zeros(10, 72)[:, :64], 72), (torch.zeros(1, 64).expand(1, 64), 64), (torch.zeros(0, 64), 64),
                  (torch.zeros(3, 4, 64), 64), (torch.zeros(3, 1, 64), 64), (torch.zeros(3, 1, 72)[..., :64], 72), (torch.zeros(10, 8)[:, :1], 8)]:
        assert fm._matrix(on_gpu(t), tuple(t.shape), F32, "x") == ld


def test_products_refuse_expanded_tensors(request):
    E, N, K, R = 2, 16, 64, 10
    op = fm.GroupedProduct(E, N, K, R, device="cpu")
    request.getfixturevalue("no_launch")
    offsets = on_gpu(torch.zeros(E + 1, dtype=torch.int32))
    x, dy, w = (on_gpu(torch.zeros(s, dtype=BF)) for s in ((R, K), (R, N), (E, N, K)))
    for f, args in [(op.forward, (expanded(R, K), w, offsets)), (op.forward, (x, expanded(E, N, K, over=0), offsets)),
                    (op.forward, (x, expanded(E, N, K, over=1), offsets)), (op.input_grad, (expanded(R, N), w, offsets)),
                    (op.weight_grad, (expanded(R, N), x, offsets)), (op.weight_grad, (dy, expanded(R, K), offsets))]:
        with pytest.raises(ValueError, match="overlap|one after another"):
            f(*args)
    with pytest.raises(ValueError):
        op.forward(x, w, offsets, y=expanded(R, N))
    with pytest.raises(ValueError):
        op.weight_grad(dy, x, offsets, dw=expanded(E, N, K, dtype=F32, over=1), accumulate=True)


def test_rounded_rows_refuse_expanded_tensors(no_launch):
    x = on_gpu(torch.zeros(10, 64))
    for kw in (dict(x=expanded(10, 64, dtype=F32)), dict(x=x, gate=expanded(10, 64, dtype=F32)), dict(x=x, q=expanded(10, 64, dtype=I8)),
               dict(x=expanded(10, 64, dtype=F32), gate=expanded(10, 64, dtype=F32))):
        with pytest.raises(ValueError, match="overlap"):
            fm.quantize_rows(**kw)


def test_every_leading_stride_of_a_stack_is_checked():
    """Stacks of any number of dimensions whose rows follow each other at one distance, and no others."""
    z = torch.zeros
    for t, ld in [(z(2, 3, 8, 16), 16), (z(2, 3, 8, 24)[..., :16], 24), (z(2, 3, 1, 16), 16), (z(2, 1, 8, 16)[:, :, :, :], 16),
                  (z(1, 3, 8, 16), 16), (z(4, 2, 3, 8, 16), 16), (z(5, 1, 1, 24)[..., :16], 24), (z(1, 1, 16), 16), (z(2, 1, 1, 1, 16), 16),
                  (z(2, 8, 16)[:, :8], 16), (z(3, 8, 16)[1:], 16)]:
        assert fm._matrix(on_gpu(t), tuple(t.shape), F32, "x") == ld, t.shape
    for t in [z(2, 3, 8, 16)[:, :, :4], z(2, 3, 8, 16)[:, :2], z(3, 2, 8, 16).transpose(0, 1), z(2, 8, 3, 16).transpose(1, 2), z(4, 8, 16)[::2],
              z(2, 3, 1, 16)[:, :2], z(2, 1, 16).expand(2, 3, 16), z(2, 1, 8, 16).expand(2, 3, 8, 16), z(2, 2, 3, 8, 16)[:, :, :2]]:
        with pytest.raises(ValueError):
            fm._matrix(on_gpu(t), tuple(t.shape), F32, "x")


def test_a_row_alone_is_no_matrix(no_launch):
    with pytest.raises(ValueError):
        fm.quantize_rows(on_gpu(torch.zeros(16)))


class Recorder:
    """Stands for the library: writes down the arguments of every call."""

    def __init__(self, real):
        self.real, self.calls = real, []

    def __getattr__(self, name):
        if name.endswith("_bytes"):
            return getattr(self.real, name)

        def call(*args):
            self.calls.append((name, args))
            return 0
        return call


@pytest.fixture
def recorder(monkeypatch):
    r = Recorder(fm.lib())
    monkeypatch.setattr(fm, "lib", lambda: r)
    return r


def test_a_dense_call_keeps_no_temporary_offsets(recorder, monkeypatch):
    """One group without offsets: every call passes the holder's own, which stay while the holder does; nothing is made on
    the current stream for work on another, nothing copied from the host."""
    op = fm.Int8Product(on_gpu(torch.zeros(1, 32, 64, dtype=I8)), on_gpu(torch.zeros(1, 32)), max_rows=8)

    def made(*_, **__):
        raise AssertionError("a tensor made during the call")

    monkeypatch.setattr(torch, "tensor", made)
    for R in (1, 5, 8):
        y = on_gpu(torch.zeros(R, 32, dtype=BF))
        op(on_gpu(torch.zeros(R, 64, dtype=BF)), y=y, stream=0)
        op.product(on_gpu(torch.zeros(R, 64, dtype=I8)), on_gpu(torch.zeros(R)), y=y, stream=0)
    used = {args[6] for name, args in recorder.calls if name == "flexmoe_quantized_forward"}
    assert len(recorder.calls) == 9 and len(used) == 1
    whole = [t for t in vars(op).values() if isinstance(t, torch.Tensor) and t.data_ptr() in used]
    assert len(whole) == 1 and whole[0].dtype == torch.int32
    assert whole[0].tolist()[0] == 0 and whole[0].tolist()[1] >= 8  # the kernels cut it to a call's rows


def test_several_groups_need_offsets(recorder):
    op = fm.Int8Product(on_gpu(torch.zeros(2, 32, 64, dtype=I8)), on_gpu(torch.zeros(2, 32)), max_rows=8)
    with pytest.raises(ValueError, match="offsets"):
        op(on_gpu(torch.zeros(3, 64, dtype=BF)), y=on_gpu(torch.zeros(3, 32, dtype=BF)), stream=0)


class Columns:
    """Stands for the native module: the same columns, of tensors that say they are on a GPU."""

    @staticmethod
    def columns(cols, count, stride):
        import ctypes
        for c, (tensors, sizes, code, dst, longer) in enumerate(cols):
            if len(tensors) != count:
                return c * (count + 1) + count
            n = (ctypes.c_int64 * count).from_address(sizes)
            for i, t in enumerate(tensors):
                if (not t.is_cuda or t.dtype != (F32, BF, torch.uint8)[code] or not t.is_contiguous()
                        or (t.numel() < n[i] if longer else t.numel() != n[i])):
                    return c * (count + 1) + i
                ctypes.c_void_p.from_address(dst + i * stride).value = t.data_ptr()
        return -1


@pytest.fixture
def steps(recorder, monkeypatch):
    """The tables that flexmoe_adamw_step was given."""
    monkeypatch.setattr(fm, "tensors", lambda: Columns)
    monkeypatch.setattr(fm, "_capturing", lambda: False)
    seen = []

    def step(desc, table, count, stream):
        assert not stream
        seen.append([{f: getattr(t, f) for f, _ in fm.flexmoe_adamw_tensor._fields_}
                     for t in (fm.flexmoe_adamw_tensor * count).from_address(table)])
        return 0

    recorder.flexmoe_adamw_step = step
    return seen


def adamw(bits=32, master=False):
    sizes = [300, 5]
    st = torch.uint8 if bits == 8 else F32

    def zeros(ns, dtype):
        return [on_gpu(torch.zeros(n, dtype=dtype)) for n in ns]

    p = zeros(sizes, BF if master else F32)
    states = (zeros(sizes, st), zeros(sizes, st)) + ((zeros([2, 1], F32), zeros([2, 1], F32)) if bits == 8 else ())
    opt = fm.AdamW(p, masters=zeros(sizes, F32) if master else None, states=states, state_bits=bits)
    return opt, zeros(sizes, F32)


@pytest.mark.parametrize("bits", [8, 32])
def test_adamw_follows_tensors_whose_storage_is_replaced(steps, bits):
    opt, grads = adamw(bits, master=True)
    lists = dict(param=opt.params, m=opt.m, v=opt.v, master=opt.masters)
    if bits == 8:
        lists.update(m_scale=opt.m_scale, v_scale=opt.v_scale)
    opt.step(grads, 1e-3, stream=0)
    kept = []
    for ts in lists.values():
        for t in ts:
            kept.append(t.data)  # the old storage stays, so that the new one is another
            t.data = on_gpu(torch.ones(t.shape, dtype=t.dtype))
    opt.step(grads, 1e-3, stream=0)
    for i in range(2):
        for field, ts in lists.items():
            assert steps[1][i][field] == ts[i].data_ptr() != steps[0][i][field]
        assert steps[1][i]["grad"] == grads[i].data_ptr() and steps[1][i]["n"] == grads[i].numel()


def test_adamw_refuses_tensors_that_no_longer_fit(steps):
    for field, bad in [("params", torch.zeros(299)), ("params", torch.zeros(301)), ("params", torch.zeros(300, dtype=BF)), ("m", torch.zeros(299)),
                       ("v", torch.zeros(600)[::2])]:
        opt, grads = adamw()
        getattr(opt, field)[0] = on_gpu(bad)
        with pytest.raises(ValueError):
            opt.step(grads, 1e-3, stream=0)
    opt, grads = adamw()
    opt.params.append(opt.params[0])  # the table has no place for it
    with pytest.raises(ValueError):
        opt.step(grads, 1e-3, stream=0)
    assert not steps and opt.t == 0


def test_native_columns_refuse_what_does_not_fit():
    import numpy as np
    table, sizes = np.zeros(4, np.uint64), np.array([3, 4], np.int64)
    f, p, at = fm.tensors().columns, sizes.ctypes.data, table.ctypes.data
    cpu = [torch.zeros(3), torch.zeros(4)]
    assert f(((cpu, p, 0, at, 0),), 2, 8) == 0               # not on the GPU
    assert f(((cpu[:1], p, 0, at, 0),), 2, 8) == 2           # another number of tensors
    assert f((([], p, 0, at, 0), (cpu, p, 0, at, 0)), 0, 8) == 1
    assert f((([None, None], p, 0, at, 1),), 2, 8) == 0
    assert not table.any()
    for bad in [((), 2), ([], 2, 8), ((), 2, 8), (((cpu, p, 0, at),), 2, 8), ((((), p, 0, at, 0),), 0, 8), (((cpu, p, "0", at, 0),), 2, 8)]:
        with pytest.raises(TypeError):
            f(*bad)


def test_adamw_clock_arguments(steps, recorder):
    p = on_gpu(torch.zeros(8))
    states = ([on_gpu(torch.zeros(8))], [on_gpu(torch.zeros(8))])
    opt = fm.AdamW([p], states=states, step=7, device_step=True)
    seen = []
    step = recorder.flexmoe_adamw_step
    recorder.flexmoe_adamw_step = lambda d, *rest: (seen.append(d._obj.clock), step(d, *rest))[1]
    opt.step([p], 1e-3, stream=0)
    assert seen == [opt.clock.data_ptr()] and opt.clock.numel() * 8 == 24
    assert opt.clock[0] == 7 and opt.t == 7  # the kernels count, not the holder


def test_adamw_refuses_a_misaligned_clock():
    D = fm.flexmoe_adamw_desc(0, 0, 32, 0, 0, 1e-3, 0.9, 0.99, 1e-8, 0.0, 1.0, 0x100004)
    assert fm.lib().flexmoe_adamw_step(fm.ctypes.byref(D), None, 0, None) == -1
    assert "clock" in fm.flexmoe_last_error()


def both(*calls):
    """The calls in turn in a thread each, many times at once; their exceptions."""
    import threading
    errors = []

    def loop(f):
        try:
            for _ in range(30):
                f()
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=loop, args=(f,)) for f in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    return errors


def test_threads_that_share_a_holder_keep_their_strides(recorder):
    """A call of the library runs without the interpreter's lock: another thread's strides must not reach its descriptor."""
    import time
    E, N, K, R = 2, 16, 64, 10
    op = fm.GroupedProduct(E, N, K, R, device="cpu")
    w, offsets = on_gpu(torch.zeros(E, N, K, dtype=BF)), on_gpu(torch.zeros(E + 1, dtype=torch.int32))
    xs = [on_gpu(torch.zeros(R, ld, dtype=BF)[:, :K]) for ld in (64, 72)]
    ys = [on_gpu(torch.zeros(R, ld, dtype=BF)[:, :N]) for ld in (16, 40)]
    want = {x.data_ptr(): (x.stride(0), y.stride(0)) for x, y in zip(xs, ys)}

    def forward(desc, rows, x, *_):
        d = desc._obj
        before = d.ldx, d.ldy
        time.sleep(0.0005)
        assert before == (d.ldx, d.ldy) == want[x]
        return 0

    recorder.flexmoe_grouped_forward = forward
    assert not both(*[lambda x=x, y=y: op.forward(x, w, offsets, y=y, stream=0) for x, y in zip(xs, ys)])


def test_threads_that_share_an_int8_holder_keep_their_rows(recorder):
    """The rounded rows lie in the holder's buffer until the product is launched."""
    import time
    op = fm.Int8Product(on_gpu(torch.zeros(1, 32, 64, dtype=I8)), on_gpu(torch.zeros(1, 32)), max_rows=8)
    xs = [on_gpu(torch.zeros(R, 64, dtype=BF)) for R in (3, 5)]
    ys = [on_gpu(torch.zeros(x.shape[0], 32, dtype=BF)) for x in xs]
    held = []

    def quantize(rows, *_):
        held.append(rows)
        time.sleep(0.0005)
        return 0

    def product(desc, rows, *_):
        assert held.pop() == rows and not held
        time.sleep(0.0005)
        return 0

    recorder.flexmoe_quantize_rows, recorder.flexmoe_quantized_forward = quantize, product
    assert not both(*[lambda x=x, y=y: op(x, y=y, stream=0) for x, y in zip(xs, ys)])


def test_threads_that_share_an_optimizer_keep_their_gradients(steps, recorder):
    import threading
    import time
    opt, one = adamw()
    two = [on_gpu(torch.ones_like(g)) for g in one]
    step, own = recorder.flexmoe_adamw_step, {}

    def slow(*args):
        time.sleep(0.0005)
        step(*args)
        assert [t["grad"] for t in steps[-1]] == own[threading.get_ident()]
        return 0

    def call(grads):
        own[threading.get_ident()] = [g.data_ptr() for g in grads]
        opt.step(grads, 1e-3, stream=0)

    recorder.flexmoe_adamw_step = slow
    assert not both(lambda: call(one), lambda: call(two))
    assert len(steps) == opt.t == 60


def test_layer_holders_refuse_what_is_not_packed(request):
    """The layer's calls take addresses alone: an expanded gradient, a transposed batch or one row too few would be read past
    its end or in the wrong places."""
    d, E, I, T, K = 16, 4, 24, 6, 3
    layer = fm.Layer(d, E, I, 2, max_tokens=T, device="cpu")
    layer.set_weights(torch.zeros(E, I, d, dtype=BF), torch.zeros(E, I, d, dtype=BF), torch.zeros(E, d, I, dtype=BF))
    sal = fm.Saliency(layer, T, transpose_once=False)
    act = fm.ActionLearner(layer, T, [0.5, 0.75, 1.0])
    recorder = request.getfixturevalue("recorder")
    x, logits, y = torch.zeros(T, d, dtype=BF), torch.zeros(T, E), torch.zeros(T, d, dtype=BF)
    dy, alpha, mask = torch.zeros(T, d), torch.zeros(E, K), torch.zeros(E, I)
    act.T = T
    good = {"forward": (layer.forward, [x, logits, y]), "saliency": (sal.add_batch, [x, logits, y]), "train": (act.forward, [x, logits, y]),
            "backward": (act.backward, [logits, dy]), "sample": (act.sample, [alpha, alpha]),
            "action_grad": (act.action_grad, [alpha, alpha, 1.0, 0.1, 0.0, mask])}
    for f, args in good.values():
        f(*args, stream=0)
    calls = len(recorder.calls)
    assert calls == len(good)
    for f, args in good.values():
        for i, t in enumerate(args):
            if not isinstance(t, torch.Tensor):
                continue
            for bad in (t[:1].expand(t.shape), t.T.contiguous().T, torch.cat([t, t], 1)[:, :t.shape[1]], t[:, 1:].contiguous()):
                with pytest.raises(ValueError):
                    f(*args[:i], bad, *args[i + 1:], stream=0)
    assert len(recorder.calls) == calls
