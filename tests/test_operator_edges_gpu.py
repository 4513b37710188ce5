"""Calls at the edges of the experts' products, the 8-bit products and AdamW: stacks, whole tensors without offsets, streams,
graphs, threads, moved storages, very small values, and every kind of tiles in one part and in several."""
import math

import pytest

torch = pytest.importorskip("torch")
from paper_2606_27866_amd import flexmoe as fm  # noqa: E402

pytestmark = pytest.mark.gpu
BF, F32, I8 = torch.bfloat16, torch.float32, torch.int8


@pytest.mark.parametrize("shape", [(2, 3, 8, 16), (2, 1, 5, 24), (1, 4, 1, 40), (2, 2, 2, 3, 9)])
def test_rounded_rows_of_a_stack(shape):
    g = torch.Generator(device="cuda")
    x = fm._padded(shape, F32, "cuda")
    x.copy_(torch.randn(shape, generator=g, device="cuda"))
    q, s = fm.quantize_rows(x)
    flat = fm._padded((x.numel() // shape[-1], shape[-1]), F32, "cuda")
    flat.copy_(x.reshape(flat.shape))
    qf, sf = fm.quantize_rows(flat)
    assert q.shape == shape and s.shape == shape[:-1]
    assert torch.equal(q.reshape(qf.shape), qf) and torch.equal(s.reshape(-1), sf)


def dense(N=200, K=336, max_rows=300):
    g = torch.Generator(device="cuda")
    op = fm.Int8Product.from_weights(torch.randn(1, N, K, generator=g, device="cuda"), max_rows, out_dtype=F32)
    return op, torch.randn(max_rows, K, generator=g, device="cuda").to(BF)


@pytest.mark.parametrize("T", [1, 33, 130, 300])
def test_dense_call_without_offsets(T):
    """The bits of the call with offsets; rows past T are left alone."""
    op, x = dense()
    want = op(x[:T], torch.tensor([0, T], dtype=torch.int32, device="cuda"))
    y = torch.full((300, 200), 7.0, device="cuda")
    op(x[:T], y=y[:T])
    assert torch.equal(y[:T], want) and bool((y[T:] == 7).all())
    assert torch.equal(op.product(op.q[:T], op.q_scale[:T]), want)


def test_dense_call_on_another_stream():
    """Work that follows on the current stream takes memory freed by the call: what the call reads is not among it."""
    op, x = dense()
    want = op(x)
    y = torch.zeros_like(want)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    busy = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(4):
            busy = (busy @ busy).clamp_(-1, 1)  # the call's kernels wait behind these
    op(x, y=y, stream=s)
    for _ in range(64):
        torch.zeros(2, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    assert torch.equal(y, want)


def test_dense_call_in_a_graph():
    op, x = dense()
    want = op(x)
    y = torch.zeros_like(want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op(x, y=y)
    for _ in range(3):
        y.fill_(-1.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
        op(x.neg())  # eager work in between


@pytest.mark.parametrize("bits", [8, 32])
def test_adamw_steps_the_storage_that_a_parameter_has_now(bits):
    g = torch.Generator(device="cuda")
    p = torch.randn(1000, generator=g, device="cuda")
    q, grad = p.clone(), torch.randn(1000, generator=g, device="cuda")
    a, b = fm.AdamW([p], state_bits=bits, seed=3), fm.AdamW([q], state_bits=bits, seed=3)
    a.step([grad], 1e-2)
    b.step([grad], 1e-2)
    old, m = p.data, a.m[0].data
    before = old.clone(), m.clone()
    p.data, a.m[0].data = p.data.clone(), a.m[0].data.clone()
    a.step([grad], 1e-2)
    b.step([grad], 1e-2)
    assert torch.equal(p, q) and torch.equal(a.m[0], b.m[0])
    assert torch.equal(old, before[0]) and torch.equal(m, before[1])  # nothing was written to the storages it had


@pytest.mark.parametrize("bits", [8, 32])
def test_a_captured_adamw_step_that_counts_on_the_device(bits):
    """Replays and eager calls in turn are the steps of an optimizer that counts on the host, bit for bit: each has its own
    bias corrections and its own random bits."""
    g = torch.Generator(device="cuda")
    sizes = [3000, 257] * 40  # two launches
    p = [torch.randn(n, generator=g, device="cuda") for n in sizes]
    q, grads = [t.clone() for t in p], [torch.randn(n, generator=g, device="cuda") for n in sizes]
    a = fm.AdamW(p, state_bits=bits, seed=3, weight_decay=0.1, device_step=True)
    b = fm.AdamW(q, state_bits=bits, seed=3, weight_decay=0.1)
    a.step(grads, 1e-2)
    b.step(grads, 1e-2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step(grads, 1e-2)
    for k in range(4):
        for t in grads:
            t.mul_(0.9)
        graph.replay()
        b.step(grads, 1e-2)
        if k == 1:
            a.step(grads, 1e-2)
            b.step(grads, 1e-2)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(p + a.m + a.v, q + b.m + b.v))
    assert int(a.clock[0]) == b.t == 6


def test_replays_that_count_on_the_device_keep_the_mean():
    """A constant gradient through replays of one captured step: the 8-bit states reach it, as those of separate calls do."""
    n = 4096
    g = torch.full((n,), 0.02, device="cuda")
    g[::256] = 0.05
    opt = fm.AdamW([torch.zeros(n, device="cuda")], state_bits=8, betas=(0.9, 0.99), seed=9, device_step=True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step([g], 0.0)
    for _ in range(600):
        graph.replay()
    m, v = fm.adamw_state_values(opt.m[0], opt.v[0], opt.m_scale[0], opt.v_scale[0])
    rest = torch.ones(n, dtype=torch.bool, device="cuda")
    rest[::256] = False
    assert abs(float(m[rest].mean()) / 0.02 - 1) < 0.02
    assert abs(float(v[rest].mean()) / 0.02 ** 2 - 1) < 0.05


def test_a_captured_step_without_a_clock_says_that_it_repeats():
    p = torch.ones(300, device="cuda")
    opt = fm.AdamW([p], state_bits=8)
    graph = torch.cuda.CUDAGraph()
    with pytest.warns(UserWarning, match="device_step"):
        with torch.cuda.graph(graph):
            opt.step([p], 1e-3)


def test_adamw_with_second_moments_below_the_normal_range():
    """v from 1e-44 to 1e-30 with eps = 1e-30: the root of a denormal is far above eps and must not be taken for 0.  Many steps
    done, so that the corrections are 1; the step's own v is the reference's (it rounds as fp32 denormals do), which leaves
    the root, the sum, the reciprocal and the products: 16 units of 2^-23 as for other values."""
    v = torch.logspace(-44, -30, 4096, dtype=torch.float64, device="cuda").float()
    m = v.double().sqrt().float()
    p, grad = torch.zeros_like(v), torch.zeros_like(v)
    opt = fm.AdamW([p], states=([m], [v]), betas=(0.9, 0.99), eps=1e-30, step=10000)
    opt.step([grad], 1e-2)
    want = -1e-2 * m.double() / (v.double().sqrt() + 1e-30)
    assert bool((v > 0).all()) and bool(((p.double() - want).abs() <= want.abs() * 16 * 2.0 ** -23).all())


@pytest.mark.parametrize("size", [1e-16, 1e-17, 1e-18, 1e-20, 1e-21, 3e-22])
def test_8_bit_second_moments_of_tiny_gradients(size):
    """Gradients whose squares lie below 1e-31, where 65025 / v leaves fp32's range at 1.9e-34: a stored v is one of the two
    codes next to the exact one (which is at least fp32's smallest denormal off), its mean over a block's draws the exact
    one (6 standard errors)."""
    n = 1 << 16
    g = torch.full((n,), 0.3 * size, device="cuda")
    g[::256] = size
    opt = fm.AdamW([torch.zeros(n, device="cuda")], state_bits=8, betas=(0.9, 0.99), seed=5)
    opt.step([g], 0.0)
    k = opt.v[0].double()
    one = torch.tensor(1.0 - 0.99, dtype=torch.float64).float().double()
    exact = (one * g.double() ** 2)
    top = float(exact[0])
    grain = 2.0 ** -149                     # of the exact values as fp32 holds them
    root = (exact / top).sqrt() * 255       # the code that stands for them
    slack = 255 * (2 * grain / top + 2.0 ** -20)
    assert bool((opt.v[0][::256] == 255).all())
    assert bool(((k >= root.floor() - slack) & (k <= root.ceil() + slack)).all())
    assert bool(((k > 0) == (g * g * float(one) > 0)).all())  # a v above 0 keeps a code above 0
    rest = torch.ones(n, dtype=torch.bool, device="cuda")
    rest[::256] = False
    count, mid = int(rest.sum()), float(root[1])
    spread = (2 * math.floor(mid) + 1) / 2  # of k^2 about its mean, at most
    assert abs(float((k[rest] ** 2).mean()) - mid ** 2) <= 6 * spread / math.sqrt(count) + mid ** 2 * (4 * grain / (0.09 * top) + 1e-5)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("cols", [40, 600, 20000])
def test_rounded_rows_of_very_small_values(dtype, cols):
    """Rows whose largest value lies on both sides of 3.7e-37, where 127 / m leaves fp32's range, down to its smallest
    numbers: whole numbers up to 127 as for any other row, from the same fp32 operations on the row times 2^64."""
    import numpy as np
    g = torch.Generator(device="cuda")
    tops = [1e-30, 8e-31, 1e-36, 3e-37, 1e-37, 2e-38, 1e-38, 1e-39] + [1e-42, 1e-44] * (dtype == F32)  # bf16 ends at 9.2e-41
    x = fm._padded((len(tops), cols), dtype, "cuda")
    x.copy_(torch.rand(len(tops), cols, generator=g, device="cuda") * 2 - 1)
    x[:, 7] = 1.0
    x.copy_(x.double() * torch.tensor(tops, dtype=torch.float64, device="cuda").unsqueeze(1))
    q, s = fm.quantize_rows(x)
    v = x.float().cpu().numpy()
    top = np.abs(v).max(1, keepdims=True)
    lift = np.where(top < np.float32(2.0) ** -100, np.float32(2.0) ** 64, np.float32(1)).astype(np.float32)
    want = np.rint((v * lift) * (np.float32(1) / (top * lift) * np.float32(127)))
    assert (top > 0).all() and want.dtype == np.float32
    np.testing.assert_array_equal(q.cpu().numpy(), want.astype(np.int8))
    np.testing.assert_array_equal(s.cpu().numpy(), (top / np.float32(127))[:, 0])
    assert bool((q[:, 7] == 127).all())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 20), (5, 23), (4, 513), (1100, 601), (2, 4099), (2, 16391)])
def test_rounded_rows_write_nothing_past_a_row(dtype, rows, cols):
    """Into columns of a wider buffer: its other columns keep what they hold."""
    g = torch.Generator(device="cuda")
    x = fm._padded((rows, cols), dtype, "cuda")
    x.copy_(torch.randn(rows, cols, generator=g, device="cuda"))
    buf = torch.full((rows, (cols + 31) // 16 * 16), 55, dtype=I8, device="cuda")
    q, _ = fm.quantize_rows(x, q=buf[:, :cols])
    assert torch.equal(q, fm.quantize_rows(x)[0]) and bool((buf[:, cols:] == 55).all())


def stream_of(t):
    """The stream in whose pool torch's allocator keeps t's memory."""
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("no segment holds the tensor")


@pytest.mark.parametrize("raw", [False, True])
def test_outputs_are_made_on_the_stream_that_writes_them(raw):
    """Memory of the current stream's pool can be in use there while another stream writes it."""
    E, N, K, R = 2, 24, 40, 6
    side = torch.cuda.Stream()
    s = side.cuda_stream if raw else side
    x, dy, w = (torch.ones(shape, device="cuda") for shape in ((R, K), (R, N), (E, N, K)))
    offsets = torch.tensor([0, 2, 6], dtype=torch.int32, device="cuda")
    op, q8 = fm.GroupedProduct(E, N, K, R, F32), fm.Int8Product.from_weights(w, R)
    opt = fm.AdamW([torch.zeros(300, device="cuda")], state_bits=8)
    side.wait_stream(torch.cuda.current_stream())
    made = [op.forward(x, w, offsets, stream=s), op.input_grad(dy, w, offsets, stream=s), op.weight_grad(dy, x, offsets, stream=s),
            q8(x, offsets, stream=s), *fm.quantize_rows(x, stream=s),
            *fm.adamw_state_values(opt.m[0], opt.v[0], opt.m_scale[0], opt.v_scale[0], stream=s)]
    made.append(q8.product(*made[4:6], offsets, stream=s))
    side.synchronize()
    assert [stream_of(t) for t in made] == [side.cuda_stream] * len(made)
    assert bool((made[0] == K).all()) and stream_of(op.forward(x, w, offsets)) == torch.cuda.current_stream().cuda_stream


@pytest.mark.parametrize("axis", ["N", "K"])
@pytest.mark.parametrize("result", [BF, F32])
@pytest.mark.parametrize("R", [40, 4000])
def test_an_added_gradient_leaves_what_lies_past_a_width(axis, result, R):
    """Bit for bit, the sign of a zero too, with the reduction in one part and in several (R = 4000)."""
    E, N, K = 2, 45, 50
    g = torch.Generator(device="cuda")
    x, dy = fm._padded((R, K), BF, "cuda"), fm._padded((R, N), BF, "cuda")
    x.copy_(torch.randn(R, K, generator=g, device="cuda"))
    dy.copy_(torch.randn(R, N, generator=g, device="cuda"))
    offsets = torch.tensor([0, R // 3, R], dtype=torch.int32, device="cuda")
    keep = torch.tensor([0, 17], dtype=torch.int32, device="cuda")
    op = fm.GroupedProduct(E, N, K, R, BF, axis)
    dw = fm._padded((E, N, K), result, "cuda")
    dw.fill_(-0.0)
    dw[:, ::3] = float("nan")
    bits = {BF: torch.int16, F32: torch.int32}[result]
    before = dw.clone()
    op.weight_grad(dy, x, offsets, keep, dw=dw, accumulate=True)
    past = torch.ones(E, N, K, dtype=torch.bool, device="cuda")
    if axis == "N":
        past[1, :17] = False
    else:
        past[1, :, :17] = False
    assert torch.equal(dw.contiguous().view(bits)[past], before.contiguous().view(bits)[past])
    assert not torch.equal(dw.contiguous().view(bits)[~past], before.contiguous().view(bits)[~past])


def test_outputs_of_the_layer_are_made_on_the_stream_that_writes_them():
    d, E, I, T = 64, 4, 48, 10
    g = torch.Generator(device="cuda")

    def normal(*shape, dtype=BF):
        return (torch.randn(shape, generator=g, device="cuda") * 0.1).to(dtype)

    side = torch.cuda.Stream()
    layer = fm.Layer(d, E, I, 2, max_tokens=T)
    layer.set_weights(normal(E, I, d), normal(E, I, d), normal(E, d, I))
    layer.set_budget([I, 7, 20, 40])
    x, logits, dy = normal(T, d), normal(T, E, dtype=F32), normal(T, d, dtype=F32)
    want = layer.forward(x, logits)
    act, sal = fm.ActionLearner(layer, T, [0.5, 1.0]), fm.Saliency(layer, T)
    act.transpose_weights()
    alpha, gumbel = normal(E, 2, dtype=F32), normal(E, 2, dtype=F32)
    side.wait_stream(torch.cuda.current_stream())
    sal.add_batch(x, logits, dy, stream=side)
    act.sample(alpha, gumbel, stream=side)
    made = [layer.forward(x, logits, stream=side), act.forward(x, logits, stream=side)]
    made += act.backward(logits, dy, stream=side)
    made += act.action_grad(alpha, gumbel, 1.0, 0.1, 0.0, made[-1], stream=side)
    made += sal.rank_reorder(stream=side)
    c = layer.export_clipped([I, 7, 20, 40], stream=side)
    made += [c.w_gate_c, c.w_up_c, c.w_down_c]
    side.synchronize()
    assert [stream_of(t) for t in made] == [side.cuda_stream] * len(made)
    assert torch.equal(made[0], want)
