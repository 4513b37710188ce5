"""The training and 8-bit operators captured in a HIP graph: replays between eager calls give the eager bits."""
import pytest

torch = pytest.importorskip("torch")
from paper_2606_27866_amd import flexmoe as fm  # noqa: E402

pytestmark = pytest.mark.gpu


def test_replays_equal_eager_calls():
    E, N, K, R = 6, 264, 520, 700
    g = torch.Generator(device="cuda")
    offsets = torch.tensor([0, 100, 100, 350, 351, 600, 700], dtype=torch.int32, device="cuda")
    x, dy = (torch.randn(R, c, generator=g, device="cuda").bfloat16() for c in (K, N))
    w = torch.randn(E, N, K, generator=g, device="cuda").bfloat16()
    op, q8 = fm.GroupedProduct(E, N, K, R), fm.Int8Product.from_weights(torch.randn(E, N, 528, generator=g, device="cuda"), R)
    x8 = torch.randn(R, 528, generator=g, device="cuda").bfloat16()
    out = [torch.empty(R, N, dtype=torch.bfloat16, device="cuda"), torch.empty(R, K, dtype=torch.bfloat16, device="cuda"),
           torch.empty(E, N, K, device="cuda"), torch.empty(R, N, dtype=torch.bfloat16, device="cuda")]

    def calls():
        op.forward(x, w, offsets, y=out[0])
        op.input_grad(dy, w, offsets, dx=out[1])
        op.weight_grad(dy, x, offsets, dw=out[2])
        q8(x8, offsets, y=out[3])

    calls()
    torch.cuda.synchronize()
    want = [t.clone() for t in out]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for _ in range(4):
        for t in out:
            t.fill_(-1.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        x.neg_()
        calls()  # eager work on other inputs in between
        x.neg_()


def test_optimizer_step_in_a_graph():
    g = torch.Generator(device="cuda")
    p, grad = torch.randn(5000, generator=g, device="cuda"), torch.randn(5000, generator=g, device="cuda")
    q = p.clone()
    a, b = fm.AdamW([p], state_bits=8, seed=3), fm.AdamW([q], state_bits=8, seed=3)
    keep = [t.clone() for t in (p, a.m[0], a.v[0], a.m_scale[0], a.v_scale[0])]
    b.step([grad], 1e-2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step([grad], 1e-2)
    for _ in range(3):  # the captured step is step 1: from the same state the same bits
        for t, k in zip((p, a.m[0], a.v[0], a.m_scale[0], a.v_scale[0]), keep):
            t.copy_(k)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(p, q) and torch.equal(a.m[0], b.m[0]) and torch.equal(a.v[0], b.v[0])
