"""Columns behind a ragged row of the norm's 8-bit output, and the router's gradient against differences of every kind, compared at every place."""
import pytest

torch = pytest.importorskip("torch")
from paper_2606_27866_amd import flexmoe as fm  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols", [(1, 1), (6, 100), (3, 513), (1030, 1001), (2, 2051), (1, 4099), (1, 8197), (2, 16390)])
def test_nothing_past_an_8_bit_row_is_written(rows, cols):
    g = torch.Generator(device="cuda")
    g.manual_seed(cols)
    for dtype in (torch.bfloat16, torch.float32):
        x = fm._padded((rows, cols), dtype, "cuda").copy_(torch.empty(rows, cols, device="cuda").normal_(generator=g))
        norm = fm.RMSNorm(torch.ones(cols, dtype=dtype, device="cuda"), rows)
        want = norm.quantized(x)
        wide = torch.full((rows, -(-cols // 16) * 16 + 32), 77, dtype=torch.int8, device="cuda")
        scales = torch.full((rows + 8,), 7.0, device="cuda")
        norm.quantized(x, q=wide[:, :cols], scale=scales[:rows])
        assert torch.equal(wide[:, :cols], want[0]) and bool((wide[:, cols:] == 77).all())
        assert torch.equal(scales[:rows], want[1]) and bool((scales[rows:] == 7).all())


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("normalize", [False, True])
@pytest.mark.parametrize("E,k", [(10, 3), (70, 4), (200, 8)])
def test_router_gradient_against_differences(score, normalize, E, k):
    """Logits a quarter apart, in any order: a step of 1e-2 changes no choice, which is asserted.  The loss is off by its third derivative
    (below scale sum |c| here, times step^2 / 6) and by 40 u of its size over the step."""
    T, step, scale = 4, 1e-2, 2.0
    g = torch.Generator(device="cuda")
    g.manual_seed(E)
    x = torch.stack([torch.randperm(E, generator=g, device="cuda").float() / 4 - E / 8 for _ in range(T)])
    x = x.clamp(min=-4.0) if E <= 10 else x - x.amax(1, keepdim=True) + 2.0
    c = torch.empty(T, k, device="cuda").normal_(generator=g)
    router = fm.Router(E, k, T, score, normalize, scale)
    ids = router.route(x).topk_idx
    dl = router.backward(x, ids, c)
    size = scale * float(c.abs().sum(1).max())
    for t in range(T):
        for e in [int(ids[t, j]) for j in range(k)] + [e for e in range(E) if e not in ids[t].tolist()][:2]:
            f = []
            for s in (step, -step):
                v = x.clone()
                v[t, e] += s
                r = router.route(v)
                assert torch.equal(r.topk_idx, ids)
                f.append(float((r.topk_w[t].double() * c[t].double()).sum()))
            assert abs((f[0] - f[1]) / (2 * step) - float(dl[t, e])) <= size * (step ** 2 / 6 + 40 * 2.0 ** -24 / step)
