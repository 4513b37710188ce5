"""Routing of the most tokens that a descriptor allows: max_tokens (top_k + 1) = 2^30. Its first kernel has 2^32 threads in all, more than one launch can have."""
import pytest

torch = pytest.importorskip("torch")
from paper_2606_27866_amd import flexmoe as fm  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1 << 29, (1 << 29) - 130])
def test_most_tokens(T):
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x = torch.empty(T, 2, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    router = fm.Router(2, 1, T, score="sigmoid", normalize=False)
    r = router.route(x)
    second = x[:, 1] > x[:, 0]  # ties to the lower id
    assert torch.equal(r.topk_idx.view(-1), second.int())
    n = int(second.sum())
    assert r.counts.tolist() == [T - n, n] and r.offsets.tolist() == [0, T - n, T]
    assert torch.equal(r.perm[:T - n], torch.nonzero(~second).view(-1).int()) and torch.equal(r.perm[T - n:], torch.nonzero(second).view(-1).int())
    for part in (slice(0, 1 << 20), slice(T // 2 - 5, T // 2 + (1 << 20)), slice(T - (1 << 20), T)):
        at = r.pos[part].long()
        assert torch.equal(r.perm[at], torch.arange(part.start, part.stop, device="cuda").int())
        want = torch.sigmoid(x[part].double().amax(1))
        assert bool(((r.topk_w[part, 0].double() - want).abs() <= 40 * 2.0 ** -24 * want).all())
    alone = router.route(x, tables=False)
    assert torch.equal(alone.topk_idx, r.topk_idx) and torch.equal(alone.topk_w, r.topk_w)
