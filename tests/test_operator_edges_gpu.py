"""Calls at the edges of the experts' products, the 8-bit products and AdamW: stacks, whole tensors without offsets, streams,
graphs, threads, moved storages, very small values, and every kind of tiles in one part and in several."""
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
