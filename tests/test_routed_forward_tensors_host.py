"""Layer.forward with a routing refuses rows that are not of the layer's type or not on the GPU before anything else: the call takes addresses alone."""
import pytest

torch = pytest.importorskip("torch")
from paper_2606_27866_amd import flexmoe as fm  # noqa: E402


@pytest.mark.parametrize("layer_type,types", [(fm.FLEXMOE_F32, (torch.bfloat16, torch.float16, torch.float32)),
                                              (fm.FLEXMOE_BF16, (torch.float32, torch.float16, torch.bfloat16))])
def test_rows(layer_type, types):
    layer = fm.Layer(64, 8, 40, 2, dtype=layer_type, device="cpu")
    r = fm.Routing(torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, 2))
    for t in types:  # the last is the layer's own, but on the CPU
        with pytest.raises(ValueError, match="^x must be 64 contiguous"):
            layer.forward(torch.zeros(1, 64, dtype=t), routing=r)
