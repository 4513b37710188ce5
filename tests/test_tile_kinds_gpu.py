"""Every kind of tiles, in one part and in several, for every form and type, against the same sums in 64 bits (the bounds of
the tests whose cases these are)."""
import pytest

torch = pytest.importorskip("torch")
from tests import test_grouped_gpu as grouped  # noqa: E402
from tests import test_quantized_gpu as quantized  # noqa: E402
from tests.tile_kinds import BIG_DEPTHS, BIG_LAST, SIZES, big_sizes, rows_of  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.mark.parametrize("form,elem,result,kind,parts,E,N,K,R", SIZES)
def test_kind(form, elem, result, kind, parts, E, N, K, R):
    rows = rows_of(E, R)
    if elem == "i8":
        quantized.product_case(rows, N, K, TYPES[result])
        return
    c = grouped.Case(rows, N, K, TYPES[elem])
    if form == "forward":
        c.check(c.op.forward(c.x, c.w, c.offsets), form)
    elif form == "input_grad":
        c.check(c.op.input_grad(c.dy, c.w, c.offsets), form)
    else:
        c.check(c.op.weight_grad(c.dy, c.x, c.offsets, dw_dtype=TYPES[result]), form)
        dw = grouped.wide(torch.Generator(device="cuda"), c.dw0.shape, TYPES[result])
        before = dw.clone()
        c.check(c.op.weight_grad(c.dy, c.x, c.offsets, dw=dw, accumulate=True), form, before)


@pytest.mark.parametrize("axis", ["N", "K"])
@pytest.mark.parametrize("form,elem,result,kind,parts,E,N,K,R", [s for s in SIZES if s[3] == "big" and s[4] == "several"])
def test_widths_of_the_largest_tiles_in_parts(form, elem, result, kind, parts, E, N, K, R, axis):
    """Reductions whose parts end before or after a group's width."""
    rows = rows_of(E, R)
    if elem == "i8":
        quantized.product_case(rows, N, K, TYPES[result], axis)
        return
    c = grouped.Case(rows, N, K, TYPES[elem], axis)
    if form == "forward":
        c.check(c.op.forward(c.x, c.w, c.offsets, c.keep), form)
    elif form == "input_grad":
        c.check(c.op.input_grad(c.dy, c.w, c.offsets, c.keep), form)
    else:
        c.check(c.op.weight_grad(c.dy, c.x, c.offsets, c.keep, dw_dtype=TYPES[result]), form)


@pytest.mark.parametrize("depth", BIG_DEPTHS)
@pytest.mark.parametrize("last", BIG_LAST)
def test_stores_behind_the_last_requests(depth, last):
    """256 x 256 tiles of two to five K tiles, an odd and an even number, each number of row steps: results leave through LDS
    that the last requests of the loop fill with zeros.  Whole numbers, so that every sum is exact and a zero in the wrong
    place shows."""
    E, N, R = big_sizes(last)
    rows = [R // E] * E
    g = torch.Generator(device="cuda")
    g.manual_seed(depth * 1000 + last)
    x = torch.randint(1, 4, (R, depth), generator=g, device="cuda").to(torch.bfloat16)
    w = torch.randint(1, 3, (E, N, depth), generator=g, device="cuda").to(torch.bfloat16)
    offsets = torch.arange(E + 1, dtype=torch.int32, device="cuda") * rows[0]
    op = grouped.fm.GroupedProduct(E, N, depth, R)
    y = op.forward(x, w, offsets)
    for e in range(E):
        a, b = e * rows[0], (e + 1) * rows[0]
        assert torch.equal(y[a:b], (x[a:b].float() @ w[e].float().T).to(torch.bfloat16))
