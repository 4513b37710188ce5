"""Rows rounded to 8 bits and the 8-bit products, against their definitions.

Bounds.  Rounded rows are compared for equality with the same fp32 operations in NumPy.  A product's sum is exact; its
conversion and the two products with the scales round once each (3 units of 2^-24), a bf16 result once more (2^-9)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from paper_2606_27866_amd import flexmoe as fm  # noqa: E402

pytestmark = pytest.mark.gpu


def reference_rows(v):
    v = np.asarray(v, np.float32)
    top = np.abs(v).max(-1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        q = np.rint(v * np.where(top > 0, np.float32(1) / top * np.float32(127), np.float32(0)).astype(np.float32))
    return np.clip(q, -127, 127).astype(np.int8), (top / np.float32(127))[..., 0]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (2, 8), (5, 9), (4, 512), (3, 513), (7, 2048), (2, 2050), (2, 4097), (1, 16384), (2, 16399)])
def test_rows(dtype, rows, cols):
    g = torch.Generator(device="cuda")
    x = fm._padded((rows, cols), torch.float32, "cuda")
    x = torch.full((rows, -(-cols // 8) * 8 + 8), float("nan"), dtype=dtype, device="cuda")[:, :cols]
    x.copy_(torch.randn(rows, cols, generator=g, device="cuda") * 3)
    q, s = fm.quantize_rows(x)
    qr, sr = reference_rows(x.float().cpu().numpy())
    np.testing.assert_array_equal(q.cpu().numpy(), qr)
    np.testing.assert_array_equal(s.cpu().numpy(), sr)


def test_rows_of_zeros_extremes_and_non_finite():
    x = torch.zeros(8, 40, device="cuda")
    x[1, 3], x[2, 39], x[3, 0] = float("nan"), float("inf"), -float("inf")
    x[4, 5] = 1e-44                     # a denormal: 127 / 1e-44 overflows
    x[5] = torch.finfo(torch.float32).max
    x[6] = torch.linspace(-1, 1, 40)
    q, s = fm.quantize_rows(x)
    assert float(s[0]) == 0 and bool((q[0] == 0).all())
    for r in (1, 2, 3):
        assert bool(torch.isnan(s[r])) and bool((q[r] == 0).all())
    assert bool((q[4].abs() <= 127).all()) and bool((q[4, 6:] == 0).all())
    assert bool((q[5] == 127).all()) and float(s[5]) == float(np.float32(3.4028235e38) / np.float32(127))
    assert int(q[6].max()) == 127 and int(q[6].min()) == -127


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(5, 40), (3, 1000), (2, 5000)])
def test_gated_rows(dtype, rows, cols):
    """silu(g) u in 64 bits; the largest value may be off by a few units (8 of 2^-24: exp, sum, quotient, product), which
    moves the scale by as much and a rounded value by at most one."""
    g = torch.Generator(device="cuda")
    gate, up = ((torch.randn(rows, cols, generator=g, device="cuda") * 2).to(dtype) for _ in range(2))
    gate[0, 0] = -200.0  # silu -> 0
    q, s = fm.quantize_rows(up, gate=gate)
    v = torch.nn.functional.silu(gate.double()) * up.double()
    top = v.abs().amax(1)
    assert bool(((s.double() * 127 - top).abs() <= 8 * 2.0 ** -24 * top).all())
    assert bool(((q.double() * s.double().unsqueeze(1) - v).abs() <= s.double().unsqueeze(1) * 0.5001 + top.unsqueeze(1) * 1e-6).all())


def product_case(rows, N, K, out, axis="none", keep=None, seed=0, most=127):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    E, R = len(rows), sum(rows)
    ends = np.concatenate([[0], np.cumsum(rows)])
    offsets = torch.from_numpy(ends.astype(np.int32)).cuda()

    def whole(shape):
        t = torch.full((*shape[:-1], -(-shape[-1] // 16) * 16 + 16), 101, dtype=torch.int8, device="cuda")[..., :shape[-1]]
        return t.copy_(torch.randint(-most, most + 1, shape, generator=g, device="cuda"))

    q, w = whole((R, K)), whole((E, N, K))
    qs, ws = torch.rand(R, generator=g, device="cuda") + 0.1, torch.rand(E, N, generator=g, device="cuda") + 0.1
    if keep is None and axis != "none":
        keep = [(3 * e + 1) * (N if axis == "N" else K) // (3 * E) for e in range(E)]
    kd = torch.tensor(keep, dtype=torch.int32, device="cuda") if axis != "none" else None
    op = fm.Int8Product(w, ws, max(R, 1), axis, out)
    y = op.product(q, qs, offsets, kd)
    ref = torch.zeros(R, N, dtype=torch.float64, device="cuda")
    for e in range(E):
        a, b = int(ends[e]), int(ends[e + 1])
        n, k = (keep[e] if axis == "N" else N), (keep[e] if axis == "K" else K)
        ref[a:b, :n] = q[a:b, :k].double() @ w[e, :n, :k].double().T * qs[a:b].double().unsqueeze(1) * ws[e, :n].double()
    bound = ref.abs() * (4 * 2.0 ** -24 + (2.0 ** -8 if out == torch.bfloat16 else 0))
    assert bool(((y.double() - ref).abs() <= bound).all()), float(((y.double() - ref).abs() - bound).max())


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,N,K", [([1], 1, 1), ([1], 4096, 1024), ([5], 33, 17), ([3, 0, 1], 40, 128), ([16, 64, 200], 136, 272), ([300], 257, 129),
                                      ([1, 2, 3, 4], 520, 2000), ([7] * 100, 48, 64), ([1000, 0, 13], 260, 96), ([2], 200, 14336)])
def test_products(out, rows, N, K):
    product_case(rows, N, K, out)


@pytest.mark.parametrize("axis", ["N", "K"])
@pytest.mark.parametrize("rows,N,K", [([3, 0, 9], 64, 80), ([200, 40], 300, 333), ([2] * 6, 140, 140)])
def test_widths(axis, rows, N, K):
    product_case(rows, N, K, torch.float32, axis)
    product_case(rows, N, K, torch.bfloat16, axis, keep=[0, 1, 17, 64, 65, 79][:len(rows)])


def test_the_largest_sums():
    """The longest reduction with the largest whole numbers: the sum fills 31 bits."""
    K = 131071
    q = torch.full((2, -(-K // 16) * 16), -128, dtype=torch.int8, device="cuda")[:, :K]
    w = torch.full((1, 3, -(-K // 16) * 16), -128, dtype=torch.int8, device="cuda")[..., :K]
    op = fm.Int8Product(w, torch.ones(1, 3, device="cuda"), 2, out_dtype=torch.float32)
    y = op.product(q, torch.ones(2, device="cuda"))
    assert bool((y.double() == float(np.float32(128 * 128 * K))).all())


def test_non_finite_rows_are_nan():
    x = torch.ones(3, 64, device="cuda")
    x[1, 7] = float("inf")
    op = fm.Int8Product.from_weights(torch.ones(1, 40, 64, device="cuda"), 3, out_dtype=torch.float32)
    y = op(x)
    assert bool(torch.isnan(y[1]).all()) and bool((y[0] == y[2]).all()) and bool(torch.isfinite(y[0]).all())


@pytest.mark.parametrize("T", [1, 8, 70, 300])
def test_whole_call(T):
    """bf16 rows through both steps, against the definition in 64 bits: where a rounding to whole numbers falls the other
    way (ties within fp32's reach), one term of the sum moves by a unit: 2 of 1000 values at most, 1e-3 of the result."""
    g = torch.Generator(device="cuda")
    w = (torch.randn(1, 200, 333, generator=g, device="cuda") * 0.05).to(torch.bfloat16)
    x = torch.randn(T, 333, generator=g, device="cuda")
    xp = torch.zeros(T, 336, dtype=torch.bfloat16, device="cuda")[:, :333]
    xp.copy_(x)
    wp = torch.zeros(1, 200, 336, dtype=torch.bfloat16, device="cuda")[..., :333]
    wp.copy_(w)
    op = fm.Int8Product.from_weights(wp, 300, out_dtype=torch.float32)
    y = op(xp)
    top = xp.double().abs().amax(1, keepdim=True)
    q = torch.round(xp.double() * 127 / top)
    ref = (q * (top / 127)) @ (op.w[0].double() * op.w_scale[0].double().unsqueeze(1)).T
    assert float((y.double() - ref).norm() / ref.norm()) <= 1e-3
    # and near the product of what was rounded: each value is off by up to half a unit of its row's scale, the errors
    # independent: 2 / 127 of the norm is far outside them
    full = xp.double() @ wp[0].double().T
    assert float((y.double() - full).norm() / full.norm()) <= 2 / 127


@pytest.mark.parametrize("axis", ["none", "N", "K"])
@pytest.mark.parametrize("rows,N,K", [([9000, 300, 0, 2700], 4099, 4003), ([12000], 4096, 2048), ([1100, 0, 700, 300], 1000, 1800), ([2300], 2049, 1033), ([70, 3, 33, 16], 700, 9000),
                                      ([3, 40, 0, 140] * 4, 1500, 4200)])
def test_large_products(rows, N, K, axis):
    """Sizes that reach every kind of tiles, reductions in parts, and weights above 96 MB."""
    product_case(rows, N, K, torch.bfloat16, axis)
