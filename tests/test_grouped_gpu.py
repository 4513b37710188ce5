"""The experts' products and their gradients against the same sums in 64 bits, with whatever must not be read set to NaN.

Bounds.  A sum of D products in fp32 is off by at most about D units of 2^-24 of the sum of magnitudes; twice that per
step (2^-23) covers any order and rounding of the matrix cores, and a bf16 result adds half a unit of its own, 2^-9 of
the result (2^-8 here, for a value next to a power of two)."""
import pytest

torch = pytest.importorskip("torch")
from paper_2606_27866_amd import flexmoe as fm  # noqa: E402

pytestmark = pytest.mark.gpu
NAN = float("nan")


def wide(gen, shape, dtype, pad=0, std=1.0):
    """Random values in rows that are `pad` 16-byte units longer than they must be; NaN where no value belongs."""
    cols = fm._pitch(shape[-1], torch.empty((), dtype=dtype).element_size()) + pad * 16 // torch.empty((), dtype=dtype).element_size()
    buf = torch.full((*shape[:-1], cols), NAN, dtype=dtype, device="cuda")
    v = buf[..., :shape[-1]]
    v.copy_(torch.randn(shape, generator=gen, device="cuda") * std)
    return v


class Case:
    def __init__(self, rows, N, K, dtype, axis="none", keep=None, pad=0, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.E, self.N, self.K, self.R, self.axis = len(rows), N, K, sum(rows), axis
        self.dtype, self.rows = dtype, rows
        ends = [0]
        for r in rows:
            ends.append(ends[-1] + r)
        self.spans = list(zip(ends, ends[1:]))
        self.offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
        full = {"N": N, "K": K, "none": 0}[axis]
        if keep is None:
            keep = [(full * (3 * e + 1)) // (3 * self.E) if e % 3 else full for e in range(self.E)]
        self.widths = keep if axis != "none" else None
        self.keep = torch.tensor(keep, dtype=torch.int32, device="cuda") if axis != "none" else None
        self.x = wide(g, (self.R, K), dtype, pad)
        self.dy = wide(g, (self.R, N), dtype, pad)
        self.w = wide(g, (self.E, N, K), dtype, pad, 0.1)
        self.dw0 = wide(g, (self.E, N, K), torch.float32, pad)
        for e, (a, b) in enumerate(self.spans):  # what lies past a width
            n, k = self.limits(e)
            self.w[e, n:] = NAN
            self.w[e, :, k:] = NAN
            self.x[a:b, k:] = NAN
            self.dy[a:b, n:] = NAN
        self.op = fm.GroupedProduct(self.E, N, K, max(self.R, 1), dtype, axis)

    def limits(self, e):
        w = self.widths[e] if self.widths else 0
        return (min(w, self.N) if self.axis == "N" else self.N), (min(w, self.K) if self.axis == "K" else self.K)

    def reference(self, form):
        """(sums in 64 bits, sums of magnitudes, terms) with zeros past the widths."""
        D = torch.float64
        shape = {"forward": (self.R, self.N), "input_grad": (self.R, self.K), "weight_grad": (self.E, self.N, self.K)}[form]
        ref, mag = torch.zeros(shape, dtype=D, device="cuda"), torch.zeros(shape, dtype=D, device="cuda")
        for e, (a, b) in enumerate(self.spans):
            n, k = self.limits(e)
            x, dy, w = self.x[a:b, :k].to(D), self.dy[a:b, :n].to(D), self.w[e, :n, :k].to(D)
            for out, f in ((ref, lambda t: t), (mag, torch.abs)):
                if form == "forward":
                    out[a:b, :n] = f(x) @ f(w).T
                elif form == "input_grad":
                    out[a:b, :k] = f(dy) @ f(w)
                else:
                    out[e, :n, :k] = f(dy).T.contiguous() @ f(x)
        terms = {"forward": self.K, "input_grad": self.N, "weight_grad": max(self.rows, default=0)}[form]
        return ref, mag, terms

    def check(self, out, form, extra=None):
        ref, mag, terms = self.reference(form)
        if extra is not None:
            ref, mag = ref + extra.to(torch.float64), mag + extra.to(torch.float64).abs()
            terms += 1
        bound = mag * ((terms + 4) * 2.0 ** -23)
        if out.dtype == torch.bfloat16:
            bound = bound + ref.abs() * 2.0 ** -8
        err = (out.to(torch.float64) - ref).abs()
        assert out.shape == ref.shape and bool((err <= bound + 1e-300).all()), \
            "%s: %d of %d values are off, the worst by %.3g (bound %.3g)" % (
                form, int((~(err <= bound + 1e-300)).sum()), ref.numel(), float(err.max()), float(bound[err == err.max()].max()) if err.numel() else 0)

    def run(self):
        self.check(self.op.forward(self.x, self.w, self.offsets, self.keep), "forward")
        self.check(self.op.input_grad(self.dy, self.w, self.offsets, self.keep), "input_grad")
        for dt in (torch.float32, torch.bfloat16):
            self.check(self.op.weight_grad(self.dy, self.x, self.offsets, self.keep, dw_dtype=dt), "weight_grad")
        for dt in (torch.float32, torch.bfloat16):
            dw = wide(torch.Generator(device="cuda"), self.dw0.shape, dt)
            before = dw.clone()
            got = self.op.weight_grad(self.dy, self.x, self.offsets, self.keep, dw=dw, accumulate=True)
            assert got is dw
            self.check(dw, "weight_grad", before)


BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,N,K", [
    ([1], 8, 8), ([1], 1, 1), ([3, 0, 1], 5, 7), ([0, 0, 2, 0], 16, 24), ([16, 33, 64], 40, 72), ([129, 1, 0, 255], 130, 129),
    ([128], 128, 128), ([127, 129, 256, 257], 136, 64), ([700], 300, 33), ([2, 5], 1000, 513), ([40] * 70, 33, 65), ([1] * 256, 24, 16),
    ([5000, 0, 37], 96, 200),
])
def test_products(dtype, rows, N, K):
    Case(rows, N, K, dtype).run()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("axis", ["N", "K"])
@pytest.mark.parametrize("rows,N,K", [([5, 0, 40, 130], 70, 90), ([300, 2, 64], 264, 201), ([20, 20, 20, 20, 20], 512, 320)])
def test_widths(dtype, axis, rows, N, K):
    Case(rows, N, K, dtype, axis).run()


@pytest.mark.parametrize("axis", ["N", "K"])
def test_widths_at_their_ends(axis):
    """Nothing kept, one, all, past the end, below zero, and both sides of 16-byte units and tiles."""
    Case([9] * 10, 140, 136, BF, axis, keep=[0, 1, 136, 7, 8, 9, 64, 65, 128, 129]).run()
    c = Case([9] * 3, 48, 40, F32, axis, keep=[0, 40, 3])
    full = {"N": 48, "K": 40}[axis]
    c.keep.copy_(torch.tensor([-5, 1 << 30, 3], dtype=torch.int32))
    c.widths = [0, full, 3]
    c.w[1] = 0.5
    c.x[9:18] = 1.0
    c.dy[9:18] = 1.0
    c.run()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_apart(dtype):
    """Row strides longer than the rows, on every matrix."""
    Case([50, 3, 200], 120, 88, dtype, "N", pad=3).run()
    Case([50, 3, 200], 117, 91, dtype, "K", pad=1).run()


def test_slices_of_wider_tensors():
    """Column halves of one buffer as x and y, whose last row ends with the buffer."""
    E, N, K, R = 2, 64, 96, 50
    g = torch.Generator(device="cuda")
    buf = torch.randn(R, 2 * K, generator=g, device="cuda").bfloat16()
    out = torch.full((R, 2 * N), 7.0, dtype=BF, device="cuda")
    w = torch.randn(E, N, K, generator=g, device="cuda").bfloat16()
    offsets = torch.tensor([0, 20, 50], dtype=torch.int32, device="cuda")
    op = fm.GroupedProduct(E, N, K, R)
    op.forward(buf[:, K:], w, offsets, y=out[:, N:])
    ref = torch.cat([buf[:20, K:].double() @ w[0].double().T, buf[20:, K:].double() @ w[1].double().T])
    assert bool((out[:, :N] == 7.0).all())
    assert float((out[:, N:].double() - ref).abs().max()) <= float(ref.abs().max()) * 2.0 ** -8


def test_rows_outside_the_groups_are_left_alone():
    R, N, K = 40, 24, 32
    op = fm.GroupedProduct(2, N, K, R, F32)
    x = torch.full((R, K), NAN, device="cuda")
    x[4:30] = 1.0
    offsets = torch.tensor([4, 10, 30], dtype=torch.int32, device="cuda")
    w = torch.ones(2, N, K, device="cuda")
    y = torch.full((R, N), 7.0, device="cuda")
    op.forward(x, w, offsets, y=y)
    assert bool((y[4:30] == K).all()) and bool((y[:4] == 7).all()) and bool((y[30:] == 7).all())
    dw = op.weight_grad(y, x, offsets)
    assert bool((dw[0] == 6.0 * K).all()) and bool((dw[1] == 20.0 * K).all())


def test_no_rows_at_all():
    op = fm.GroupedProduct(3, 16, 24, 8, F32)
    offsets = torch.zeros(4, dtype=torch.int32, device="cuda")
    x, dy = torch.empty(0, 24, device="cuda"), torch.empty(0, 16, device="cuda")
    assert op.forward(x, torch.ones(3, 16, 24, device="cuda"), offsets).shape == (0, 16)
    assert bool((op.weight_grad(dy, x, offsets) == 0).all())


@pytest.mark.parametrize("dtype", [BF, F32])
def test_gradients_against_differences(dtype):
    """L = <c, y(x, W)> is linear in x and in W: a difference over a step of 2 is the gradient itself.  Values are small
    whole numbers, so that every sum is exact in fp32 and the comparison too."""
    rows, N, K = [6, 0, 11], 20, 12
    c = Case(rows, N, K, dtype)
    g = torch.Generator(device="cuda")

    def whole(shape):
        t = wide(g, shape, dtype)
        return t.copy_(torch.randint(-3, 4, shape, generator=g, device="cuda"))

    x, w, cy = whole((17, K)), whole((3, N, K)), whole((17, N))
    op = fm.GroupedProduct(3, N, K, 17, dtype)
    dx, dw = op.input_grad(cy, w, c.offsets), op.weight_grad(cy, x, c.offsets)

    def loss():
        return float((op.forward(x, w, c.offsets).double() * cy.double()).sum())

    for r, k in [(0, 0), (5, 11), (6, 3), (16, 7)]:
        old = float(x[r, k])
        x[r, k] = old + 1
        up = loss()
        x[r, k] = old - 1
        assert (up - loss()) / 2 == float(dx[r, k])
        x[r, k] = old
    for e, n, k in [(0, 0, 0), (0, 19, 11), (1, 4, 4), (2, 7, 2)]:
        old = float(w[e, n, k])
        w[e, n, k] = old + 1
        up = loss()
        w[e, n, k] = old - 1
        assert (up - loss()) / 2 == float(dw[e, n, k])
        w[e, n, k] = old


def test_same_bits_again_and_on_another_stream():
    c = Case([100, 3, 900], 200, 136, BF, "N")
    first = [c.op.forward(c.x, c.w, c.offsets, c.keep), c.op.weight_grad(c.dy, c.x, c.offsets, c.keep)]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        again = [c.op.forward(c.x, c.w, c.offsets, c.keep), c.op.weight_grad(c.dy, c.x, c.offsets, c.keep)]
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_refused_tensors():
    op = fm.GroupedProduct(2, 16, 24, 8, F32)
    offsets = torch.zeros(3, dtype=torch.int32, device="cuda")
    x, w = torch.zeros(8, 24, device="cuda"), torch.zeros(2, 16, 24, device="cuda")
    for bad in (dict(x=x.bfloat16()), dict(x=x[:, :20]), dict(x=torch.zeros(24, 8, device="cuda").T), dict(w=w[:, :8]),
                dict(w=torch.zeros(2, 32, 24, device="cuda")[:, ::2][:, :16].transpose(0, 1)), dict(offsets=offsets.long()),
                dict(offsets=offsets[:2]), dict(x=x.cpu())):
        a = dict(dict(x=x, w=w, offsets=offsets), **bad)
        with pytest.raises((ValueError, fm.FlexMoEError)):
            op.forward(a["x"], a["w"], a["offsets"])
    with pytest.raises(fm.FlexMoEError):
        op.forward(torch.zeros(9, 24, device="cuda"), w, offsets)  # more rows than max_rows
    with pytest.raises(ValueError):
        op.weight_grad(torch.zeros(8, 16, device="cuda"), x, offsets, accumulate=True)


# Sizes that reach every kind of tiles, with ends inside tiles, 16-byte units and K tiles, and reductions in parts.
LARGE = [
    ([9000, 300, 0, 2700], 4099, 2003),  # 256 x 256 tiles, 4 to 1 steps of 64 rows, odd sides
    ([12000], 4096, 2048),              # the same with whole tiles
    ([1100, 0, 700, 300], 1000, 900),
    ([2300], 2049, 1033),               # one group, rows of 16-byte units that end past the matrix
    ([4100, 900], 520, 300),            # few tiles of a long reduction over rows: parts
    ([70, 3, 33, 16], 700, 5000),       # few rows, long rows: parts of the forward
    ([9, 1, 0, 31, 32, 40], 5000, 700),  # few rows, many columns: parts of the input gradient
]


@pytest.mark.parametrize("axis", ["none", "N", "K"])
@pytest.mark.parametrize("rows,N,K", LARGE)
def test_large_products(rows, N, K, axis):
    Case(rows, N, K, BF, axis, pad=1 if axis == "K" else 0).run()


@pytest.mark.parametrize("rows,N,K", [([600, 5], 300, 260), ([20, 2], 300, 2100), ([3000], 140, 200)])
def test_large_products_fp32(rows, N, K):
    Case(rows, N, K, F32, "N").run()


def test_weights_larger_than_the_last_level_cache():
    """Weights above 96 MB are read with another cache hint."""
    Case([3, 40, 0, 140] * 4, 1500, 2100, BF, "N").run()


def test_a_reduction_that_passes_2_31_bytes():
    """One group whose rows lie further apart than 32 bits of bytes: 40000 rows, 32768 values apart."""
    R, N, K, ld = 40000, 8, 16, 32768
    g = torch.Generator(device="cuda")
    x = torch.empty(R, ld, dtype=BF, device="cuda")[:, :K]
    x.copy_(torch.randint(-2, 3, (R, K), generator=g, device="cuda"))
    dy = torch.randint(-2, 3, (R, N), generator=g, device="cuda").to(BF)
    w = torch.randint(-2, 3, (1, N, K), generator=g, device="cuda").to(BF)
    op = fm.GroupedProduct(1, N, K, R)
    offsets = torch.tensor([0, R], dtype=torch.int32, device="cuda")
    assert torch.equal(op.weight_grad(dy, x, offsets)[0].double(), dy.double().T.contiguous() @ x.double())
    assert torch.equal(op.forward(x, w, offsets).double(), x.double() @ w[0].double().T)


def test_without_a_workspace():
    """No partial sums: one part, the same values within the sums' bound."""
    c = Case([70, 3, 33, 16], 700, 5000, BF)
    y = torch.empty(c.R, 704, dtype=BF, device="cuda")[:, :700]
    c.op.forward(c.x, c.w, c.offsets)  # sets the descriptor's strides
    fm.flexmoe_grouped_forward(c.op.desc, c.R, c.x, c.w, c.offsets, None, y, None, 0)
    c.check(y, "forward")
