"""AdamW over many tensors against its formulas in 64 bits, and the 8-bit states against their definition.

Bounds.  A step's fp32 operations are fewer than 16, each within 2^-23 of its result (the root and the reciprocal included);
the update is bounded by lr times the largest ratio.  8-bit states: a stored value is one of the two codes next to the exact
one (the code spacing), and its mean over many draws is the exact one (6 standard errors)."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
from paper_2606_27866_amd import flexmoe as fm  # noqa: E402

pytestmark = pytest.mark.gpu
B1, B2, EPS, WD, LR = 0.9, 0.99, 1e-8, 0.1, 1e-2


def exact_step(p, g, m, v, t, grad_scale=1.0):
    g = g.double() * grad_scale
    m = B1 * m.double() + (1 - B1) * g
    v = B2 * v.double() + (1 - B2) * g * g
    upd = LR / (1 - B1 ** t) * m / ((v / (1 - B2 ** t)).sqrt() + EPS)
    return p.double() * (1 - LR * WD) - upd, m, v, upd


def tensors(sizes, dtype, gen, std=1.0, shift=0):
    """Tensors of these sizes, `shift` elements away from a 16-byte boundary."""
    out = []
    for n in sizes:
        t = torch.empty(n + 16, device="cuda").normal_(0, std, generator=gen).to(dtype)[shift:shift + n]
        out.append(t)
    return out


def close(got, ref, scale, units):
    assert bool(((got.double() - ref).abs() <= scale.abs() * (units * 2.0 ** -23) + 1e-42).all())


SIZES = [1, 3, 4, 255, 256, 257, 1024, 4095, 4096, 4097, 10000, 0, 7]


@pytest.mark.parametrize("pdt,gdt,master", [(torch.float32, torch.float32, False), (torch.float32, torch.bfloat16, False),
                                            (torch.bfloat16, torch.bfloat16, True), (torch.bfloat16, torch.float32, False)])
@pytest.mark.parametrize("shift", [0, 1])
def test_32_bit_states(pdt, gdt, master, shift):
    g = torch.Generator(device="cuda")
    p = tensors(SIZES, pdt, g, shift=shift)
    mast = [t.float().clone() + 1e-4 for t in p] if master else None
    m = tensors(SIZES, torch.float32, g, 0.1, shift)
    v = [t.square() for t in tensors(SIZES, torch.float32, g, 0.3, shift)]
    opt = fm.AdamW(p, masters=mast, states=(m, v), betas=(B1, B2), eps=EPS, weight_decay=WD, step=4)
    for t in (5, 6):
        grads = tensors(SIZES, gdt, g, 0.5, shift)
        before = [(a.clone(), b.clone(), c.clone()) for a, b, c in zip(mast or p, m, v)]
        opt.step(grads, LR, grad_scale=0.25)
        for i in range(len(SIZES)):
            rp, rm, rv, upd = exact_step(before[i][0], grads[i], before[i][1], before[i][2], t, 0.25)
            close(m[i], rm, before[i][1].double().abs() + grads[i].double().abs(), 4)
            close(v[i], rv, rv, 8)
            # the update's error goes by |m| / (sqrt(v) + eps), m's own error by its terms
            size = LR / (1 - B1 ** t) * (before[i][1].double().abs() + grads[i].double().abs()) / ((rv / (1 - B2 ** t)).sqrt() + EPS)
            full = mast[i] if master else p[i]
            if full.dtype == torch.bfloat16:
                assert bool(((p[i].double() - rp).abs() <= rp.abs() * 2.0 ** -8 + size * 2.0 ** -18).all())
            else:
                close(full, rp, before[i][0].double().abs() + 2 * size, 16)
            if master:
                assert torch.equal(p[i], full.to(torch.bfloat16))


def codes_m():
    k = np.arange(1, 128)
    mag = np.concatenate([[0.0], ((896 + k).astype(np.uint32) << 20).view(np.float32).astype(np.float64)])
    return torch.from_numpy(mag).cuda()


def neighbours_ok(value, exact, grid):
    """|value| is one of the two grid magnitudes around |exact| (1e-6 of slack for the fp32 arithmetic before it)."""
    a, e = value.abs(), exact.abs()
    i = torch.searchsorted(grid, e.contiguous()).clamp(1, grid.numel() - 1)
    lo, hi = grid[i - 1], grid[i]
    near = (a >= lo * (1 - 1e-6) - 1e-300) & (a <= hi * (1 + 1e-6))
    return near | ((a - e).abs() <= 1e-6 * e)


@pytest.mark.parametrize("pdt,gdt,master", [(torch.float32, torch.float32, False), (torch.float32, torch.bfloat16, False),
                                            (torch.bfloat16, torch.bfloat16, True), (torch.bfloat16, torch.float32, False)])
@pytest.mark.parametrize("shift", [0, 1])
def test_8_bit_states(pdt, gdt, master, shift):
    g = torch.Generator(device="cuda")
    p = tensors(SIZES, pdt, g, shift=shift)
    mast = [t.float().clone() for t in p] if master else None
    opt = fm.AdamW(p, masters=mast, state_bits=8, betas=(B1, B2), eps=EPS, weight_decay=WD, seed=77)
    grid = codes_m()
    for t in (1, 2, 3):
        grads = [x * torch.exp2(torch.randint(-12, 3, x.shape, generator=g, device="cuda").float()).to(gdt) for x in tensors(SIZES, gdt, g, 0.5, shift)]
        grads = [x.contiguous() if not shift else torch.cat([x[:0].new_zeros(shift), x])[shift:] for x in grads]
        state = [fm.adamw_state_values(opt.m[i], opt.v[i], opt.m_scale[i], opt.v_scale[i]) if n else None for i, n in enumerate(SIZES)]
        before = [x.clone() for x in (mast or p)]
        opt.step(grads, LR)
        for i, n in enumerate(SIZES):
            if not n:
                continue
            rp, rm, rv, upd = exact_step(before[i], grads[i], *state[i], t)
            m, v = fm.adamw_state_values(opt.m[i], opt.v[i], opt.m_scale[i], opt.v_scale[i])
            for b in range(0, n, 256):
                s = slice(b, min(n, b + 256))
                top = float(rm[s].abs().max())
                sm = float(opt.m_scale[i][b // 256])
                assert sm == 2.0 ** math.floor(math.log2(sm)) and 0.9375 * sm * (1 - 1e-6) < top <= 1.875 * sm * (1 + 1e-6)
                assert bool(neighbours_ok(m[s].double(), rm[s], grid * sm).all())
                assert bool((torch.sign(m[s]) * torch.sign(rm[s]) >= 0).all())
                sv = float(opt.v_scale[i][b // 256])
                assert abs(sv * 255 / math.sqrt(float(rv[s].max())) - 1) < 1e-6
                vgrid = (torch.arange(256, dtype=torch.float64, device="cuda") * sv) ** 2
                assert bool(neighbours_ok(v[s].double(), rv[s], vgrid).all())
                assert bool(((v[s] > 0) == (rv[s] > 0)).all())
            # the step itself uses the unrounded states
            size = upd.abs() + LR / (1 - B1 ** t) * (state[i][0].double().abs() + grads[i].double().abs()) / ((rv / (1 - B2 ** t)).sqrt() + EPS)
            full = mast[i] if master else p[i]
            if full.dtype == torch.bfloat16:
                assert bool(((full.double() - rp).abs() <= rp.abs() * 2.0 ** -8 + size * 2.0 ** -18).all())
            else:
                close(full, rp, before[i].double().abs() + 2 * size, 16)
            if master:
                assert torch.equal(p[i], full.to(torch.bfloat16))


def test_8_bit_states_keep_their_mean():
    """One value in every place: over n draws the stored values' mean is the exact one within 6 of its standard errors (a
    code spacing d gives at most d / 2 per draw), for m and for v."""
    n = 1 << 16
    for mag in (1.0, 0.37, 3e-3):
        g = torch.full((n,), 0.11 * mag, device="cuda")
        g[::256] = 1.0  # sets the blocks' scales
        opt = fm.AdamW([torch.zeros(n, device="cuda")], state_bits=8, betas=(B1, B2), seed=5)
        opt.step([g], LR)
        m, v = (x.double() for x in fm.adamw_state_values(opt.m[0], opt.v[0], opt.m_scale[0], opt.v_scale[0]))
        rest = torch.ones(n, dtype=torch.bool, device="cuda")
        rest[::256] = False
        count = int(rest.sum())
        em = (1 - B1) * float(g[1].double())
        assert abs(float(m[rest].mean()) - em) <= 6 * (em / 8) / 2 / math.sqrt(count) + 1e-7 * em
        ev = (1 - B2) * float(g[1].double()) ** 2
        sv = float(opt.v_scale[0][0])
        k = math.floor(math.sqrt(ev) / sv)
        if k >= 1:  # below the first code v is held up on purpose
            assert abs(float(v[rest].mean()) - ev) <= 6 * (2 * k + 1) * sv * sv / 2 / math.sqrt(count) + 1e-6 * ev
        else:
            assert bool((v[rest] == np.float32(sv) * np.float32(sv)).all())


def test_8_bit_states_follow_a_long_run():
    """A constant gradient: m and v reach it though a step moves them by a tenth and a hundredth, less than a code spacing."""
    n = 4096
    g = torch.full((n,), 0.02, device="cuda")
    g[::256] = 0.05
    opt = fm.AdamW([torch.zeros(n, device="cuda")], state_bits=8, betas=(B1, B2), seed=9)
    for _ in range(600):
        opt.step([g], 0.0)
    m, v = fm.adamw_state_values(opt.m[0], opt.v[0], opt.m_scale[0], opt.v_scale[0])
    rest = torch.ones(n, dtype=torch.bool, device="cuda")
    rest[::256] = False
    assert abs(float(m[rest].mean()) / 0.02 - 1) < 0.02
    assert abs(float(v[rest].mean()) / 0.02 ** 2 - 1) < 0.05


def test_8_bit_codes_come_from_sums_rounded_step_by_step():
    """Every product and sum of the running means rounded by itself, 65025 times the reciprocal of v's largest: the codes of
    that arithmetic and no others.  A value that one rounding less leaves a bit away can pass its random threshold, and
    where v's code is small the next update doubles or halves.  No code may differ: both sides compute the same numbers.
    (Only sqrt's last bit is not fixed, and it decides nothing: a root that falls just short of k has a remainder that
    takes it up to k but for one draw in 65536 of the values, few, that lie within a bit of a square.)"""
    n, t, seed = 1 << 22, 7, 5
    g = torch.Generator(device="cuda").manual_seed(3)
    grad = torch.empty(n, device="cuda").normal_(0, 1e-3, generator=g)
    opt = fm.AdamW([torch.zeros(n, device="cuda")], state_bits=8, betas=(B1, 0.95), eps=EPS, step=t - 1, seed=seed)
    opt.m[0].random_(0, 256, generator=g)
    opt.v[0].random_(0, 256, generator=g)
    for s in (opt.m_scale[0], opt.v_scale[0]):
        s.uniform_(1e-5, 3e-5, generator=g)
    opt.m_scale[0].copy_(torch.exp2(torch.floor(torch.log2(opt.m_scale[0]))))
    f, u = np.float32, np.uint32
    mc, vc = (x[0].cpu().numpy().reshape(-1, 256) for x in (opt.m, opt.v))
    ms, vs = (x[0].cpu().numpy().reshape(-1, 1) for x in (opt.m_scale, opt.v_scale))
    grad_h = grad.cpu().numpy().reshape(-1, 256)
    opt.step([grad], LR)
    k = (mc & 127).astype(u)
    m = np.where(k > 0, ((k + u(896)) << u(20)).view(f), f(0)) * ms
    m = np.where(mc > 127, -m, m) * f(B1) + grad_h * f(1 - B1)
    root = vc.astype(f) * vs
    v = (root * root) * f(0.95) + (grad_h * grad_h) * f(1 - 0.95)
    h = np.arange(n, dtype=np.uint64) + np.uint64(seed * 0x3504F335 + t * 0x5851F42D)
    h = h.astype(u)
    h = (h ^ (h >> u(16))) * u(0x45D9F3B5)
    h = (h ^ (h >> u(15))) * u(0x2C1B3C6D)
    r = (h ^ (h >> u(16))).reshape(-1, 256)
    top = np.abs(m).max(1, keepdims=True)
    scale = ((top.view(u) + u(0xFFFFF)) & u(0x7F800000)).view(f)
    y = np.abs(m) / scale
    c = np.clip(((y.view(u).astype(np.int64) + ((r >> u(16)).astype(np.int64) << 4)) >> 20) - 896, 0, 127)
    least = f(1.125 / 32768)
    c = np.where(y < least, (r >> u(16)).astype(f) * (least / f(65536)) < y, c) + np.where(m < 0, 128, 0)
    z = v * (f(65025) * (f(1) / v.max(1, keepdims=True)))
    low = np.floor(np.sqrt(z))
    up = (r & u(0xFFFF)).astype(f) * f(1 / 65536) * (2 * low + f(1)) < z - low * low
    d = np.clip(low + up, (v > 0).astype(f), f(255))
    assert z.dtype == f and y.dtype == f and m.dtype == f and v.dtype == f
    assert int((opt.m[0].cpu().numpy().reshape(-1, 256) != c).sum()) == 0
    assert int((opt.v[0].cpu().numpy().reshape(-1, 256) != d).sum()) == 0


def test_same_bits_again_and_other_bits_from_another_seed():
    def run(seed):
        g = torch.Generator(device="cuda")
        p = tensors([5000, 300], torch.float32, g)
        opt = fm.AdamW(p, state_bits=8, betas=(B1, B2), seed=seed)
        for _ in range(2):
            opt.step(tensors([5000, 300], torch.float32, g), LR)
        return torch.cat(opt.m + opt.v)

    a, b, c = run(1), run(1), run(2)
    assert torch.equal(a, b) and not torch.equal(a, c)


def test_non_finite_gradients_show():
    """A NaN or an infinity makes its block NaN, and no other."""
    for bad in (float("nan"), float("inf")):
        g = torch.ones(1000, device="cuda")
        g[300] = bad
        opt = fm.AdamW([torch.zeros(1000, device="cuda")], state_bits=8, betas=(B1, B2))
        opt.step([g], LR)
        m, v = fm.adamw_state_values(opt.m[0], opt.v[0], opt.m_scale[0], opt.v_scale[0])
        for x in (m, v):
            assert bool(torch.isnan(x[256:512]).all()) and not bool(torch.isnan(x[:256]).any()) and not bool(torch.isnan(x[512:]).any())


def test_zero_and_tiny_gradients():
    g = torch.zeros(512, device="cuda")
    g[256:] = 1e-25  # g^2 underflows to 0 in fp32
    opt = fm.AdamW([torch.ones(512, device="cuda")], state_bits=8, betas=(B1, B2), weight_decay=0.0)
    opt.step([g], LR)
    m, v = fm.adamw_state_values(opt.m[0], opt.v[0], opt.m_scale[0], opt.v_scale[0])
    assert bool((m[:256] == 0).all()) and bool((v == 0).all()) and bool((opt.params[0] == 1).all())
    assert bool(((m[256:].double() / 1e-26 - 1).abs() <= 1 / 8).all())


def test_more_tensors_than_a_launch_takes():
    sizes = [(37 * i) % 700 for i in range(150)]
    g = torch.Generator(device="cuda")
    p, grads = tensors(sizes, torch.float32, g), tensors(sizes, torch.float32, g)
    before = [x.clone() for x in p]
    opt = fm.AdamW(p, betas=(B1, B2), eps=EPS, weight_decay=WD)
    opt.step(grads, LR)
    for i, n in enumerate(sizes):
        z = torch.zeros(n, device="cuda")
        rp, rm, rv, upd = exact_step(before[i], grads[i], z, z, 1)
        close(p[i], rp, before[i].double().abs() + 2 * upd.abs(), 16)


def test_a_long_tensor():
    """Past 2^31 bytes, with an odd end."""
    n = (1 << 29) + 12345
    p = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g = torch.full((n,), 0.5, dtype=torch.bfloat16, device="cuda")
    opt = fm.AdamW([p], state_bits=8, betas=(B1, B2), eps=EPS)
    opt.step([g], 0.25)
    assert bool((p[-20000:] == -0.25).all()) and bool((p[:20000] == -0.25).all()) and bool((p[n // 2:n // 2 + 20000] == -0.25).all())
    assert bool((opt.m[0][-300:] > 0).all()) and bool((opt.v[0][-300:] == 255).all())


def test_refused_tensors():
    p = torch.zeros(10, device="cuda")
    for bad in (dict(params=[]), dict(params=[p.double()]), dict(params=[torch.zeros(10)]), dict(params=[p[::2]]),
                dict(params=[p], state_bits=4), dict(params=[p], states=([p[:9]], [p])), dict(params=[p], masters=[p.bfloat16()])):
        with pytest.raises(ValueError):
            fm.AdamW(**bad)
    opt = fm.AdamW([p])
    for grads in ([], [p[:9]], [p.double()], [p, p]):
        with pytest.raises(ValueError):
            opt.step(grads, LR)
    with pytest.raises(fm.FlexMoEError):
        fm.AdamW([p], masters=[p]).step([p], LR)  # a master copy of fp32 parameters
