"""Log probabilities, entropy and the most likely tokens against their definitions in 64 bits.

Listed ids are compared for equality (value descending, id ascending).  Bounds, u = 2^-24, d = (largest - x) / temperature: a thread
sums up to ceil(range / 256) positive terms and 20 joins follow, each term off by 4 u + 2 u d of itself (where e^-d d < 0.4 it adds less than 2 u):
log s is off by (range / 256 + 30) u.  x's own part adds 3 u d, the largest's 2 u of its size to lse.  The entropy's second sum has the
same relative error on terms of size up to 1 + log V."""
import math

import pytest

torch = pytest.importorskip("torch")
from paper_2606_27866_amd import flexmoe as fm  # noqa: E402

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
NEG = -math.inf
BF16, F32 = torch.bfloat16, torch.float32


def logits_of(rows, V, dtype, seed=0, std=2.0, extra=8):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 77 + rows + V)
    wide = torch.full((rows, -(-V // 8) * 8 + extra), float("nan"), dtype=dtype, device="cuda")
    wide[:, :V] = torch.empty(rows, V, device="cuda").normal_(0, std, generator=g).to(dtype)
    return g, wide[:, :V]


def best(x, K):
    """Ids in order: value descending, NaN last, id ascending."""
    key = torch.where(torch.isnan(x), -math.inf, x.double() + 0.0)
    last = torch.isnan(x).long()  # after -inf
    first = torch.sort(key, dim=1, descending=True, stable=True).indices
    again = torch.sort(last.gather(1, first), dim=1, stable=True).indices
    return first.gather(1, again)[:, :K]


def check(x, K=0, tokens=None, temperature=1.0, max_rows=None, holder=None):
    rows, V = x.shape
    h = holder or fm.TokenLogprobs(V, rows if max_rows is None else max_rows, top=K, temperature=temperature)
    got = h(x, tokens)
    z = x.double() / temperature
    z[(z == math.inf).any(1)] = math.nan  # by definition (torch's logsumexp says inf)
    top = z.amax(1, keepdim=True)
    empty = (top == NEG).squeeze(1)
    below = z - torch.where(top == NEG, 0.0, top)  # differences first: next to 3e38 even 64 bits lose a row's logarithm
    log_s = below.exp().sum(1).log()
    lse = top.squeeze(1) + torch.where(empty, 0.0, log_s)
    lp = torch.where(empty.unsqueeze(1), NEG, below - log_s.unsqueeze(1))
    p = torch.where(z == NEG, 0.0, lp.exp())
    entropy = -(p * torch.where(p == 0, 0.0, lp)).sum(1)
    entropy = torch.where(top.squeeze(1) == NEG, 0.0, entropy)
    err = (min(V, 131072) / 256 + 30) * U
    deep = torch.where(torch.isfinite(z), (top - z).clamp(min=0), 0.0)

    def near(a, b, bound):
        a = a.double()
        assert torch.equal(torch.isnan(a), torch.isnan(b))
        whole = torch.isfinite(b)
        assert torch.equal(a[torch.isinf(b)], b[torch.isinf(b)])
        assert bool(((a - b).abs()[whole] <= bound[whole]).all()), float(((a - b).abs() / bound)[whole].max())

    near(got.lse, lse, err + 3 * U * (lse.abs() + top.squeeze(1).abs()))
    near(got.entropy, entropy, torch.full_like(entropy, 2 * (err + 20 * U) * (2 + math.log(V))))
    if tokens is not None:
        t = tokens.long()
        inside = (t >= 0) & (t < V)
        at = t.clamp(0, V - 1).unsqueeze(1)
        want = torch.where(inside, lp.gather(1, at).squeeze(1), 0.0)
        near(got.logprob, want, err + 4 * U * (deep.gather(1, at).squeeze(1) + 20))
    else:
        assert got.logprob is None
    assert got.top_ids.shape == (rows, K) and got.top_logprobs.shape == (rows, K)
    if K:
        ids = best(x, K)
        assert torch.equal(got.top_ids.long(), ids)
        near(got.top_logprobs, lp.gather(1, ids), err + 4 * U * (deep.gather(1, ids) + 20))
    return got


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,V,K", [(1, 1, 1), (3, 7, 7), (2, 8, 3), (5, 9, 1), (1, 128, 128), (4, 1000, 128), (2, 2047, 20), (1, 2048, 5), (3, 2049, 0),
                                      (1, 4097, 64), (7, 8192, 8), (70, 8200, 16), (600, 5000, 33), (2, 50001, 128), (1, 131072, 20),
                                      (3, 131073, 40), (530, 20000, 4), (2, 300007, 100)])
def test_rows(dtype, rows, V, K):
    g, x = logits_of(rows, V, dtype)
    tokens = torch.randint(0, V, (rows,), generator=g, device="cuda").int()
    check(x, K, tokens)
    check(x, 0, None, temperature=0.5)


@pytest.mark.parametrize("temperature", [1e-6, 0.01, 0.7, 3.0, 1e6])
def test_temperatures(temperature):
    g, x = logits_of(5, 3000, F32)
    check(x, 10, torch.arange(5, device="cuda").int(), temperature)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V", [500, 5000, 70000, 140000])
def test_order_of_the_values(dtype, V):
    """Equal values, a few different ones, sorted rows, the largest values side by side, -0 beside 0: ties go to the lower id."""
    i = torch.arange(V, device="cuda")
    rows = [torch.zeros(V, device="cuda"), -(i % 3).float(), i / V * 10, -i / V * 10, (i < 200).float() * (i % 7), ((i >= V - 300) * (i % 5)).float(),
            torch.where(i % 2 == 0, 0.0, -0.0), (i % 256 == 3).float()]
    x = fm._padded((len(rows), V), dtype, "cuda").copy_(torch.stack(rows))
    for K in (1, 40, 128):
        check(x, K)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,V", [(12, 3000), (12, 40000), (12, 140000)])
def test_masks_and_values_that_are_no_numbers(dtype, rows, V):
    low = torch.finfo(dtype).min
    g, x = logits_of(rows, V, dtype)
    x[0] = NEG
    x[1, 5:] = NEG                       # fewer than are listed
    x[2, torch.rand(V, generator=g, device="cuda") < 0.9] = NEG
    x[3, V // 2] = float("nan")
    x[4, 7] = float("inf")
    x[5] = low
    x[6, 3:] = low
    x[7] = torch.finfo(dtype).max
    x[8, 10] = torch.finfo(dtype).max
    x[9, : V // 2] = NEG
    x[10] = float("nan")
    tokens = torch.tensor([0, 2, 5, 1, 7, 4, 1, V - 1, 10, 3, 0, V], device="cuda").int()
    check(x, 20, tokens)
    check(x[:1], 20, tokens[:1])
    check(x[3:4], 20, tokens[3:4])


def test_tokens_outside_the_vocabulary():
    _, x = logits_of(4, 100, F32)
    got = check(x, 2, torch.tensor([-1, 100, -100, 2 ** 31 - 1], device="cuda").int())
    assert bool((got.logprob == 0).all())


def test_deterministic_and_smaller_calls():
    """The same bits again, and from a holder for more rows; fewer rows in more parts give the same ids."""
    _, x = logits_of(40, 30000, BF16)
    a, b = fm.TokenLogprobs(30000, 40, top=30), fm.TokenLogprobs(30000, 5000, top=30)
    first = a(x)
    for h in (a, b):
        again = h(x)
        assert all(torch.equal(p, q) for p, q in zip(again[1:], first[1:]))
    assert torch.equal(a(x[:1]).top_ids, first.top_ids[:1])


def test_offsets_past_32_bits():
    V, rows = 131080, 16500  # 2.16e9 values
    x = torch.zeros(rows, V, dtype=BF16, device="cuda")
    x[-1, 77], x[-2, V - 1] = 9.0, 8.0
    got = fm.TokenLogprobs(V, rows, top=1)(x, torch.full((rows,), 77, dtype=torch.int32, device="cuda"))
    assert int(got.top_ids[-1, 0]) == 77 and int(got.top_ids[-2, 0]) == V - 1
    ref = torch.log_softmax(x[-2:].double(), 1)[:, 77]
    assert bool(((got.logprob[-2:].double() - ref).abs() < 1e-4).all())


def test_no_rows():
    got = fm.TokenLogprobs(100, 4, top=3)(torch.empty(0, 104, device="cuda")[:, :100])
    assert got.lse.shape == (0,) and got.top_ids.shape == (0, 3)
