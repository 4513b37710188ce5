"""Norm, router, log probabilities and distillation as they are used together: a block trained against its teacher, a block
served in 8 bits, and each of them on other streams, in graphs and in threads.

A chain of fp32 stages: every stage's result is within (terms of its longest sum) units of 2^-24 of its inputs' norms: 64 for
the products over d, 1000 for those over V, below 100 for the operators (their own tests).  The weights keep each stage's norm
below 4 times its input's, and the longest path has eight stages: 1000 * 2^-24 * 4 ~ 2.4e-4 would be reached only if all
roundings pointed one way; gradients are held to 1e-4 of their largest value."""
import threading

import pytest

torch = pytest.importorskip("torch")
from paper_2606_27866_amd import flexmoe as fm  # noqa: E402

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
NEG = float("-inf")


class Block:
    """x + delta -> norm -> router -> experts tanh(y a_e) -> residual -> norm -> head -> distillation, and all gradients."""

    def __init__(self, T=70, d=64, E=8, k=2, V=1000, K=16, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape, std=1.0):
            return torch.empty(shape, device="cuda").normal_(0, std, generator=g)

        self.T, self.k, self.V = T, k, V
        self.x, self.delta = normal(T, d), normal(T, d)
        self.n1, self.n2 = 1 + normal(d, std=0.1), 1 + normal(d, std=0.1)
        self.wr, self.a, self.wh = normal(d, E, std=d ** -0.5), normal(E, d, std=0.5), normal(d, V, std=d ** -0.5)
        self.bias = normal(E, std=0.05)
        self.teacher = normal(T, V, std=2)
        self.labels = torch.randint(0, V, (T,), generator=g, device="cuda").int()
        self.scale = torch.full((T,), 1.0 / T, device="cuda")
        self.scale[-1] = 0  # padding
        self.norm1, self.norm2 = fm.RMSNorm(self.n1, T), fm.RMSNorm(self.n2, T)
        self.router = fm.Router(E, k, T, score="sigmoid", scale=1.5, groups=4, top_groups=2, group_best=1)
        self.list = fm.TokenLogprobs(V, T, top=K, temperature=2.0)
        self.loss = fm.Distillation(V, K, T, temperature=2.0, tail=True, ce_weight=0.5)

    def step(self, stream=None):
        """Losses and the gradients of x (delta's is the same), both norms' weights, the router's and the head's."""
        kw = dict(stream=stream)
        t = self.list(self.teacher, **kw)
        y, r, rstd = self.norm1.forward(self.delta, self.x, **kw)
        rl = y @ self.wr
        rl[-1] = NEG
        R = self.router.route(rl, self.bias, **kw)
        ids, w = R.topk_idx.clamp(min=0).long(), R.topk_w
        o = torch.tanh(y.unsqueeze(1) * self.a[ids])
        c = (w.unsqueeze(2) * o).sum(1)
        z, r2, rstd2 = self.norm2.forward(c, r, **kw)
        logits = z @ self.wh
        kl, ce, dl = self.loss.gradient(logits, t.top_ids, t.top_logprobs, self.labels, self.scale, **kw)
        dwh, dz = z.T @ dl, dl @ self.wh.T
        dr, dn2 = self.norm2.backward(dz, r2, rstd2, **kw)
        dw = (dr.unsqueeze(1) * o).sum(2).contiguous()
        dy = (w.unsqueeze(2) * dr.unsqueeze(1) * (1 - o * o) * self.a[ids]).sum(1)
        drl = self.router.backward(rl, R.topk_idx, dw, **kw)
        dx, dn1 = self.norm1.backward(dy + drl @ self.wr.T, r, rstd, dr=dr, **kw)
        return kl, ce, dx, dn1, dn2, y.T @ drl, dwh, R.topk_idx

    def exact(self, ids):
        x, n1, n2, wr, wh = [p.double().requires_grad_() for p in (self.x, self.n1, self.n2, self.wr, self.wh)]
        r = (self.delta + self.x).double() - self.x.double() + x  # the rounded sum, as a function of x

        def norm(v, weight):
            return v * torch.rsqrt(v.square().mean(1, keepdim=True) + 1e-6) * weight

        y = norm(r, n1)
        s = torch.sigmoid(y @ wr).gather(1, ids.clamp(min=0).long()) * (ids >= 0)
        w = 1.5 * s / s.sum(1, keepdim=True).clamp(min=1e-30)
        c = (w.unsqueeze(2) * torch.tanh(y.unsqueeze(1) * self.a.double()[ids.clamp(min=0).long()])).sum(1)
        logits = norm(c + r, n2) @ wh
        lp, at = torch.log_softmax(self.teacher.double() / 2, 1).topk(16, 1)
        logq, p = torch.log_softmax(logits / 2, 1), lp.exp()
        rest, qrest = 1 - p.sum(1), 1 - logq.gather(1, at).exp().sum(1)
        kl = (p * (lp - logq.gather(1, at))).sum(1) + rest * (rest.log() - qrest.log())
        ce = -torch.log_softmax(logits, 1).gather(1, self.labels.long().unsqueeze(1)).squeeze(1)
        (self.scale.double() * (4 * kl + 0.5 * ce)).sum().backward()
        on = self.scale != 0
        return kl.detach() * on, ce.detach() * on, x.grad, n1.grad, n2.grad, wr.grad, wh.grad


def same(a, b):
    return all(torch.equal(p, q) for p, q in zip(a, b))


def test_block_and_its_gradients():
    b = Block()
    got = b.step()
    assert bool((got[7][-1] == -1).all()) and bool((got[7][:-1] >= 0).all())
    for name, a, ref in zip(("kl", "ce", "x", "norm 1", "norm 2", "router", "head"), got, b.exact(got[7])):
        assert float((a.double() - ref).abs().max()) <= 1e-4 * float(ref.abs().max()), name
    assert not bool(got[2][-1].any())  # padding has no gradient


def test_block_twice_keeps_the_first_results():
    b = Block()
    first = b.step()
    kept = [t.clone() for t in first]
    b.x.neg_()
    second = b.step()
    torch.cuda.synchronize()
    assert same(first, kept) and not same(first, second)


def test_block_on_another_stream():
    b = Block()
    want = b.step()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    busy = torch.randn(4096, 4096, device="cuda")
    for _ in range(3):
        for _ in range(4):
            busy = busy @ busy * 1e-3  # the current stream's own work goes on meanwhile
        with torch.cuda.stream(s):
            got = b.step()
        s.synchronize()
        assert same(want, got)
    torch.cuda.synchronize()
    # the operators' `stream` alone: outputs are made on it
    x = b.teacher
    want = b.list(x)
    torch.cuda.synchronize()
    for handle in (s, s.cuda_stream):
        got = b.list(x, stream=handle)
        R = b.router.route(x[:, :8].contiguous(), stream=handle)
        y, r, rstd = b.norm1.forward(b.delta, b.x, stream=handle)
        s.synchronize()
        assert same([t for t in want if t is not None], [t for t in got if t is not None])
        assert R.topk_idx.shape == (70, 2) and same((y, r, rstd), b.norm1.forward(b.delta, b.x))


def test_captured_and_replayed_between_eager_calls():
    """Two graphs and eager calls share the holders' workspaces, one after another on one stream."""
    b, other = Block(), Block(seed=1)
    b.step(), other.step()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graphs, outs = [], []
    for inputs in (b.x, other.x):
        b.x = inputs
        with torch.cuda.stream(s):
            b.step()
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            outs.append(b.step())
        graphs.append((graph, inputs))
    torch.cuda.synchronize()
    for turn in range(4):
        for (graph, inputs), out in zip(graphs, outs):
            inputs.mul_(-0.5)
            b.labels.copy_((b.labels + 17) % b.V)
            graph.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in out]
            b.x = inputs
            assert same(got, b.step()), turn


def test_holders_shared_by_threads():
    b = Block()
    x = [torch.randn(70, 64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(i)) for i in range(4)]
    big = [torch.randn(70, 1000, device="cuda", generator=torch.Generator(device="cuda").manual_seed(i)) for i in range(4)]

    def calls(i):
        bf = x[i].to(BF16)
        return (*b.norm1.forward(x[i], b.x), *b.norm1.quantized(bf), *b.router.route(x[i][:, :8].contiguous()), *b.list(big[i])[1:],
                *b.list(big[i].to(BF16))[1:])

    want = [calls(i) for i in range(4)]
    torch.cuda.synchronize()
    got, failed = [None] * 4, []

    def work(i):
        try:
            for _ in range(30):
                got[i] = calls(i)
        except BaseException as e:  # noqa: BLE001  (a thread's failure is the test's)
            failed.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed
    for w, g in zip(want, got):
        assert same(w, g)


@pytest.mark.parametrize("T", [1, 9, 300])
def test_block_served_in_8_bits(T):
    """Norm with rows in 8 bits, router, and the experts' 8-bit products of the routed rows: whole numbers all the way, so the
    product is that of the rounded values up to its own rounding to bf16 (2^-8) and the scales' (a few 2^-24)."""
    E, k, d, N = 12, 3, 256, 136
    g = torch.Generator(device="cuda").manual_seed(T)
    x, res = (torch.empty(T, d, device="cuda").normal_(0, 1, generator=g).to(BF16) for _ in range(2))
    norm = fm.RMSNorm(torch.empty(d, device="cuda").normal_(1, 0.2, generator=g).to(BF16), T)
    wr = torch.empty(d, E, device="cuda").normal_(0, 0.1, generator=g)
    experts = fm.Int8Product.from_weights(torch.empty(E, N, d, device="cuda").normal_(0, 0.1, generator=g).to(BF16), T * k)
    y, q, scale, r = norm.both(x, res)
    R = fm.Router(E, k, T).route(y.float() @ wr)
    token = (R.perm // k).long()  # no id is masked: every slot has its row
    out = experts.product(q[token].contiguous(), scale[token], R.offsets)
    e_of = torch.repeat_interleave(torch.arange(E, device="cuda"), R.counts.long())
    whole = torch.stack([experts.w[e].double() @ q[t].double() for e, t in zip(e_of.tolist(), token.tolist())])  # exact
    ref = whole * experts.w_scale.view(E, N).double()[e_of] * scale.double()[token].unsqueeze(1)
    assert bool(((out.double() - ref).abs() <= (2.0 ** -8 + 16 * 2.0 ** -24) * ref.abs() + 1e-30).all())
    assert torch.equal(e_of.int(), R.topk_idx.view(-1)[R.perm.long()])
    assert torch.equal(R.pos[R.perm.long()].long(), torch.arange(T * k, device="cuda"))


def test_routing_feeds_the_grouped_products():
    """Tokens without an expert and masked experts: the products' groups end before the rows that go nowhere."""
    E, k, d, T = 16, 4, 128, 333
    g = torch.Generator(device="cuda").manual_seed(5)
    logits = torch.empty(T, E, device="cuda").normal_(0, 1, generator=g)
    logits[::7] = NEG
    logits[:, 5] = NEG
    R = fm.Router(E, k, T).route(logits)
    rows = int(R.offsets[-1])
    assert rows == k * int((torch.arange(T) % 7 != 0).sum()) and int(R.counts[5]) == 0
    assert bool((R.perm[rows:] == -1).all()) and bool((R.pos.view(T, k)[::7] == -1).all())
    x = torch.empty(T, d, device="cuda").normal_(0, 1, generator=g).to(BF16)
    w = torch.empty(E, 64, d, device="cuda").normal_(0, 0.1, generator=g).to(BF16)
    out = fm.GroupedProduct(E, 64, d, T * k).forward(x[(R.perm.clamp(min=0) // k).long()], w, R.offsets)
    got = out[R.pos.clamp(min=0).long()].view(T, k, 64).double()
    ids = R.topk_idx.clamp(min=0).long()
    ref = (w.double().cpu()[ids.cpu()] @ x.double().cpu().view(T, 1, d, 1)).squeeze(3).cuda()
    size = (w.double().abs().cpu()[ids.cpu()] @ x.double().abs().cpu().view(T, 1, d, 1)).squeeze(3).cuda()
    on = (R.topk_idx >= 0).unsqueeze(2)
    # fp32 sums of 128 exact products, then one rounding to bf16
    assert bool(((got - ref).abs() <= 2.0 ** -8 * ref.abs() + 130 * 2.0 ** -24 * size)[on.expand_as(ref)].all())


def test_a_teacher_lists_and_an_optimizer_steps_in_one_graph():
    """Logits as parameters: list, loss and update captured together; each replay equals the eager step from the same state."""
    R, V, K = 33, 5000, 32
    g = torch.Generator(device="cuda").manual_seed(3)
    teacher = torch.empty(R, V, device="cuda").normal_(0, 2, generator=g).to(BF16)
    p = torch.empty(R, V, device="cuda").normal_(0, 2, generator=g)
    q = p.clone()
    lists, loss = fm.TokenLogprobs(V, R, top=K), fm.Distillation(V, K, R, tail=True)
    opts = [fm.AdamW([t], device_step=True) for t in (p, q)]

    def step(t, opt):
        top = lists(teacher)
        kl, ce, d = loss.gradient(t, top.top_ids, top.top_logprobs)
        opt.step([d], 1e-2)
        return kl

    step(p, opts[0]), step(q, opts[1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kl = step(p, opts[0])
    for _ in range(4):
        graph.replay()
        torch.cuda.synchronize()
        want = step(q, opts[1])
        assert torch.equal(kl, want) and torch.equal(p, q)
    assert bool(torch.isfinite(p).all())


@pytest.mark.parametrize("cols", [64, 2048, 20000])
@pytest.mark.parametrize("onto", ["dy", "dr"])
def test_input_gradient_in_place(cols, onto):
    g = torch.Generator(device="cuda").manual_seed(cols)
    dy, r, dr = (torch.empty(1500, cols, device="cuda").normal_(0, 1, generator=g).to(BF16) for _ in range(3))
    n = fm.RMSNorm(torch.ones(cols, device="cuda"), 1500)
    rstd = torch.ones(1500, device="cuda")
    want, dw = n.backward(dy, r, rstd, dr=dr)
    into = dict(dy=dy, dr=dr)[onto]
    dx, dw2 = n.backward(dy, r, rstd, dr=dr, dx=into)
    assert dx is into and torch.equal(dx, want) and torch.equal(dw, dw2)
