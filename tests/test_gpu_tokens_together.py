"""The operators between hidden states and tokens one behind the other, as a receiver that verifies drafts and a student that learns use
them: on another stream, in graphs of their own, and with data beyond 2^32 bytes."""
import pytest
import torch

import paper_2605_06534_amd as R

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def normal(*shape, seed, std=1.0, dtype=torch.bfloat16):
    return (torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda") * std).to(dtype)


class Pass:
    """Hidden states to verified tokens, and the loss and gradients of a student that drafts."""

    def __init__(self, requests, most, hidden, vocab, rank=8, adapters=5, top=16, seed=1):
        g = torch.Generator("cuda").manual_seed(seed)
        lengths = torch.arange(requests, device="cuda") % (most + 1)
        self.offsets = torch.cat((torch.zeros(1, dtype=torch.int64, device="cuda"), lengths.cumsum(0)))
        n = int(self.offsets[-1])
        rows = n + requests
        self.x, self.weight, self.bias = normal(rows, hidden, seed=seed), normal(hidden, seed=seed + 1, std=0.1) + 1, normal(hidden, seed=seed + 2)
        self.head = R.Mx4(vocab, hidden)
        R.mx4_quantize(normal(vocab, hidden, seed=seed + 3, std=hidden ** -0.5), self.head)
        self.adapters = R.Adapters(normal(adapters, rank, hidden, seed=seed + 4, std=hidden ** -0.5), normal(adapters, vocab, rank, seed=seed + 5, std=rank ** -0.5),
                                   torch.rand(adapters, generator=g, device="cuda"))
        self.chosen = torch.randint(-1, adapters, (rows,), generator=g, device="cuda").int()
        self.drafted, self.u = torch.randint(0, vocab, (n,), generator=g, device="cuda"), torch.rand(rows, generator=g, device="cuda")
        self.draft = torch.softmax(normal(n, vocab, seed=seed + 6, dtype=torch.float32), 1)
        self.student, self.top = normal(rows, vocab, seed=seed + 7, std=2.0), top
        self.d_loss = torch.full((rows,), 1.0 / rows, device="cuda")
        self.ws = (R.mx4_linear_workspace(rows, vocab, hidden), R.adapter_linear_workspace(rows, self.adapters), R.draft_verify_workspace(requests, vocab),
                   R.distill_workspace(rows, vocab), R.layer_norm_grad_workspace(rows, hidden))
        e = torch.empty
        f32 = dict(device="cuda")
        self.y, self.mean, self.rstd, self.logits = torch.empty_like(self.x), e(rows, **f32), e(rows, **f32), e(rows, vocab, **f32)
        self.p, self.tokens, self.accepted = e(rows, vocab, **f32), e(rows, dtype=torch.int64, device="cuda"), e(requests, dtype=torch.int32, device="cuda")
        self.ids, self.teacher = e(rows, top, dtype=torch.int64, device="cuda"), e(rows, top, **f32)
        self.loss, self.lse, self.d, self.dx, self.dw, self.db = e(rows, **f32), e(rows, **f32), torch.empty_like(self.student), torch.empty_like(self.x), e(hidden, **f32), e(hidden, **f32)
        self.results = (self.y, self.mean, self.rstd, self.logits, self.tokens, self.accepted, self.ids, self.loss, self.lse, self.d, self.dx, self.dw, self.db)

    def run(self):
        R.layer_norm(self.x, self.weight, self.y, bias=self.bias, mean=self.mean, rstd=self.rstd)
        R.mx4_linear(self.y, self.head, self.logits, self.ws[0])
        R.adapter_linear(self.y, self.adapters, self.chosen, self.logits, self.ws[1])
        self.p.copy_(torch.softmax(self.logits, 1))
        R.draft_verify(self.p, self.draft, self.drafted, self.offsets, self.u, self.tokens, self.accepted, self.ws[2])
        teacher, ids = self.logits.topk(self.top, 1)
        self.ids.copy_(ids), self.teacher.copy_(teacher)
        R.distill_loss_grad(self.student, self.ids, self.teacher, self.d_loss, self.loss, self.lse, self.d, self.ws[3])
        R.layer_norm_grad(self.y, self.x, self.weight, self.rstd, self.dx, self.dw, self.ws[4], mean=self.mean, dbias=self.db)

    def taken(self):
        self.run()
        torch.cuda.synchronize()
        return [t.clone() for t in self.results]


@pytest.mark.parametrize("requests,most,hidden,vocab", [(1, 3, 64, 1000), (40, 4, 320, 3000), (300, 5, 512, 4099)])
def test_a_pass_and_its_parts(requests, most, hidden, vocab):
    print("case: together", requests, hidden, vocab, flush=True)
    p = Pass(requests, most, hidden, vocab)
    p.taken()
    # each hands to the next what the formulas say (bounds as in the parts' own tests, the products by their own differences)
    x = p.x.double()
    y = (x - x.mean(1, keepdim=True)) * (x.var(1, unbiased=False, keepdim=True) + 1e-5) ** -0.5 * p.weight.double() + p.bias.double()
    assert ((p.y.double() - y).abs() <= 2.0 ** -8 * y.abs() + 2 * (hidden / 64 + 60) * U * (1 + y.abs())).all()
    shared = torch.empty_like(p.logits)
    R.mx4_linear(p.y, p.head, shared, p.ws[0])
    delta = torch.zeros_like(p.logits, dtype=torch.float64)
    size = torch.zeros_like(delta)
    for a in range(5):
        rows = (p.chosen == a).nonzero().view(-1)
        d, u, v = p.adapters.down[a].double(), p.adapters.up[a].double(), p.y[rows].double()
        delta[rows] = p.adapters.scales[a].double() * ((v @ d.t().contiguous()) @ u.t().contiguous())
        size[rows] = p.adapters.scales[a].double() * ((v.abs() @ d.abs().t().contiguous()) @ u.abs().t().contiguous())
    assert ((p.logits.double() - shared.double() - delta).abs() <= (hidden + 20) * 2.0 ** -23 * size + 2.0 ** -22 * (shared.double().abs() + delta.abs())).all()
    assert ((p.tokens >= 0).sum() == p.accepted.sum() + requests) and (p.tokens < vocab).all()
    q, t = torch.log_softmax(p.student.double(), 1), torch.softmax(p.teacher.double(), 1)
    loss = (t * (torch.log(t) - q.gather(1, p.ids))).sum(1)
    assert ((p.loss.double() - loss).abs() <= U * (2 * (vocab / 256 + 60) + 4 * 20) + U * loss.abs()).all()
    grad = torch.exp(q).scatter_add_(1, p.ids, -t) * p.d_loss.double()[:, None]
    assert ((p.d.double() - grad).abs() <= 2.0 ** -8 * grad.abs() + U * (2 * (vocab / 256 + 60) + 100) * p.d_loss.double()[:, None]).all()


def test_on_a_stream_of_their_own_behind_other_work():
    print("case: another stream", flush=True)
    p = Pass(50, 4, 320, 3000, seed=5)
    want = p.taken()
    for t in p.results:
        t.fill_(3)
    busy, stream = torch.randn(3000, 3000, device="cuda"), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        for _ in range(20):
            torch.mm(busy, busy)
        p.run()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, p.results))
    # the same by argument
    other = torch.empty_like(p.y)
    R.layer_norm(p.x, p.weight, other, bias=p.bias, stream=stream)
    out = p.logits.clone()
    torch.cuda.synchronize()
    R.adapter_linear(p.y, p.adapters, p.chosen, out, p.ws[1], stream=stream)
    stream.synchronize()
    assert torch.equal(other, p.y)


def test_two_graphs_with_workspaces_of_their_own_on_two_streams():
    print("case: two graphs", flush=True)
    passes, graphs, streams = [Pass(30, 4, 320, 2000, seed=s) for s in (10, 30)], [], []

    def own(p):
        R.layer_norm(p.x, p.weight, p.y, bias=p.bias, mean=p.mean, rstd=p.rstd)
        R.adapter_linear(p.y, p.adapters, p.chosen, p.logits, p.ws[1])
        R.draft_verify(p.draft_rows, p.draft, p.drafted, p.offsets, p.u, p.tokens, p.accepted, p.ws[2])
        R.distill_loss_grad(p.student, p.ids, p.teacher, p.d_loss, p.loss, p.lse, p.d, p.ws[3])
        R.layer_norm_grad(p.y, p.x, p.weight, p.rstd, p.dx, p.dw, p.ws[4], mean=p.mean, dbias=p.db)

    for p in passes:
        p.taken()
        p.draft_rows = p.p.clone()
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            own(p)
        graphs.append(graph), streams.append(stream)
    for turn in range(3):
        want = []
        for i, p in enumerate(passes):
            p.x.copy_(normal(*p.x.shape, seed=100 + 2 * turn + i))
            p.logits.zero_()
            own(p)
            want.append([t.clone() for t in p.results])
            p.logits.zero_()
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for p, w in zip(passes, want):
            assert all(torch.equal(a, b) for a, b in zip(w, p.results))


def test_norms_and_distillation_beyond_4_gb():
    print("case: beyond 4 GB", flush=True)
    rows, cols = 140000, 16384                          # 2.29 G elements
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    pattern = normal(7, cols, seed=1)
    for i in range(7):
        x[i::7] = pattern[i]
    w, out, rstd = torch.ones(cols, dtype=torch.bfloat16, device="cuda"), torch.empty_like(x), torch.empty(rows, device="cuda")
    R.layer_norm(x, w, out, rstd=rstd, center=False)
    for i in range(7):
        assert (out[i::7] == out[i]).all() and (rstd[i::7] == rstd[i]).all()
    dw, ws = torch.empty(cols, device="cuda"), R.layer_norm_grad_workspace(rows, cols)
    R.layer_norm_grad(x, x, w, rstd, out, dw, ws)
    assert all((out[i::7] == out[i]).all() for i in range(7))
    want = ((pattern.double() ** 2) * rstd[:7, None].double() * (rows // 7)).sum(0)
    assert ((dw.double() - want).abs() <= (rows + 4) * U * want).all()
    ids, teacher, d_loss = torch.randint(0, cols, (7, 4), generator=torch.Generator("cuda").manual_seed(2), device="cuda").repeat(rows // 7, 1), torch.ones(rows, 4, device="cuda"), torch.ones(rows, device="cuda")
    loss, lse, ws = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), R.distill_workspace(rows, cols)
    R.distill_loss_grad(x, ids, teacher, d_loss, loss, lse, out, ws)
    for i in range(7):
        assert (out[i::7] == out[i]).all() and (loss[i::7] == loss[i]).all() and (lse[i::7] == lse[i]).all()
    assert ((lse[:7].double() - torch.logsumexp(pattern.double(), 1)).abs() < 1e-5).all()
    R.distill_grad(x, ids, teacher, lse, d_loss, x)
    assert all((x[i::7] == x[i]).all() for i in range(7))


def test_probabilities_beyond_4_gb():
    print("case: probabilities beyond 4 GB", flush=True)
    requests, length, cols = 3000, 4, 152064            # 15000 rows of 304 KB
    target = torch.zeros(requests * (length + 1), cols, dtype=torch.bfloat16, device="cuda")
    at = torch.randint(0, cols, (len(target),), generator=torch.Generator("cuda").manual_seed(3), device="cuda")
    target[torch.arange(len(target), device="cuda"), at] = 1.0
    offsets = torch.arange(requests + 1, device="cuda") * length
    drafted = at.view(requests, length + 1)[:, :length].reshape(-1).clone()
    drafted[2::length * 3] += 1                         # the third token of each third request
    tokens, accepted = torch.empty(len(target), dtype=torch.int64, device="cuda"), torch.empty(requests, dtype=torch.int32, device="cuda")
    R.draft_verify(target, None, drafted, offsets, torch.full((len(target),), 0.5, device="cuda"), tokens, accepted, R.draft_verify_workspace(requests, cols))
    third = torch.arange(requests, device="cuda") % 3 == 0
    assert (accepted == torch.where(third, 2, length)).all()
    want = at.view(requests, length + 1).clone()
    want[third, 3:] = -1
    assert torch.equal(tokens.view(requests, -1), want)


def test_host_memory_is_refused():
    print("case: host memory", flush=True)
    p = Pass(3, 2, 64, 500, seed=40)
    p.taken()
    for call in (lambda: R.layer_norm(p.x.cpu(), p.weight, p.y), lambda: R.layer_norm(p.x, p.weight, p.y, rstd=p.rstd.cpu()),
                 lambda: R.layer_norm_grad(p.y, p.x, p.weight, p.rstd.cpu(), p.dx, p.dw, p.ws[4]), lambda: R.layer_norm_grad(p.y, p.x, p.weight, p.rstd, p.dx, p.dw.cpu(), p.ws[4]),
                 lambda: R.distill_loss(p.student, p.ids.cpu(), p.teacher, p.loss, p.lse, p.ws[3]), lambda: R.distill_loss(p.student, p.ids, p.teacher, p.loss.cpu(), p.lse, p.ws[3]),
                 lambda: R.distill_loss(p.student, p.ids, p.teacher, p.loss, p.lse, p.ws[3].cpu()),
                 lambda: R.draft_verify(p.p, p.draft.cpu(), p.drafted, p.offsets, p.u, p.tokens, p.accepted, p.ws[2]),
                 lambda: R.draft_verify(p.p, p.draft, p.drafted, p.offsets.cpu(), p.u, p.tokens, p.accepted, p.ws[2]),
                 lambda: R.adapter_linear(p.y, p.adapters, p.chosen.cpu(), p.logits, p.ws[1]),
                 lambda: R.adapter_linear(p.y, R.Adapters(p.adapters.down, p.adapters.up.cpu()), p.chosen, p.logits, p.ws[1])):
        with pytest.raises(R.RoseError) as e:
            call()
        assert e.value.status == 2
