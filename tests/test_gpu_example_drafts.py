"""The example's small model that drafts for the receiver: it runs, and its gradients are those of its formulas."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("train_and_serve", os.path.join(ROOT, "examples", "train_and_serve.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_drafts_are_answered(example):
    print("case: drafts", flush=True)
    *_, shards = example.main(steps=10)
    losses, tokens, accepted, _ = example.draft_and_verify(shards, steps=5)
    assert all(math.isfinite(v) and v > 0 for v in losses)
    place = torch.arange(tokens.shape[1], device="cuda")
    assert ((tokens >= 0) == (place <= accepted[:, None])).all() and (tokens < example.VOCAB).all() and ((accepted >= 0) & (accepted <= 3)).all()


def test_gradients(example):
    """Against the gradients that torch forms of the same loss in 64 bits.  The library's own parts keep fp32, as do the products, of 2048 and 64
    terms: (2048 + 300) * 2^-24 of the sums of magnitudes bounds each of the three that follow one another (products, norm, rows of a token)."""
    print("case: gradients of the draft", flush=True)
    d, g, n = example.Draft(hidden=64, top=8, seed=3), torch.Generator("cuda").manual_seed(4), 500
    tokens = torch.randint(0, example.VOCAB, (n,), generator=g, device="cuda")
    teacher, ids = (torch.randn(n, example.VOCAB, generator=g, device="cuda") * 3).topk(8, 1)
    loss, got = d.gradients(tokens, ids, teacher, temperature=2.0)
    e, w, h = (t.double().cpu().requires_grad_() for t in (d.embedding, d.norm, d.head))
    x = e[tokens.cpu()] * d.scale
    y = x * (x.square().mean(1, keepdim=True) + 1e-5).rsqrt() * w
    q, p = torch.log_softmax(y @ h.t() / 2, 1), torch.softmax(teacher.double().cpu() / 2, 1)
    want = (p * (p.log() - q.gather(1, ids.cpu()))).sum(1)
    want.mean().backward()
    assert ((loss.double().cpu() - want).abs() < 3 * 2400 * 2.0 ** -24 * (1 + want.abs())).all()
    for a, b in zip(got, (e.grad, w.grad, h.grad)):
        assert ((a.double().cpu() - b).abs() <= 3 * 2400 * 2.0 ** -24 * b.abs().max()).all()
