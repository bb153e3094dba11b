"""The example that trains, synchronises and answers: what each part hands to the next."""
import importlib.util
import math
import os

import pytest
import torch

import paper_2605_06534_amd as R

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_train_and_serve():
    print("case: example", flush=True)
    spec = importlib.util.spec_from_file_location("train_and_serve", os.path.join(ROOT, "examples", "train_and_serve.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    history, right, alone, trainer, shards = m.main(steps=40)
    losses = [loss for loss, _, _ in history]
    assert abs(losses[0] - math.log(m.VOCAB)) < 1 and losses[-1] < 0.5 * losses[0]
    assert all(norm > 0 and math.isfinite(norm) and entries > 0 for _, norm, entries in history)
    clipped = math.sqrt(sum((g.double() ** 2).sum().item() for g in trainer.grads))
    assert clipped <= m.MAX_NORM * 1.00001
    # the receivers hold the trainer's weights, bit for bit, and those are the rounded masters
    for i, (w, master) in enumerate(zip(trainer.weights, trainer.master)):
        assert torch.equal(w, master.to(torch.bfloat16))
        parts = [s.weights[i].view(-1) for s in shards]
        assert all(torch.equal(p, w.view(-1)) for p in parts) if i == 1 else torch.equal(torch.cat(parts), w.view(-1))
    # a token alone and among others: the same products added up in another order, k additions that lose 2^-23 each on either side
    together = m.serve(shards, torch.arange(m.VOCAB, device="cuda"))[5:6]
    x = sum(s.rows_of(torch.tensor([5], device="cuda")) for s in shards) * trainer.weights[1]
    q, values, heads = R.Mx4(1, m.HIDDEN), torch.empty(1, m.HIDDEN, device="cuda"), []
    R.mx4_quantize(x, q)
    R.mx4_dequantize(q, values)
    for s in shards:
        heads.append(torch.empty(s.rows, m.HIDDEN, device="cuda"))
        R.mx4_dequantize(s.head, heads[-1])
    size = values.double().abs() @ torch.cat(heads).double().abs().t().contiguous()
    assert ((alone.double() - together.double()).abs() <= 2 * m.HIDDEN * 2.0 ** -23 * size).all()
    assert right > 0.9
