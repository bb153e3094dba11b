"""Temperatures whose inverse, times log2(e), is no normal number of fp32 are refused; at the borders of what is taken, results are still numbers."""
import math

import pytest
import torch

import paper_2605_06534_amd as R
from paper_2605_06534_amd import binding
from test_more_operator_refusals import ARG, BF16, F32, OK, P
from test_operator_refusals import refused

LEAST, MOST = 2.0 ** -126, 2.0 ** 126


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_refusals(dtype):
    entries = dict(z=P, zt=dtype, rows=4, cols=50, zs=50, ids=P, ib=8, teacher=P, top=3, t=1.0)
    none = dict(rows=0, z=None, ids=None, teacher=None)
    bad = [(dict(t=t), ARG) for t in (LEAST * (1 - 2.0 ** -52), 4e-39, 1e-45, 1e-300, 5e-324, MOST * (1 + 2.0 ** -52), 3e38, 1e46, 1e300)]
    good = [(dict(none, t=t), OK) for t in (LEAST, MOST, 1e-30, 1e30)]
    work = dict(ws=P, wb=1 << 20, stream=None)
    refused("rose_distill_loss", dict(entries, loss=P, lse=P, **work), bad + good)
    refused("rose_distill_grad", dict(entries, lse=P, d_loss=P, d=P, ds=50, stream=None), bad + good)
    refused("rose_distill_loss_grad", dict(entries, d_loss=P, loss=P, lse=P, d=P, ds=50, **work), bad + good)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(3, 70), (5, 6000), (1100, 3001)])
def test_at_the_borders(rows, cols, dtype):
    """d_loss = T, so that the gradient is q - p.  Very hot: as likely as one another but for masked columns; very cold: the largest alone.  (q has
    8 units of its own, the sum cols / 256 + 40 additions, the result half a step of its type; p is 1.)"""
    for t in (LEAST, MOST):
        print("case: temperature", rows, cols, dtype, t, flush=True)
        z = -1.0 - torch.rand(rows, cols, generator=torch.Generator("cuda").manual_seed(1), device="cuda").to(dtype)
        z[:, 7::11] = 0.0
        z[:, 3::5] = -math.inf
        alive = (z > -math.inf) if t == MOST else (z == 0)
        ids, teacher, d_loss = torch.full((rows, 1), 7, device="cuda"), torch.ones(rows, 1, device="cuda"), torch.full((rows,), t, device="cuda")
        loss, lse, d, ws = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(z), R.distill_workspace(rows, cols)
        n = alive.sum(1, keepdim=True).double()
        want = torch.where(alive, 1.0 / n, 0.0)
        e = want * 2.0 ** -24 * (2 * (cols / 256 + 40) + 20)
        want[:, 7] -= 1.0
        bound = (e + torch.finfo(dtype).eps / 2 * want.abs()) * (1 + 2.0 ** -8) + 2.0 ** -24 * (want.abs() > 0.5)
        for again in range(2):
            if again:
                # (the lse of a sum of n, rounded: q is off by half a unit of it)
                bound = bound + torch.where(alive, 1.0 / n, 0.0) * 2.0 ** -24 * n.log().clamp(min=1) * 2
                R.distill_grad(z, ids, teacher, lse, d_loss, d, temperature=t)
            else:
                R.distill_loss_grad(z, ids, teacher, d_loss, loss, lse, d, ws, temperature=t)
                assert ((loss.double() - n.log().view(-1)).abs() <= 1e-5 * n.log().view(-1) + 1e-6).all()
            assert ((d.double() - want).abs() <= bound).all(), (d.double() - want).abs().max()
            assert (d[z == -math.inf] == 0).all()
