"""Columns of minus infinity beside columns of the type's lowest value and nothing else: the lowest ones have all of the probability, minus
infinity none, in the gradient from an lse as well."""
import math

import pytest
import torch

import paper_2605_06534_amd as R


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(3, 70), (5, 6000), (1100, 3001)])
@pytest.mark.parametrize("temperature", [1.0, 0.7, 3.0])
def test_minus_infinity_beside_the_lowest_value(rows, cols, dtype, temperature):
    print("case: lowest values", rows, cols, dtype, temperature, flush=True)
    z = torch.full((rows, cols), -math.inf, dtype=dtype, device="cuda")
    z[:, 5:9] = torch.finfo(dtype).min
    ids, teacher = torch.full((rows, 1), 6, device="cuda"), torch.ones(rows, 1, device="cuda")
    loss, lse, d_loss = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.ones(rows, device="cuda")
    d, ws = torch.full_like(z, 7.0), R.distill_workspace(rows, cols)
    R.distill_loss_grad(z, ids, teacher, d_loss, loss, lse, d, ws, temperature=temperature)
    masked = z == -math.inf
    # (the four have a quarter each: a power of two, of which d_loss / T is one rounding of 24 bits, and the result's)
    half = torch.finfo(dtype).eps / 2 + 2.0 ** -22
    want = torch.tensor([0.25, -0.75, 0.25, 0.25], dtype=torch.float64, device="cuda") / temperature
    assert (d[masked] == 0).all() and ((d[:, 5:9].double() - want).abs() <= half * want.abs()).all()
    d.fill_(7.0)
    if temperature == 1.0:                        # (else lse itself, of 3.4e38 / T and more, may be beyond fp32, or tell nothing of the columns)
        R.distill_grad(z, ids, teacher, lse, d_loss, d, temperature=temperature)
        assert (d[masked] == 0).all()
