"""A few rows of bf16 activations with many rows of weights, on either side of where the product no longer quantises the
activations itself: whole numbers with equal scales, whose sums are exact."""
import pytest
import torch

import paper_2605_06534_amd as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,n,k", [(5, 32768, 1024), (8, 32768, 1024), (8, 32769, 1024), (8, 16384, 2048), (8, 16400, 2048), (6, 70000, 511),
                                   (8, 32768, 33), (4, 40000, 2048)])
def test_few_rows_with_many_weights(m, n, k):
    print("case: few rows, many weights", m, n, k, flush=True)
    g = torch.Generator("cuda").manual_seed(94)
    # (4 in each block: its scale is 1)
    x = torch.randint(-4, 5, (m, k), generator=g, device="cuda").to(torch.bfloat16)
    w = torch.randint(-4, 5, (n, k), generator=g, device="cuda").to(torch.bfloat16)
    x[:, ::32], w[:, ::32] = 4, 4
    q, out = R.Mx4(n, k), torch.empty(m, n, device="cuda")
    R.mx4_quantize(w, q)
    R.mx4_linear(x, q, out, R.mx4_linear_workspace(m, n, k))
    assert torch.equal(out.double(), x.double() @ w.double().t().contiguous())
