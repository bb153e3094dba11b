"""Products of 4-bit matrices whose sums are exact, in every way that a product may go: values of the format with scales of 1/2, 1 and
2 where k is at most 7000 (multiples of 1/16 whose magnitudes add up to at most 144 k, fewer than 2^24 sixteenths), of 1 beyond
(multiples of 1/4 that add up to at most 36 k).  Every partial sum is a number of fp32 in any order, so one element lost, or
multiplied with another block's scale, shows."""
import pytest
import torch

import paper_2605_06534_amd as R

pytestmark = pytest.mark.gpu

MAGNITUDES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def matrix(rows, k, seed):
    """Values of the format, and the 4-bit matrix of them."""
    g = torch.Generator("cuda").manual_seed(seed)
    x = torch.tensor(MAGNITUDES, device="cuda")[torch.randint(0, 8, (rows, k), generator=g, device="cuda")]
    x *= torch.randint(0, 2, (rows, k), generator=g, device="cuda") * 2 - 1
    if k <= 7000:
        blocks = -(-k // 32)
        x *= torch.exp2(torch.randint(-1, 2, (rows, blocks), generator=g, device="cuda").float()).repeat_interleave(32, 1)[:, :k]
    q, back = R.Mx4(rows, k), torch.empty_like(x)
    R.mx4_quantize(x, q)
    R.mx4_dequantize(q, back)
    assert torch.equal(back, x)
    return x, q


# rows: taken in by the product itself (1 to 8), 16, 32, 64 at a time, divided sums of more, tiles of 64, 128 and 256
@pytest.mark.parametrize("m,n,k", [(1, 1, 9001), (1, 300, 1), (1, 6912, 5120), (3, 77, 4083), (4, 1003, 14336), (5, 500, 2048), (8, 130, 1025), (7, 90, 33),
                                   (9, 400, 5120), (16, 1003, 4083), (16, 20000, 1056), (17, 6143, 2080), (31, 6145, 5121), (32, 300, 9001),
                                   (33, 500, 4096), (47, 4099, 4083), (64, 9003, 5120), (64, 60, 31), (50, 7000, 9001),
                                   (65, 100, 5121), (128, 4096, 2080), (130, 1000, 14336), (513, 900, 4100),
                                   (65, 70, 31), (100, 1003, 1024), (300, 1700, 2048), (700, 1500, 5120), (700, 1500, 5100), (1500, 1500, 288),
                                   (256, 19008, 5120), (1600, 2100, 1024), (1600, 2100, 4083), (129, 26000, 992),
                                   (3400, 3600, 1024), (3329, 3841, 5120), (3500, 3500, 5121), (300, 49000, 1000), (49000, 300, 96)])
def test_exact_products(m, n, k):
    print("case: exact product", m, n, k, flush=True)
    (x, qx), (w, qw) = matrix(m, k, 121), matrix(n, k, 122)
    want = (x.double() @ w.double().t().contiguous()).float()
    ws = R.mx4_linear_workspace(m, n, k)
    for dtype in (torch.float32, torch.bfloat16):
        out = torch.empty(m, n, dtype=dtype, device="cuda")
        R.mx4_matmul(qx, qw, out)
        assert torch.equal(out, want.to(dtype)), (dtype, (out != want.to(dtype)).nonzero()[:5].tolist())
        for activations in (x, x.to(torch.bfloat16)):       # (values of the format are numbers of bf16)
            out.fill_(77.0)
            R.mx4_linear(activations, qw, out, ws)
            assert torch.equal(out, want.to(dtype)), (dtype, activations.dtype)
