"""Products of 4-bit matrices at the sizes between few rows and many: tiles of 64, and groups of rows whose sums are
divided among waves.  Against the products of the values in 64 bits; bounds as k additions that lose a unit in the last
place each, and the rounding to the result's type."""
import pytest
import torch

import paper_2605_06534_amd as R

pytestmark = pytest.mark.gpu


def rounded_matrix(rows, cols, seed, std=1.0):
    x = torch.randn(rows, cols, generator=torch.Generator("cuda").manual_seed(seed), device="cuda") * std
    q, values = R.Mx4(rows, cols), torch.empty(rows, cols, device="cuda")
    R.mx4_quantize(x, q)
    R.mx4_dequantize(q, values)
    return x, q, values.double()


@pytest.mark.parametrize("k", [31, 544, 2080, 5121])
@pytest.mark.parametrize("m,n", [(65, 70), (100, 1003), (129, 4100), (640, 130), (333, 2500), (1500, 1500), (3000, 20)])
def test_products_between_few_rows_and_many(m, n, k):
    print("case: product", m, n, k, flush=True)
    x, qa, a = rounded_matrix(m, k, 71)
    _, qw, w = rounded_matrix(n, k, 72, 0.05)
    want, size = a @ w.t().contiguous(), a.abs() @ w.abs().t().contiguous()
    for dtype, pad in ((torch.float32, 0), (torch.bfloat16, 3)):
        half = torch.finfo(dtype).eps / 2
        bound = k * 2.0 ** -23 * size * (1 + half) + want.abs() * half + 2.0 ** -134
        out = torch.full((m, n + pad), 7.0, dtype=dtype, device="cuda")
        R.mx4_matmul(qa, qw, out[:, :n])
        assert ((out[:, :n].double() - want).abs() <= bound).all() and (out[:, n:] == 7).all()
        again = torch.empty(m, n, dtype=dtype, device="cuda")
        R.mx4_linear(x, qw, again, R.mx4_linear_workspace(m, n, k))
        assert torch.equal(again, out[:, :n])                     # the same bits, also from values that are rounded on the way


def test_a_row_that_is_no_number_stays_alone():
    print("case: product with NaN in groups of rows", flush=True)
    m, n, k = 200, 300, 4096
    x, _, _ = rounded_matrix(m, k, 73)
    _, qw, _ = rounded_matrix(n, k, 74)
    x[77, 4000] = float("nan")
    out = torch.empty(m, n, device="cuda")
    R.mx4_linear(x, qw, out, R.mx4_linear_workspace(m, n, k))
    bad = torch.isnan(out)
    assert bad[77].all() and bad.sum().item() == n


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("m,n", [(1, 1), (5, 300), (65, 70), (400, 400), (70000, 3), (4000, 4000)])
def test_sums_of_nothing(m, n, dtype):
    """No columns: zeros, whichever way a product of that many rows would go."""
    print("case: product without columns", m, n, dtype, flush=True)
    out = torch.full((m, n + 1), 9.0, dtype=dtype, device="cuda")
    R.mx4_matmul(R.Mx4(m, 0), R.Mx4(n, 0), out[:, :n])
    assert (out[:, :n] == 0).all() and (out[:, n:] == 9).all()
    out.fill_(9.0)
    R.mx4_linear(torch.empty(m, 0, dtype=torch.bfloat16, device="cuda"), R.Mx4(n, 0), out[:, :n], R.mx4_linear_workspace(m, n, 0))
    assert (out[:, :n] == 0).all() and (out[:, n:] == 9).all()


@pytest.mark.parametrize("shifted", [False, True], ids=["aligned", "scales_anywhere"])
@pytest.mark.parametrize("k", [1024, 2048, 5120])
@pytest.mark.parametrize("m,n", [(66, 9000), (200, 1500), (1000, 1003), (1600, 2100), (129, 26000)])
def test_whole_groups_of_scales(m, n, k, shifted):
    """Columns in whole groups of 32 blocks, whose scales may go another way; also where their rows begin at odd addresses."""
    print("case: product of whole groups", m, n, k, shifted, flush=True)

    def matrix(rows, seed, std):
        x = torch.randn(rows, k, generator=torch.Generator("cuda").manual_seed(seed), device="cuda") * std
        x *= torch.exp2(torch.randint(-6, 6, (rows, k // 32, 1), generator=torch.Generator("cuda").manual_seed(seed + 1), device="cuda").float()).expand(-1, -1, 32).reshape(rows, k)
        buffer = torch.full((rows * k // 32 + 1,), 255, dtype=torch.uint8, device="cuda")       # (NaN, should a neighbour be read)
        scales = buffer[1:].view(rows, k // 32) if shifted else None
        q, values = R.Mx4(rows, k, scales=scales), torch.empty(rows, k, device="cuda")
        R.mx4_quantize(x, q)
        R.mx4_dequantize(q, values)
        return q, values.double()

    (qa, a), (qw, w) = matrix(m, 81, 1.0), matrix(n, 83, 0.05)
    want, size = a @ w.t().contiguous(), a.abs() @ w.abs().t().contiguous()
    for dtype in (torch.float32, torch.bfloat16):
        half = torch.finfo(dtype).eps / 2
        bound = k * 2.0 ** -23 * size * (1 + half) + want.abs() * half + 2.0 ** -134
        out = torch.empty(m, n, dtype=dtype, device="cuda")
        R.mx4_matmul(qa, qw, out)
        assert ((out.double() - want).abs() <= bound).all()
    # NaN in one row of either: of that row and column only
    qa.scales[m - 1, k // 32 - 1] = 255
    qw.scales[n // 2, 0] = 255
    out = torch.empty(m, n, device="cuda")
    R.mx4_matmul(qa, qw, out)
    bad = torch.isnan(out)
    assert bad[m - 1].all() and bad[:, n // 2].all() and bad.sum().item() == m + n - 1


@pytest.mark.parametrize("m,k", [(4, 2049), (5, 2048), (5, 2080), (8, 2048), (8, 33), (9, 2048), (6, 1), (7, 1025)])
def test_rows_that_a_product_rounds_itself(m, k):
    """On either side of where the activations go through memory: the same values as through it."""
    print("case: rounded on the way", m, k, flush=True)
    n = 1003
    x = torch.randn(m, k + 1, generator=torch.Generator("cuda").manual_seed(92), device="cuda").to(torch.bfloat16)[:, :k]
    _, qw, w = rounded_matrix(n, k, 93)
    q, values, out = R.Mx4(m, k), torch.empty(m, k, device="cuda"), torch.empty(m, n, device="cuda")
    R.mx4_quantize(x, q)
    R.mx4_dequantize(q, values)
    R.mx4_linear(x, qw, out, R.mx4_linear_workspace(m, n, k))
    a = values.double()
    want, size = a @ w.t().contiguous(), a.abs() @ w.abs().t().contiguous()
    assert ((out.double() - want).abs() <= k * 2.0 ** -23 * size * (1 + 2.0 ** -24) + want.abs() * 2.0 ** -24 + 2.0 ** -134).all()


@pytest.mark.parametrize("m,n,k", [(3400, 3600, 1024), (3329, 3841, 2048), (3500, 3500, 5120), (300, 49000, 1024)])
def test_large_tiles_of_whole_groups(m, n, k):
    print("case: large tiles, whole groups", m, n, k, flush=True)
    _, qa, a = rounded_matrix(m, k, 95)
    _, qw, w = rounded_matrix(n, k, 96, 0.05)
    qw.scales[n - 1, k // 32 - 1] = 255                           # NaN, of the last column only
    want, size = a @ w.t().contiguous(), a.abs() @ w.abs().t().contiguous()
    for dtype in (torch.float32, torch.bfloat16):
        half = torch.finfo(dtype).eps / 2
        bound = k * 2.0 ** -23 * size * (1 + half) + want.abs() * half + 2.0 ** -134
        out = torch.empty(m, n, dtype=dtype, device="cuda")
        R.mx4_matmul(qa, qw, out)
        assert torch.isnan(out[:, n - 1]).all()
        assert ((out.double() - want).abs() <= bound)[:, :n - 1].all()
