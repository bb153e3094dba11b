"""The operators at the ends of a synchronisation where size decides how they go about it: products in large tiles and of few
rows with wide matrices, totals of gradients that many workgroups share, vectors of several a lane, and data beyond 4 GB.

Bounds, where there are any: products as k additions that lose a unit in the last place each, k * 2^-23 * sum |a w|, and the
rounding to the result's type; the norm and the scaled gradients as roundings of fp32 (2^-24 each: the norm, the sum with
1e-6, the quotient, the product) and of bf16 (half of its eps)."""
import math

import pytest
import torch

import paper_2605_06534_amd as R

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float32]
IDS = ["bf16", "f32"]


def on_gpu(*shape, seed, dtype=torch.float32, std=1.0):
    return (torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda") * std).to(dtype)


def rounded_matrix(x):
    """The 4-bit matrix of x and its values (expanding is exact, as its own tests show)."""
    q, values = R.Mx4(*x.shape), torch.empty(x.shape, device="cuda")
    R.mx4_quantize(x, q)
    R.mx4_dequantize(q, values)
    return q, values.double()


def check_product(got, a, w, what):
    want, size = a @ w.t().contiguous(), a.abs() @ w.abs().t().contiguous()
    half = torch.finfo(got.dtype).eps / 2
    bound = a.shape[1] * 2.0 ** -23 * size * (1 + half) + want.abs() * half + 2.0 ** -134
    off = (got.double() - want).abs()
    assert (off <= bound).all(), (what, (off - bound).max().item())


@pytest.mark.parametrize("m,n,k", [(3400, 3600, 300), (3329, 3841, 1000), (20000, 700, 65), (300, 49000, 512),     # large tiles, ragged
                                   (17, 9001, 1056), (32, 8192, 640), (33, 8200, 500), (64, 9003, 2080)])         # few rows, many of the weights
def test_products_by_size(m, n, k):
    print("case: product", m, n, k, flush=True)
    qa, a = rounded_matrix(on_gpu(m, k, seed=61))
    qw, w = rounded_matrix(on_gpu(n, k, seed=62, std=0.05))
    for dtype, pad in ((torch.bfloat16, 5), (torch.float32, 0), (torch.float32, 2)):
        out = torch.full((m, n + pad), 7.0, dtype=dtype, device="cuda")
        R.mx4_matmul(qa, qw, out[:, :n])
        check_product(out[:, :n], a, w, (m, n, k, dtype))
        assert (out[:, n:] == 7).all()


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("numels", [[17000001, 5, 3000, 0, 9999999], [1, 40000000], [123] * 200 + [20000000]], ids=["odd", "one", "small_first"])
def test_clip_of_many(numels, dtype):
    """More than the workgroups' first pieces: the sum in a launch of its own, and tensors that begin inside every piece."""
    print("case: clip of many", numels[:3], dtype, flush=True)
    flat = on_gpu(sum(numels) + len(numels), seed=63, dtype=dtype)
    at, views = 1, []
    for k in numels:
        views.append(flat[at:at + k])
        at += k + 1
    used = torch.ones_like(flat, dtype=torch.bool)
    for v in views:
        if v.data_ptr() > flat.data_ptr():
            used[(v.data_ptr() - flat.data_ptr()) // flat.element_size() - 1] = False
    exact = math.sqrt(sum((v.double() ** 2).sum().item() for v in views))
    limit = exact / 3
    want = flat.double() * (limit / (exact + 1e-6))
    kept = flat.clone()
    tab, offsets, norm, ws = R.ptr_table(views), R.offset_table(numels), torch.zeros(1, device="cuda"), R.grad_workspace()
    s = torch.zeros(1, dtype=torch.float64, device="cuda")
    R.grad_sum_squares(tab, offsets, sum(numels), dtype, s, ws)
    R.grad_clip_norm(tab, offsets, sum(numels), dtype, tab, limit, norm, ws)
    assert abs(norm.item() - exact) <= exact * (2.0 ** -24 + sum(numels) * 2.0 ** -53)
    off = (flat.double() - want).abs()
    bound = want.abs() * (1.02 * 4 * 2.0 ** -24 + (torch.finfo(dtype).eps / 2 if dtype == torch.bfloat16 else 0)) + 2.0 ** -134
    inside = torch.zeros_like(used)
    at = 1
    for k in numels:
        inside[at:at + k] = True
        at += k + 1
    assert (off <= bound)[inside].all()
    assert torch.equal(flat[~inside], kept[~inside])          # between the tensors nothing was written
    # in two calls: the same bits
    twice, at, twos = kept.clone(), 1, []
    for k in numels:
        twos.append(twice[at:at + k])
        at += k + 1
    t = R.ptr_table(twos)
    R.grad_clip(t, offsets, sum(numels), dtype, t, s, limit, None)
    assert torch.equal(twice, flat)


@pytest.mark.parametrize("out", DTYPES, ids=IDS)
@pytest.mark.parametrize("table", DTYPES, ids=IDS)
@pytest.mark.parametrize("cols", [4, 6, 8, 1001, 4096])
def test_lookup_of_many(cols, table, out):
    print("case: lookup of many", cols, table, out, flush=True)
    n, rows = 5000001 // cols, 999
    values = on_gpu(rows, cols + 3, seed=64, dtype=table)[:, :cols]
    tokens = torch.randint(-1, rows + 2, (n,), generator=torch.Generator("cuda").manual_seed(65), device="cuda")
    got = torch.full((n, cols + 1), 5.0, dtype=out, device="cuda")
    R.embedding_lookup(values, tokens, got[:, :cols], scale=3.0)
    here = (tokens >= 0) & (tokens < rows)
    want = values[tokens.clamp(0, rows - 1)].float() * 3.0 * here[:, None]
    assert torch.equal(got[:, :cols], want.to(out)) and (got[:, cols:] == 5).all()


def test_tables_and_gradients_beyond_4_gb():
    print("case: embedding beyond 4 GB", flush=True)
    rows, cols = 560000, 4096
    table = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    table.copy_((torch.arange(rows, device="cuda") % 251).to(torch.bfloat16)[:, None].expand(rows, cols))
    tokens = torch.arange(rows - 1, -1, -1, device="cuda")
    out = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    R.embedding_lookup(table, tokens, out)
    assert torch.equal(out[:, 0], (tokens % 251).to(torch.bfloat16)) and torch.equal(out[:, cols - 1], out[:, 0])
    # (one token each, in reverse, and none for every 256th row: those become zero)
    tokens[tokens % 256 == 3] = -1
    grad = torch.full((rows, cols), 9.0, dtype=torch.float32, device="cuda")
    ws = R.embedding_grad_workspace(rows, cols, rows)
    R.embedding_grad(out, tokens, grad, ws, scale=2.0)
    at = torch.arange(rows, device="cuda")
    want = torch.where(at % 256 == 3, 0.0, 2.0 * (at % 251).float())
    for c in (0, 1777, cols - 1):
        assert torch.equal(grad[:, c], want)
    R.embedding_grad(out, tokens, grad, ws, scale=1.0, accumulate=True)
    for c in (0, 1777, cols - 1):
        assert torch.equal(grad[:, c], want * 1.5)


def test_gradients_of_more_than_2_to_the_32_elements():
    print("case: clip beyond 2^32 elements", flush=True)
    numels = [(1 << 31) + 5, 3, (1 << 31) + 9]
    flat = torch.ones(sum(numels), dtype=torch.bfloat16, device="cuda")
    views = list(flat.split(numels))
    tab, norm = R.ptr_table(views), torch.zeros(1, device="cuda")
    R.grad_clip_norm(tab, R.offset_table(numels), sum(numels), torch.bfloat16, tab, math.sqrt(sum(numels)) / 4, norm, R.grad_workspace())
    assert abs(norm.item() - math.sqrt(sum(numels))) <= norm.item() * 2.0 ** -23
    assert (flat == 0.25).all()


def test_4_bit_matrices_beyond_4_gb():
    print("case: 4-bit beyond 4 GB", flush=True)
    rows, cols = 1100000, 8192
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    step = 10000
    for r in range(0, rows, step):
        x[r:r + step] = on_gpu(step, cols, seed=r, dtype=torch.bfloat16)
    q = R.Mx4(rows, cols)
    R.mx4_quantize(x, q)
    ends = [slice(0, 300), slice(rows - 300, rows)]
    for s in ends:
        part = R.Mx4(300, cols)
        R.mx4_quantize(x[s], part)
        assert torch.equal(part.codes, q.codes[s]) and torch.equal(part.scales, q.scales[s])
    back = torch.empty_like(x)
    R.mx4_dequantize(q, back)
    for s in ends:
        part, values = R.Mx4(300, cols), torch.empty(300, cols, dtype=torch.bfloat16, device="cuda")
        R.mx4_quantize(x[s], part)
        R.mx4_dequantize(part, values)
        assert torch.equal(values, back[s])
    del x
    for m in (1, 40, 200):
        a, va = rounded_matrix(on_gpu(m, cols, seed=66))
        out = torch.empty(m, rows, device="cuda")
        R.mx4_matmul(a, q, out)
        for s in ends:
            check_product(out[:, s], va, back[s].double(), m)
    # and as the many rows of a product
    w, vw = rounded_matrix(on_gpu(100, cols, seed=67))
    out = torch.empty(rows, 100, device="cuda")
    R.mx4_matmul(q, w, out)
    for s in ends:
        check_product(out[s], back[s].double(), vw, "rows")


@pytest.mark.parametrize("n", [1, 7, 64, 1500, 20000])
@pytest.mark.parametrize("rows,cols,pad,dtype", [(40000, 1024, 0, torch.float32), (70001, 1001, 3, torch.bfloat16), (33333333, 3, 0, torch.bfloat16),
                                                 (9001, 4099, 1, torch.float32)])
def test_rows_that_no_token_names_become_zero(rows, cols, pad, dtype, n):
    """Gradients of more than is filled while the tokens are sorted; no row has two tokens, so every value is exact."""
    print("case: zeros", rows, cols, pad, dtype, n, flush=True)
    g = torch.Generator("cuda").manual_seed(68 + n)
    n = min(n, rows)
    tokens = torch.randperm(rows, generator=g, device="cuda")[:n]
    tokens[n // 2::3] = rows                          # (of no row)
    dy = on_gpu(n, cols, seed=69, dtype=torch.bfloat16)
    grad = torch.full((rows, cols + pad), 9.0, dtype=dtype, device="cuda")
    want = grad.clone()
    want[:, :cols] = 0
    here = tokens < rows
    want[tokens[here], :cols] = (dy[here].float() * 2.0).to(dtype)
    R.embedding_grad(dy, tokens, grad[:, :cols], R.embedding_grad_workspace(rows, cols, n), scale=2.0)
    assert torch.equal(grad, want)
