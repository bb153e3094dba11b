"""The operators at the limits of what a launch can hold: values that are known exactly, whatever is launched for them."""
import pytest
import torch

import paper_2605_06534_amd as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("total", [0, 1, 50000, 1 << 37, 1 << 40, (1 << 63) - 1])
def test_clipping_with_a_total_that_is_wrong(total, dtype):
    """Gradients of ones and a factor of 1 / 4 (the norm and what 1e-6 adds to it are far from where that could round elsewhere)."""
    print("case: clip with another total", total, dtype, flush=True)
    numels = [70000, 3, 50001]
    flat = torch.ones(sum(numels) + 1, dtype=dtype, device="cuda")
    views = list(flat[1:].split(numels))
    tab, offsets, norm, ws = R.ptr_table(views), R.offset_table(numels), torch.zeros(1, device="cuda"), R.grad_workspace()
    exact = sum(numels) ** 0.5
    for two_calls in (False, True):
        out = torch.full_like(flat, 9.0)
        out_tab = R.ptr_table(list(out[1:].split(numels)))
        if two_calls:
            s = torch.zeros(1, dtype=torch.float64, device="cuda")
            R.grad_sum_squares(tab, offsets, total, dtype, s, ws)
            assert s.item() == sum(numels)                        # (whole numbers add up exactly)
            R.grad_clip(tab, offsets, total, dtype, out_tab, s, exact / 4, norm)
        else:
            R.grad_clip_norm(tab, offsets, total, dtype, out_tab, exact / 4, norm, ws)
        assert abs(norm.item() - exact) <= exact * 2.0 ** -24
        # the norm, the sum with 1e-6 and the quotient are rounded to fp32, then the result to its type
        assert ((out[1:].double() - 0.25 * exact / (exact + 1e-6)).abs() <= 0.25 * (4 * 2.0 ** -24 + torch.finfo(dtype).eps / 2)).all()
        assert out[0].item() == 9.0


@pytest.mark.parametrize("n", [5, 20000])
def test_a_gradient_of_more_rows_than_one_launch_clears(n):
    """Rows that differ, so every value is one token's; all other rows become zero."""
    print("case: gradient of 2^30 rows", n, flush=True)
    rows, cols = (1 << 30) + 3, 1
    tokens = torch.arange(n, device="cuda") * (rows // n)
    tokens[-1], tokens[n // 2] = rows - 1, rows           # (the last row, and no row)
    dy = (torch.arange(n, device="cuda") % 255 + 1).to(torch.bfloat16)[:, None]
    grad = torch.full((rows, cols), 9.0, dtype=torch.bfloat16, device="cuda")
    R.embedding_grad(dy, tokens, grad, R.embedding_grad_workspace(rows, cols, n), scale=2.0)
    here = tokens < rows
    assert torch.equal(grad[tokens[here]], dy[here] * 2)
    grad[tokens[here]] = 0
    assert not grad.any().item()


def room_for(gigabytes):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gigabytes << 30:
        pytest.skip("needs %d GB of free GPU memory" % gigabytes)


def test_a_lookup_of_more_vectors_than_a_launch_has_threads_for():
    print("case: lookup of 2^33 vectors", flush=True)
    room_for(130)
    n, cols = (1 << 31) - 1, 25
    tokens = torch.arange(n, dtype=torch.int32, device="cuda").remainder_(251).sub_(1)       # (a token of no row among them)
    table = torch.randn(250, cols, generator=torch.Generator("cuda").manual_seed(3), device="cuda").to(torch.bfloat16)
    out = torch.empty(n, cols, dtype=torch.bfloat16, device="cuda")
    R.embedding_lookup(table, tokens, out, scale=0.5)
    ends = torch.cat([torch.zeros(1, cols, dtype=torch.bfloat16, device="cuda"), table * 0.5])
    for at in (0, 1 << 30, n - 100000, n - 1000):
        part = slice(at, min(n, at + 100000))
        assert torch.equal(out[part], ends[tokens[part].long() + 1])
    assert torch.equal(out[:, 24], ends[:, 24].repeat(n // 251 + 1)[:n])
    del out, tokens
    torch.cuda.empty_cache()


def test_a_4_bit_matrix_of_more_vectors_than_a_launch_has_threads_for():
    """Whole numbers up to 4 and a power of two for every row come back as they were."""
    print("case: mx4 of 2^33 vectors", flush=True)
    room_for(110)
    rows, cols = (1 << 29) + 5, 33
    small = torch.randint(-4, 5, (255, cols), generator=torch.Generator("cuda").manual_seed(4), device="cuda").float()
    small[:, 0] = 4.0
    small[:, 32] = 4.0
    small *= torch.exp2(torch.arange(255, device="cuda") % 20 - 10.0)[:, None]
    x = small.repeat(rows // 255 + 1, 1)[:rows]
    q = R.Mx4(rows, cols)
    R.mx4_quantize(x, q)
    want = R.Mx4(255, cols)
    R.mx4_quantize(small, want)
    for at in (0, 1 << 28, (1 << 29) - 700, rows - 600):
        part = slice(at, min(rows, at + 600))
        which = torch.arange(part.start, part.stop, device="cuda") % 255
        assert torch.equal(q.codes[part], want.codes[which]) and torch.equal(q.scales[part], want.scales[which])
    x.fill_(77.0)
    R.mx4_dequantize(q, x)
    for at in range(0, rows, 255 * 100000):
        part = x[at:at + 255 * 100000]
        assert torch.equal(part, small.repeat(100001, 1)[:len(part)])
    del x, q
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_a_product_with_more_rows_of_weights_than_a_launch_has_threads_for(dtype):
    """One activation of ones, weights of one value a row: sums of whole numbers."""
    print("case: product with 2^30 rows of weights", dtype, flush=True)
    room_for(70)
    n, k = (1 << 30) + 50, 32
    q = R.Mx4(n, k)
    q.codes.copy_((torch.arange(n, device="cuda") % 8 * 0x11).to(torch.uint8)[:, None].expand(n, 16))
    q.scales.fill_(127)
    out = torch.empty(1, n, dtype=dtype, device="cuda")
    R.mx4_linear(torch.ones(1, k, dtype=torch.bfloat16, device="cuda"), q, out, R.mx4_linear_workspace(1, n, k))
    values = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda").to(dtype) * k
    assert torch.equal(out[0], values.repeat(n // 8 + 1)[:n])
    del q, out
    torch.cuda.empty_cache()


def test_places_for_a_norm_that_hold_none_are_refused():
    """The address of an empty tensor is null, as where no norm is asked for."""
    print("case: empty places for results", flush=True)
    x, s, empty = torch.ones(8, device="cuda"), torch.ones(1, dtype=torch.float64, device="cuda"), torch.empty(0, device="cuda")
    tab, offsets = R.ptr_table([x]), R.offset_table([8])
    for call in (lambda: R.grad_clip(tab, offsets, 8, torch.float32, tab, s, 0.5, empty),
                 lambda: R.grad_clip(tab, offsets, 8, torch.float32, tab, s[:0], 0.5),
                 lambda: R.grad_clip_norm(tab, offsets, 8, torch.float32, tab, 0.5, empty, R.grad_workspace())):
        with pytest.raises(R.RoseError):
            call()
    assert (x == 1).all()


def test_the_norm_of_no_tensors_is_zero():
    print("case: no tensors", flush=True)
    none, offsets = R.ptr_table([]), R.offset_table([])
    s, norm = torch.full((1,), 5.0, dtype=torch.float64, device="cuda"), torch.full((1,), 5.0, device="cuda")
    R.grad_sum_squares(none, offsets, 0, torch.float32, s, R.grad_workspace())
    R.grad_clip(none, offsets, 0, torch.float32, none, s, 1.0, norm)
    assert s.item() == 0 and norm.item() == 0
    norm.fill_(5.0)
    R.grad_clip_norm(none, offsets, 0, torch.bfloat16, none, 1.0, norm, R.grad_workspace())
    assert norm.item() == 0
