"""Embedding lookups and their gradient against the definition in 64 bits: types, strides, id widths, shards, tokens of
no shard, lengths from none to several sorting tiles, one row named by everyone, rows and columns of odd sizes.

Bounds: a lookup is one fp32 product and one rounding, so its bits are known.  A gradient's row is a sum of c terms in
fp32 in some order (at most c - 1 additions), a product with the scale and an addition: its error is at most
(c + 2) 2^-24 (|scale| sum |dy| + |old|) (the first-order bound, with 2 % for what it leaves out), and half a unit in the
last place of bf16 (2^-8 of the result, which has eight significant bits, and half of the smallest subnormal) where it is
rounded to that."""
import numpy as np
import pytest
import torch

import paper_2605_06534_amd as R

pytestmark = pytest.mark.gpu

HALF = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16)}     # 2^-24, 2^-8
NAMES = {torch.float32: "f32", torch.bfloat16: "bf16"}


def matrix(rows, cols, pad, dtype, seed, offset=0):
    """Rows pad elements further apart than they are long, the first at element `offset` of its buffer."""
    g = torch.Generator().manual_seed(seed)
    flat = torch.randn(offset + rows * (cols + pad) + 8, generator=g).to(dtype).cuda()
    return flat[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]


def host(t):
    return t.detach().cpu().double().numpy()


def rounded(x32, dtype):
    return torch.from_numpy(np.ascontiguousarray(x32)).to(dtype)


LOOKUPS = [
    # tokens, rows, cols, first row, table, out, id width, pad, scale
    (1, 1, 1, 0, torch.float32, torch.float32, torch.int64, 0, 1.0),
    (1, 7, 8, 0, torch.bfloat16, torch.bfloat16, torch.int32, 0, 1.0),
    (5, 9, 7, 3, torch.bfloat16, torch.float32, torch.int64, 1, 3.5),
    (33, 100, 129, 50, torch.float32, torch.bfloat16, torch.int32, 3, 11.3137),
    (257, 64, 2048, 0, torch.bfloat16, torch.bfloat16, torch.int64, 0, 45.25),
    (64, 300, 2056, 300, torch.float32, torch.float32, torch.int64, 8, 0.5),
    (9001, 777, 515, 111, torch.bfloat16, torch.bfloat16, torch.int64, 5, 22.7),
    (20000, 333, 4100, 0, torch.float32, torch.bfloat16, torch.int32, 0, 1.0),
]


@pytest.mark.parametrize("case", LOOKUPS, ids=lambda c: "%dx%dx%d_%s_%s" % (c[0], c[1], c[2], NAMES[c[4]], NAMES[c[5]]))
def test_lookup(case):
    n, rows, cols, first, tt, ot, it, pad, scale = case
    print("case: lookup", case, flush=True)
    table = matrix(rows, cols, pad, tt, 1, offset=1)
    g = torch.Generator().manual_seed(2)
    tokens = torch.randint(max(0, first - 3), first + rows + 3, (n,), generator=g).to(it)
    tokens[::7] = -1 - torch.arange(len(tokens[::7]), dtype=it)
    out = torch.full((n, cols + pad), 77.0, dtype=ot, device="cuda")
    R.embedding_lookup(table, tokens.cuda(), out[:, :cols], scale=scale, first_row=first)
    at = tokens.long().numpy() - first
    here = (at >= 0) & (at < rows)
    want = np.zeros((n, cols), dtype=np.float32)
    want[here] = table.float().cpu().numpy()[at[here]] * np.float32(scale)
    assert torch.equal(out[:, :cols].cpu(), rounded(want, ot))
    assert (out[:, cols:] == 77).all()               # what lies between the rows stays


def test_lookup_of_far_ids_and_values():
    print("case: lookup of far ids, infinities, NaN", flush=True)
    table = matrix(4, 24, 0, torch.float32, 3)
    table[1, 3], table[2, 5], table[3, 6] = float("inf"), float("nan"), -0.0
    far = [-(1 << 63), (1 << 63) - 1, 1 << 32, (1 << 32) + 1, 5, 6, 7, 8]
    out = torch.empty(8, 24, device="cuda")
    R.embedding_lookup(table, torch.tensor(far, device="cuda"), out, scale=float("inf"), first_row=5)
    want = (table.cpu() * float("inf"))
    got = out.cpu()
    assert (got[:4] == 0).all()                      # of no shard: zeros whatever the scale
    assert torch.equal(torch.nan_to_num(got[4:], 9.5, 8.5, -8.5), torch.nan_to_num(want, 9.5, 8.5, -8.5))


def test_empty_sizes():
    print("case: no tokens, no rows, no columns", flush=True)
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    R.embedding_lookup(matrix(3, 8, 0, torch.float32, 1), none, torch.empty(0, 8, device="cuda"))
    out = torch.full((2, 8), 5.0, device="cuda")
    R.embedding_lookup(torch.empty(0, 8, device="cuda"), torch.tensor([0, 1], device="cuda"), out)
    assert (out == 0).all()
    R.embedding_lookup(torch.empty(3, 0, device="cuda"), torch.tensor([0, 1], device="cuda"), torch.empty(2, 0, device="cuda"))
    grad = torch.full((5, 9), 3.0, device="cuda")
    ws = R.embedding_grad_workspace(5, 9, 0)
    R.embedding_grad(torch.empty(0, 9, device="cuda"), none, grad, ws, accumulate=True)
    assert (grad == 3).all()
    R.embedding_grad(torch.empty(0, 9, device="cuda"), none, grad, ws)
    assert (grad == 0).all()
    R.embedding_grad(torch.empty(2, 9, device="cuda"), torch.tensor([0, 1], device="cuda"), torch.empty(0, 9, device="cuda"),
                     R.embedding_grad_workspace(0, 9, 2))


GRADS = [
    # tokens, rows, cols, first row, dy, grad, id width, pad, scale, how the tokens are spread
    (1, 1, 1, 0, torch.float32, torch.float32, torch.int64, 0, 1.0, "any"),
    (2, 3, 9, 1, torch.bfloat16, torch.bfloat16, torch.int32, 1, 2.0, "any"),
    (31, 5, 33, 0, torch.bfloat16, torch.float32, torch.int64, 0, 1.0, "any"),
    (32, 5, 64, 0, torch.float32, torch.float32, torch.int64, 0, 0.3, "any"),
    (33, 1, 65, 4, torch.bfloat16, torch.bfloat16, torch.int32, 3, 1.0, "one"),
    (64, 1000, 129, 0, torch.float32, torch.bfloat16, torch.int64, 0, 5.0, "any"),
    (97, 40, 2049, 7, torch.bfloat16, torch.float32, torch.int64, 7, 1.0, "text"),
    (1023, 513, 96, 0, torch.bfloat16, torch.float32, torch.int32, 0, 8.0, "text"),
    (1025, 2000, 264, 100, torch.float32, torch.float32, torch.int64, 8, 1.0, "text"),
    (4096, 32000, 40, 0, torch.bfloat16, torch.float32, torch.int64, 0, 1.0, "text"),
    (4097, 7, 520, 0, torch.bfloat16, torch.bfloat16, torch.int64, 0, 1.0, "any"),
    (16384, 300000, 8, 5, torch.bfloat16, torch.float32, torch.int64, 0, 1.0, "any"),
    (16385, 100, 24, 0, torch.float32, torch.float32, torch.int64, 0, 1.0, "one"),
    (20001, 19008, 17, 19008, torch.bfloat16, torch.float32, torch.int32, 2, 71.5, "text"),
    (70000, 600, 33, 0, torch.float32, torch.bfloat16, torch.int64, 0, 1.0, "text"),
    (530000, 4000000, 3, 0, torch.bfloat16, torch.float32, torch.int32, 0, 1.0, "text"),
]


def spread(n, rows, first, it, how, seed):
    g = torch.Generator().manual_seed(seed)
    if how == "one":
        ids = torch.full((n,), first, dtype=torch.int64)
        ids[n // 3] = -5
    elif how == "text":
        u = torch.rand(n, generator=g, dtype=torch.float64)
        ids = torch.exp(u * np.log(rows * 1.2 + 1)).long() - 1 + first
    else:
        ids = torch.randint(max(0, first - 1), first + rows + 1, (n,), generator=g)
    return ids.to(it)


def check_grad(got, dy, tokens, first, scale, old, dtype):
    rows, cols = got.shape
    at = tokens.long().cpu().numpy() - first
    here = np.flatnonzero((at >= 0) & (at < rows))
    order = here[np.argsort(at[here], kind="stable")]
    total, size, count = np.zeros((rows, cols)), np.zeros((rows, cols)), np.zeros((rows, 1))
    if len(order):
        named, begin = np.unique(at[order], return_index=True)
        total[named] = np.add.reduceat(dy[order], begin, axis=0)
        size[named] = np.add.reduceat(np.abs(dy[order]), begin, axis=0)
        count[named, 0] = np.diff(np.append(begin, len(order)))
    s = float(np.float32(scale))
    want = old + total * s
    bound = 1.02 * (count + 2) * 2.0 ** -24 * (abs(s) * size + np.abs(old))
    if dtype == torch.bfloat16:
        bound = bound * (1 + HALF[dtype]) + np.abs(want) * HALF[dtype] + 2.0 ** -134
    off = np.abs(host(got) - want)
    assert (off <= bound).all(), (off - bound).max()
    return count[:, 0] > 0


@pytest.mark.parametrize("accumulate", [False, True], ids=["set", "add"])
@pytest.mark.parametrize("case", GRADS, ids=lambda c: "%dx%dx%d_%s_%s_%s" % (c[0], c[1], c[2], NAMES[c[4]], NAMES[c[5]], c[9]))
def test_grad(case, accumulate):
    n, rows, cols, first, dt, gt, it, pad, scale, how = case
    print("case: embedding gradient", case, accumulate, flush=True)
    dy = matrix(n, cols, pad, dt, 5, offset=1)
    tokens = spread(n, rows, first, it, how, 6).cuda()
    whole = matrix(rows, cols + pad, 0, gt, 7)
    before = whole.clone()
    grad = whole[:, :cols]
    ws = R.embedding_grad_workspace(rows, cols, n)
    ws.fill_(0xA5)                                   # its contents before the call do not matter
    R.embedding_grad(dy, tokens, grad, ws, scale=scale, first_row=first, accumulate=accumulate)
    old = host(before[:, :cols]) if accumulate else np.zeros((rows, cols))
    named = check_grad(grad, host(dy), tokens, first, scale, old, gt)
    assert torch.equal(whole[:, cols:], before[:, cols:])
    rest = torch.from_numpy(~named).cuda()
    assert torch.equal(grad[rest], before[:, :cols][rest]) if accumulate else (grad[rest] == 0).all()
    # the same bits every time
    again = before.clone()
    R.embedding_grad(dy, tokens, again[:, :cols], ws, scale=scale, first_row=first, accumulate=accumulate)
    assert torch.equal(again, whole)


def test_grad_against_differences():
    """L = sum(c * lookup(table)) is linear in the table: moving one element of it by h moves L by h * the gradient's."""
    print("case: embedding gradient against differences", flush=True)
    rows, cols, n, scale, first = 11, 6, 50, 1.5, 4
    table = matrix(rows, cols, 0, torch.float32, 8)
    c = matrix(n, cols, 0, torch.float32, 9)
    tokens = spread(n, rows, first, torch.int64, "any", 10).cuda()
    grad = torch.empty(rows, cols, device="cuda")
    R.embedding_grad(c, tokens, grad, R.embedding_grad_workspace(rows, cols, n), scale=scale, first_row=first)

    def loss(t):
        out = torch.empty(n, cols, device="cuda")
        R.embedding_lookup(t, tokens, out, scale=scale, first_row=first)
        return (out.double() * c.double()).sum().item()

    size = (c.double().abs().sum() * scale).item()
    for r, k in ((0, 0), (3, 5), (10, 2), (7, 1)):
        up, down, h = table.clone(), table.clone(), 0.5
        up[r, k] += h
        down[r, k] -= h
        # (each output is rounded once, 2^-24 of it, on either side; |table| stays below 6)
        step = (up[r, k] - down[r, k]).item()
        assert abs((loss(up) - loss(down)) / step - grad[r, k].item()) <= 6 * size * 2.0 ** -22


def test_values_that_are_no_numbers_stay_in_their_rows():
    print("case: embedding gradient with infinities and NaN", flush=True)
    n, rows, cols = 200, 6, 40
    dy = matrix(n, cols, 0, torch.bfloat16, 11)
    tokens = (torch.arange(n) % 6).cuda()
    dy[2, 7], dy[9, 8] = float("nan"), float("inf")
    dy[4::6, 3] = -float("inf")
    dy[5, 0] = float("nan")
    tokens[5] = 77                                    # of another shard: its values are not looked at
    grad = torch.empty(rows, cols, device="cuda")
    R.embedding_grad(dy, tokens, grad, R.embedding_grad_workspace(rows, cols, n))
    bad = ~torch.isfinite(grad).cpu()
    want = torch.zeros(rows, cols, dtype=torch.bool)
    want[2, 7], want[3, 8], want[4, 3] = True, True, True
    assert torch.equal(bad, want)
    assert torch.isnan(grad[2, 7]) and grad[3, 8].item() == float("inf") and grad[4, 3].item() == -float("inf")


def test_in_a_graph_and_on_another_stream():
    print("case: embedding in a graph", flush=True)
    n, rows, cols = 3000, 900, 200
    table = matrix(rows, cols, 0, torch.bfloat16, 12)
    dy = matrix(n, cols, 0, torch.bfloat16, 13)
    tokens = spread(n, rows, 0, torch.int64, "text", 14).cuda()
    out, grad = torch.empty(n, cols, dtype=torch.bfloat16, device="cuda"), torch.empty(rows, cols, device="cuda")
    ws = R.embedding_grad_workspace(rows, cols, n)

    def step():
        R.embedding_lookup(table, tokens, out, scale=2.0)
        R.embedding_grad(dy, tokens, grad, ws, scale=2.0)

    step()
    torch.cuda.synchronize()
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            step()
    torch.cuda.synchronize()
    for rep in range(4):
        tokens.copy_(torch.roll(tokens, 17))
        dy.copy_(torch.roll(dy, 1, 0))
        out.fill_(3), grad.fill_(3), ws.fill_(rep)
        g.replay()
        torch.cuda.synchronize()
        got = out.clone(), grad.clone()
        step()
        assert torch.equal(got[0], out) and torch.equal(got[1], grad)
