"""The divergence from a teacher's top logits and its gradient, against the formulas in 64 bits.

Bounds, u = 2^-24, d = (largest logit - z) / T: a term of the sum over the columns is off by 4 u d (difference, factor, its rounding, product)
and 2 u (exponential) of itself, the sum by its terms, weighted, and by twice the additions and rescalings that a thread makes one after
the other (of 256 threads: columns / 256 + 40).  lse and loss are off by as much and half a unit of their type.  A probability in the gradient by 4 u d + 8 u of itself and by
what the sum is off (from lse: 4 u |z / T - lse|, and u |z / T| for results in bf16, whose 1 / T is one number), an entry's p by 4 u for
each time that its column is named; d_loss / T is in both.  A loss whose terms cancel (one column: they all do) has the roundings of 64 bits of each
left, 2^-53 of their magnitudes for each of the entries and a few operations more.  bf16 and fp32 results: half a step more, and 2^-126 where exponentials end."""
import math

import pytest
import torch

import paper_2605_06534_amd as R

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def case(rows, cols, top, dtype, seed, pad=0, index=torch.int64, std=2.0, shift=0.0):
    g = torch.Generator("cuda").manual_seed(seed)
    flat = (torch.randn(rows * (cols + pad) + 8, generator=g, device="cuda") * std + shift).to(dtype)
    z = flat[1:1 + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    ids = torch.rand(rows, cols, generator=g, device="cuda").topk(min(top, cols), 1)[1] if rows * cols < 1 << 26 else (
        (torch.randint(0, cols, (rows, 1), generator=g, device="cuda") + torch.arange(top, device="cuda") * max(1, cols // max(1, top))) % cols)
    if ids.shape[1] < top:
        ids = torch.cat((ids, torch.full((rows, top - ids.shape[1]), -1, device="cuda")), 1)
    teacher = torch.randn(rows, top, generator=g, device="cuda") * 3 + 5
    kept = torch.randint(0, top + 1, (rows, 1), generator=g, device="cuda")
    kept[::3] = top
    ids = torch.where(torch.arange(top, device="cuda") < kept, ids, -1)
    if rows > 1 and top > 1:
        ids[1, :] = cols                               # numbers beyond the columns are no entries either
    if rows > 2 and top > 2:
        ids[2, 1] = ids[2, 0]                          # the same column twice
        teacher[2, 2] = -math.inf
    return z, ids.to(index), teacher, torch.rand(rows, generator=g, device="cuda") + 0.5


def exact(z, ids, teacher, t, d_loss=None, lse=None):
    """loss, lse, gradient and bounds, in 64 bits"""
    rows, cols = z.shape
    out = {k: [] for k in ("loss", "lse", "grad", "e_lse", "e_grad", "some", "e_64")}
    for a in range(0, rows, max(1, (1 << 24) // cols)):
        b = min(rows, a + max(1, (1 << 24) // cols))
        x, i, k = z[a:b].double() / t, ids[a:b].long(), teacher[a:b].double() / t
        here = (i >= 0) & (i < cols) & (k != -math.inf)
        some = here.any(1)
        p = torch.softmax(torch.where(here, k, -math.inf), 1)
        p = torch.where(some[:, None] & here, p, 0.0)
        s = torch.logsumexp(x, 1)
        most = x.amax(1, keepdim=True)
        q = torch.exp(x - s[:, None])
        e_sum = U * (2 * (cols / 256 + 40) + 4 * torch.nan_to_num(q * (most - x), 0.0).sum(1) + 4)
        terms = torch.where(p > 0, p * (torch.log(p.clamp(min=1e-320)) - x.gather(1, i.clamp(0, cols - 1)) + s[:, None]), 0.0)
        out["loss"].append(terms.sum(1)), out["lse"].append(s), out["e_lse"].append(e_sum), out["some"].append(some)
        sizes = p * (torch.log(p.clamp(min=1e-320)).abs() + 2 * torch.where(here, k, 0.0).abs() + 2 * x.gather(1, i.clamp(0, cols - 1)).abs())
        out["e_64"].append((len(p[0]) + 16) * 2.0 ** -53 * (torch.where(p > 0, sizes, 0.0).sum(1) + s.abs() + 1))
        if d_loss is not None:
            used = s if lse is None else lse[a:b].double()
            q = torch.exp(x - used[:, None])
            if lse is None:
                e = q * (U * (4 * (most - x) + 8) + e_sum[:, None])
            else:
                e = q * U * (4 * (x - used[:, None]).abs() + 8 + (x.abs() if z.dtype == torch.bfloat16 else 0))
            e, q = torch.where(x == -math.inf, 0.0, e), torch.where(some[:, None], q, 0.0)
            spare = torch.zeros(b - a, cols + 1, dtype=torch.float64, device="cuda")
            spare.scatter_add_(1, torch.where(here, i, cols), p)
            named = torch.zeros_like(spare).scatter_add_(1, torch.where(here, i, cols), torch.ones_like(p))
            d = torch.where(some, d_loss[a:b].double(), 0.0)[:, None] / t
            out["grad"].append(d * (q - spare[:, :-1]))
            out["e_grad"].append(torch.where(some[:, None], d.abs() * (e + 4 * U * spare[:, :-1] * (1 + named[:, :-1]) + 2.0 ** -126), 0.0))
    return {k: torch.cat(v) for k, v in out.items() if v}


def check_gradient(got, want, what):
    half = torch.finfo(got.dtype).eps / 2
    off, bound = (got.double() - want["grad"]).abs(), want["e_grad"] * (1 + half) + half * want["grad"].abs() + 2.0 ** -134
    assert (off <= bound).all(), (what, (off - bound).max().item())


def check(rows, cols, top, dtype, t, seed=1, pad=0, index=torch.int64, std=2.0, shift=0.0):
    print("case: distill", rows, cols, top, dtype, t, pad, flush=True)
    z, ids, teacher, d_loss = case(rows, cols, top, DTYPES[dtype], seed, pad, index, std, shift)
    ws = R.distill_workspace(rows, cols)
    ws.fill_(0xFF)
    loss, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    R.distill_loss(z, ids, teacher, loss, lse, ws, temperature=t)
    want = exact(z, ids, teacher, t, d_loss)

    def check_loss(loss, lse):
        assert ((lse.double() - want["lse"]).abs() <= want["e_lse"] + U * want["lse"].abs()).all()
        assert ((loss.double() - want["loss"]).abs() <= torch.where(want["some"], want["e_lse"] + want["e_64"], 0.0) + U * want["loss"].abs()).all()

    check_loss(loss, lse)
    whole = torch.full((rows, cols + pad), 7.0, dtype=z.dtype, device="cuda")
    loss2, lse2, d = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), whole[:, :cols]
    ws.fill_(0x7F)
    R.distill_loss_grad(z, ids, teacher, d_loss, loss2, lse2, d, ws, temperature=t)
    check_loss(loss2, lse2)                       # (sums may be divided in another way than above)
    assert (whole[:, cols:] == 7).all()
    check_gradient(d, want, "together")
    whole.fill_(7)
    R.distill_grad(z, ids, teacher, lse, d_loss, d, temperature=t)
    assert (whole[:, cols:] == 7).all()
    check_gradient(d, exact(z, ids, teacher, t, d_loss, lse), "from lse")
    return z, ids, teacher, d_loss, loss, lse, d


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [1, 2, 3, 4, 5, 8, 9, 63, 100, 1000, 1025, 2048, 2049, 4099, 8200, 16384, 16385, 32000])
def test_by_columns(cols, dtype):
    for rows, top, t, pad, index in ((1, 1, 1.0, 0, torch.int64), (5, 20, 2.0, 3, torch.int32), (40, 7, 0.7, 8, torch.int64)):
        check(rows, cols, top, dtype, t, pad=pad, index=index)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(600, 1000), (520, 2500), (1500, 16400), (1030, 32003), (300, 40001), (513, 151936), (257, 152064), (17, 300001), (2, 1000003)])
def test_of_many(rows, cols, dtype):
    check(rows, cols, 64, dtype, 1.0, seed=2, pad=3)


@pytest.mark.parametrize("top", [0, 1, 63, 64, 65, 256, 257, 1000, 1024])
def test_by_entries(top):
    for rows, cols in ((3, 900), (3, 5000), (600, 1500)):
        check(rows, cols, top, "f32", 1.5, seed=3)
        check(rows, cols, top, "bf16", 0.25, seed=4)


def test_logits_far_from_zero():
    for shift in (300.0, -5000.0):
        check(9, 5000, 10, "f32", 1.0, seed=5, shift=shift)
        check(1100, 3000, 10, "f32", 3.0, seed=6, shift=shift)
    check(9, 5000, 10, "f32", 0.05, seed=7, std=30.0)


@pytest.mark.parametrize("rows,cols", [(4, 6000), (1100, 700)])
def test_masked_columns(rows, cols):
    """Minus infinity or a type's lowest value in most columns, whole stretches of threads among them, and at an entry."""
    for dtype in (torch.float32, torch.bfloat16):
        for mask in (-math.inf, torch.finfo(dtype).min):
            print("case: masked columns", rows, dtype, mask, flush=True)
            z, ids, teacher, d_loss = case(rows, cols, 6, dtype, 8)
            ids[:] = torch.arange(6, device="cuda") * 3 + 40
            z[:, :30], z[:, 60:] = mask, mask
            loss, lse, d, ws = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(z), R.distill_workspace(rows, cols)
            R.distill_loss_grad(z, ids, teacher, d_loss, loss, lse, d, ws)
            want = exact(z[:, 30:60], ids - 30, teacher, 1.0, d_loss)
            assert ((loss.double() - want["loss"]).abs() <= want["e_lse"] + U * want["loss"].abs()).all()
            check_gradient(d[:, 30:60].contiguous(), want, "together")
            assert (d[:, :30] == 0).all() and (d[:, 60:] == 0).all()
            R.distill_grad(z, ids, teacher, lse, d_loss, d)
            check_gradient(d[:, 30:60].contiguous(), exact(z[:, 30:60], ids - 30, teacher, 1.0, d_loss, lse), "from lse")
            assert (d[:, :30] == 0).all() and (d[:, 60:] == 0).all()
            ids[0, 0] = 20                            # an entry where the student has nothing
            R.distill_loss_grad(z, ids, teacher, d_loss, loss, lse, d, ws)
            assert loss[0] > 1e30 and loss[1:].isfinite().all() and d[0].isfinite().all() and d[0, 20] < 0


@pytest.mark.parametrize("rows,cols", [(6, 6000), (1100, 700)])
def test_rows_without_entries_and_numbers_that_are_none(rows, cols):
    print("case: rows without entries", rows, flush=True)
    z, ids, teacher, d_loss = case(rows, cols, 5, torch.float32, 9)
    ids[:] = torch.arange(5, device="cuda") * 7
    teacher[2, :] = 1.0
    z[0, 3], z[1, cols - 1], d_loss[1], z[3, :], z[4, 100] = math.nan, math.inf, math.nan, -math.inf, math.nan
    ids[0], teacher[1] = -1, -math.inf
    loss, lse, d, ws = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(z), R.distill_workspace(rows, cols)
    for again in range(2):
        R.distill_loss_grad(z, ids, teacher, d_loss, loss, lse, d, ws)
        if again:
            R.distill_grad(z, ids, teacher, lse, d_loss, d)
        assert (loss[:2] == 0).all() and (d[:2] == 0).all()
        assert not loss[3:5].isfinite().any() and d[3:5].isnan().any(1).all()
        assert loss[5:].isfinite().all() and d[5:].isfinite().all() and d[2].isfinite().all()


@pytest.mark.parametrize("rows,cols", [(5, 5003), (1100, 1003), (520, 20001)])
def test_in_place(rows, cols):
    print("case: in place", rows, cols, flush=True)
    for dtype in DTYPES:
        z, ids, teacher, d_loss, loss, lse, _ = check(rows, cols, 30, dtype, 1.0, seed=10, pad=3)
        d, ws, kept = torch.empty_like(z), R.distill_workspace(rows, cols), z.clone()
        R.distill_grad(z, ids, teacher, lse, d_loss, d)
        R.distill_grad(z, ids, teacher, lse, d_loss, z)
        assert torch.equal(z, d)
        z.copy_(kept)
        R.distill_loss_grad(z, ids, teacher, d_loss, loss, lse, d, ws)
        again, last = torch.empty_like(loss), torch.empty_like(lse)
        R.distill_loss_grad(z, ids, teacher, d_loss, again, last, z, ws)
        assert torch.equal(z, d) and torch.equal(again, loss) and torch.equal(last, lse)


def test_gradient_against_differences():
    """Central differences of the loss in 64 bits; their own error is h^2 times a third derivative (below 1) and 2^-50 / h."""
    print("case: differences", flush=True)
    z, ids, teacher, d_loss, *_, d = check(4, 50, 5, "f32", 2.0, seed=11)
    h = 1e-4
    for row in range(4):
        for col in list(range(0, 50, 7)) + [int(i) for i in ids[row] if 0 <= i < 50]:
            ends = []
            for s in (h, -h):
                moved = z.double().clone()
                moved[row, col] += s
                ends.append(exact(moved, ids, teacher, 2.0)["loss"][row].item())
            assert abs((ends[0] - ends[1]) / (2 * h) * d_loss[row].item() - d[row, col].item()) < 2e-8 + 40 * U


def test_the_same_bits_twice_and_in_a_graph():
    print("case: graph", flush=True)
    for rows, cols in ((6, 9000), (700, 1200)):
        z, ids, teacher, d_loss = case(rows, cols, 12, torch.bfloat16, 12)
        loss, lse, d, ws = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(z), R.distill_workspace(rows, cols)
        other = torch.empty_like(z)

        def step():
            R.distill_loss_grad(z, ids, teacher, d_loss, loss, lse, d, ws)
            R.distill_grad(z, ids, teacher, lse, d_loss, other)

        step()
        graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            step()
        for seed in range(3):
            z.copy_(torch.randn(rows, cols, generator=torch.Generator("cuda").manual_seed(seed), device="cuda"))
            step()
            want = [v.clone() for v in (loss, lse, d, other)]
            for v in (loss, lse, d, other):
                v.fill_(3)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, (loss, lse, d, other)))


def test_nothing_to_do():
    z, ids, teacher, none = torch.empty(0, 10, device="cuda"), torch.empty(0, 4, dtype=torch.int64, device="cuda"), torch.empty(0, 4, device="cuda"), torch.empty(0, device="cuda")
    ws = R.distill_workspace(0, 10)
    R.distill_loss(z, ids, teacher, none, none, ws)
    R.distill_loss_grad(z, ids, teacher, none, none, none, z, ws)
    R.distill_grad(z, ids, teacher, none, none, z)
