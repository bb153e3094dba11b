"""Low-rank adapters of rows against their products in 64 bits.

Bounds: products of two bf16 numbers are exact in fp32; a sum of n terms is bounded by n additions that lose a unit in the last place each,
n * 2^-23 * the sum of magnitudes: k of them for what lies between the products, rank + 4 (scale, product, the sum with out) behind it; then
half a step of the result's type."""
import pytest
import torch

import paper_2605_06534_amd as R

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
STEP = 2.0 ** -23


def on_gpu(*shape, seed, dtype=torch.bfloat16, std=1.0):
    return (torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda") * std).to(dtype)


def matrix(rows, cols, pad, seed, dtype):
    flat = on_gpu(rows * (cols + pad) + 8, seed=seed, dtype=dtype)
    return flat[(pad > 0):(pad > 0) + rows * (cols + pad)].view(rows, cols + pad)


def exact(x, w, chosen, out):
    want, size = out.double(), torch.zeros(out.shape, dtype=torch.float64, device="cuda")
    for a in range(w.adapters):
        rows = (chosen == a).nonzero().view(-1)
        if not len(rows):
            continue
        s = 1.0 if w.scales is None else w.scales[a].double()
        d, u, v = w.down[a].double(), w.up[a].double(), x[rows].double()
        h, e_h = v @ d.t().contiguous(), x.shape[1] * STEP * (v.abs() @ d.abs().t().contiguous())
        want[rows] += s * (h @ u.t().contiguous())
        size[rows] = abs(s) * ((e_h + (w.rank + 4) * STEP * h.abs()) @ u.abs().t().contiguous())
    return want, size + 2 * STEP * (want.abs() + out.double().abs())


def check(m, n, k, rank, adapters, out="bf16", run=1, pad=0, seed=1, scales=True, index=torch.int32, chosen=None, ws=None):
    print("case: adapters", m, n, k, rank, adapters, out, run, pad, flush=True)
    dtype = DTYPES[out]
    x = matrix(m, k, pad, seed, torch.bfloat16)[:, :k]
    w = R.Adapters(on_gpu(adapters, rank, k, seed=seed + 1, std=k ** -0.5), on_gpu(adapters, n, rank, seed=seed + 2, std=rank ** -0.5),
                   on_gpu(adapters, seed=seed + 3, dtype=torch.float32) if scales else None)
    whole = matrix(m, n, pad, seed + 4, dtype)
    if chosen is None:
        chosen = torch.randint(-1, adapters + 1, ((m + run - 1) // run,), generator=torch.Generator("cuda").manual_seed(seed + 5), device="cuda").repeat_interleave(run)[:m]
    kept, got = whole.clone(), whole[:, :n]
    if ws is None:
        ws = R.adapter_linear_workspace(m, w)
    ws.fill_(0xFF)
    R.adapter_linear(x, w, chosen.to(index), got, ws)
    want, bound = exact(x, w, chosen, kept[:, :n])
    half = torch.finfo(dtype).eps / 2
    off = (got.double() - want).abs()
    none = (chosen < 0) | (chosen >= adapters)
    assert torch.equal(got[none], kept[:, :n][none]) and torch.equal(whole[:, n:], kept[:, n:])
    assert (off <= bound * (1 + half) + half * want.abs()).all(), (off - bound).max().item()
    return x, w, chosen, kept, got


@pytest.mark.parametrize("out", DTYPES)
@pytest.mark.parametrize("rank", [1, 3, 4, 8, 15, 16, 17, 31, 32, 33, 50, 64, 65, 100, 128, 129, 200, 1024])
def test_by_rank(rank, out):
    check(1, 200, 300, rank, 3, out, chosen=torch.tensor([2], device="cuda"))
    check(37, 130, 257, rank, 5, out, pad=3)
    check(70, 96, 128, rank, 2, out, run=20, pad=8)


@pytest.mark.parametrize("out", DTYPES)
@pytest.mark.parametrize("n,k", [(1, 1), (1, 64), (64, 1), (7, 9), (15, 31), (16, 32), (17, 33), (63, 65), (64, 64), (100, 1000), (129, 2050), (1000, 100), (4099, 4083)])
def test_by_columns(n, k, out):
    for m, adapters, run in ((1, 1, 1), (5, 3, 1), (40, 40, 1), (130, 4, 30)):
        check(m, n, k, 16, adapters, out, run, pad=3 if n % 2 else 0, seed=7)
        check(m, n, k, 12, adapters, out, run, seed=8, scales=False, index=torch.int64)


@pytest.mark.parametrize("m,adapters,run", [(1, 48, 1), (2, 1, 1), (15, 2, 1), (16, 1, 1), (17, 1, 17), (64, 200, 1), (96, 40, 1), (255, 3, 1), (256, 16, 1), (257, 16, 1),
                                            (300, 1, 300), (500, 5, 7), (1000, 48, 1), (1025, 2, 1), (2000, 3, 300), (3000, 700, 2), (5000, 33, 77), (9001, 16, 300)])
def test_by_rows(m, adapters, run):
    check(m, 320, 256, 16, adapters, "f32", run, seed=9)
    check(m, 200, 520, 40, adapters, "bf16", run, pad=8, seed=10)


def test_all_rows_of_one_adapter_and_none_at_all():
    for m in (1, 20, 300, 1500):
        check(m, 256, 256, 32, 6, chosen=torch.full((m,), 5, device="cuda"), seed=11)
        check(m, 256, 256, 32, 6, chosen=torch.full((m,), -1, device="cuda"), seed=12)
        check(m, 256, 256, 32, 6, chosen=torch.full((m,), 1 << 40, device="cuda"), index=torch.int64, seed=12)


def test_more_adapters_than_rows_by_far():
    check(3, 64, 64, 2, 65536, chosen=torch.tensor([65535, 0, 65536], device="cuda"), seed=13)
    check(600, 64, 64, 2, 65536, seed=14)


@pytest.mark.parametrize("m,run", [(3, 1), (90, 1), (700, 50)])
def test_sums_that_are_exact(m, run):
    """Whole numbers: a term that is lost or added twice shows.  (|h| <= 320 * 9, * 3 * rank 48 < 2^24)"""
    print("case: exact sums", m, flush=True)
    n, k, rank, adapters = 333, 320, 48, 7
    g = torch.Generator("cuda").manual_seed(15)
    x, down, up = (torch.randint(-3, 4, s, generator=g, device="cuda").to(torch.bfloat16) for s in ((m, k), (adapters, rank, k), (adapters, n, rank)))
    chosen = torch.randint(-1, adapters, ((m + run - 1) // run,), generator=g, device="cuda").repeat_interleave(run)[:m].int()
    out = torch.randint(-100, 100, (m, n), generator=g, device="cuda").float()
    w = R.Adapters(down, up, torch.tensor([1.0, 2.0, -1.0, 0.5, 4.0, 0.0, -2.0], device="cuda"))
    want, _ = exact(x, w, chosen, out)
    R.adapter_linear(x, w, chosen, out, R.adapter_linear_workspace(m, w))
    assert torch.equal(out.double(), want)


def test_between_the_products_nothing_is_rounded_to_fewer_bits():
    """h = 1 + 2^-20 and -1, which cancel: 16 bits between the products would lose what is left."""
    print("case: cancelling", flush=True)
    k, n, rank = 64, 48, 16
    down = torch.zeros(1, rank, k, dtype=torch.bfloat16, device="cuda")
    down[0, 0, 0], down[0, 0, 1], down[0, 1, 0] = 1.0, 2.0 ** -20, -1.0
    x, up = torch.ones(5, k, dtype=torch.bfloat16, device="cuda"), torch.ones(1, n, rank, dtype=torch.bfloat16, device="cuda")
    out, w = torch.zeros(5, n, device="cuda"), R.Adapters(down, up)
    R.adapter_linear(x, w, torch.zeros(5, dtype=torch.int32, device="cuda"), out, R.adapter_linear_workspace(5, w))
    assert (out == 2.0 ** -20).all()


def test_infinities_stay_in_their_rows():
    print("case: infinities", flush=True)
    for m, adapters in ((6, 2), (400, 2)):
        x, w, chosen, kept, _ = check(m, 100, 80, 9, adapters, "f32", chosen=torch.arange(m, device="cuda") % 2, seed=16)
        x[2, 5] = float("inf")
        w.up[1, 30, :] = float("nan")
        out = kept.clone()
        R.adapter_linear(x, w, chosen.int(), out, R.adapter_linear_workspace(m, w))
        bad = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
        bad[2], bad[1::2, 30] = True, True
        assert (~out[bad].isfinite()).all() and out[~bad].isfinite().all()


def test_large_outputs():
    """Beyond 2^32 bytes."""
    check(70000, 16000, 64, 8, 3, "f32", 5000, seed=17)


def test_the_same_bits_twice_and_in_a_graph():
    print("case: graph", flush=True)
    for m, run in ((10, 1), (600, 60)):
        x, w, chosen, kept, got = check(m, 300, 512, 24, 5, "bf16", run, seed=18)
        ws, out, chosen = R.adapter_linear_workspace(m, w), kept[:, :300].clone(), chosen.int()
        R.adapter_linear(x, w, chosen, out, ws)
        assert torch.equal(out, got)
        graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            R.adapter_linear(x, w, chosen, out, ws)
        for seed in range(3):
            chosen.copy_(torch.randint(-1, 5, (m,), generator=torch.Generator("cuda").manual_seed(seed), device="cuda"))
            out.copy_(kept[:, :300])
            R.adapter_linear(x, w, chosen, out, ws)
            want = out.clone()
            out.copy_(kept[:, :300])
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)


def test_nothing_to_do():
    for m, n, k, rank, adapters in ((0, 8, 8, 2, 3), (4, 0, 8, 2, 3), (4, 8, 0, 2, 3), (4, 8, 8, 0, 3), (4, 8, 8, 2, 0)):
        print("case: nothing", m, n, k, rank, adapters, flush=True)
        w = R.Adapters(torch.zeros(adapters, rank, k, dtype=torch.bfloat16, device="cuda"), torch.ones(adapters, n, rank, dtype=torch.bfloat16, device="cuda"))
        out = torch.full((m, n), 3.0, device="cuda")
        R.adapter_linear(torch.zeros(m, k, dtype=torch.bfloat16, device="cuda"), w, torch.zeros(m, dtype=torch.int32, device="cuda"), out, R.adapter_linear_workspace(m, w))
        assert (out == 3).all()


@pytest.mark.parametrize("out", DTYPES)
@pytest.mark.parametrize("rank,m", [(1, 66000), (3, 22000), (8, 8300), (15, 4400), (17, 3900), (33, 2000), (50, 1400), (64, 1100), (65, 1100), (100, 1100), (129, 1100),
                                    (200, 1100), (1024, 1100)])
def test_many_rows_by_rank(rank, m, out):
    """Enough rows and ranks for groups of 64."""
    check(m, 130, 257, rank, 2, out, pad=3, seed=21)
    check(m, 96, 128, rank, 5, out, run=50, pad=8, seed=22, index=torch.int64, scales=False)


@pytest.mark.parametrize("out", DTYPES)
@pytest.mark.parametrize("n,k", [(1, 1), (1, 64), (64, 1), (7, 9), (15, 31), (17, 33), (63, 65), (100, 1000), (129, 2050), (1000, 100), (4099, 4083)])
def test_many_rows_by_columns(n, k, out):
    check(1111, n, k, 64, 3, out, 1, pad=3 if n % 2 else 0, seed=23)
    check(1111, n, k, 60, 4, out, 300, seed=24)


@pytest.mark.parametrize("m", [1, 15, 16, 17, 63, 64, 65, 100, 127, 128, 129])
def test_few_rows_however_they_are_distributed(m):
    """All of one adapter, each its own, two in turn, one row apart: groups of 16 that begin anywhere."""
    place = torch.arange(m, device="cuda")
    for chosen in (place * 0 + 3, place, place % 2, (place > m // 2).long() * 7 - 1, torch.where(place == m // 3, 2, 6), place // 17, place * 0 - 1):
        check(m, 70, 90, 10, 130, "f32", chosen=chosen, seed=25)
        check(m, 70, 90, 10, 8, "bf16", chosen=chosen, seed=26)
