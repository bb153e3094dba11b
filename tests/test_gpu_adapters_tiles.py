"""Adapters of many rows, which go through tiles of 64 rows: sums that are exact, 24 bits between the products, rows that stay by themselves,
empty groups, repeated and captured calls.  That these sizes go that way is shown on the host by their launches: a sort, the first product, the
cutting, the second product; groups of 16 rows do without the cutting."""
import pytest
import torch

import paper_2605_06534_amd as R
from paper_2605_06534_amd import binding
from test_gpu_adapters import check, exact
from test_operator_launches import launched, recorder  # noqa: F401  (recorder: a fixture)

P, WORK = 1 << 20, 1 << 62

# rows, n, k, rank, adapters
EXACT = [(1500, 333, 320, 48, 7), (2100, 130, 1030, 33, 3), (1100, 257, 64, 70, 4), (1100, 64, 300, 150, 2)]
CANCELS = (4200, 72, 128, 16, 1)
INFINITIES = (8000, 100, 80, 9, 2)
UNEVEN = (2100, 256, 256, 32, 6)
GRAPH = (3000, 300, 512, 24, 5)


def test_these_sizes_go_in_tiles(recorder):  # noqa: F811
    calls = [("rose_adapter_linear", (P, m, k, k, P, P, None, adapters, rank, P, 4, P, dt, n, n, P, WORK, None))
             for m, n, k, rank, adapters in EXACT + [CANCELS, INFINITIES, UNEVEN, GRAPH] for dt in (binding.DTYPE_BF16, binding.DTYPE_F32)]
    for call, (status, launches) in zip(calls, launched(recorder, calls)):
        assert status == binding.OK and len(launches) == 4, (call, launches)
    # (and one that does not: rows times ranks are too few)
    (status, launches), = launched(recorder, [("rose_adapter_linear", (P, 600, 512, 512, P, P, None, 5, 24, P, 4, P, binding.DTYPE_F32, 300, 300, P, WORK, None))])
    assert status == binding.OK and len(launches) == 3


@pytest.mark.gpu
@pytest.mark.parametrize("index", [torch.int32, torch.int64])
@pytest.mark.parametrize("run", [1, 50, 700])
@pytest.mark.parametrize("sizes", EXACT, ids=str)
def test_sums_that_are_exact(sizes, run, index):
    """Whole numbers, and halves: a term that is lost or added twice shows.  (|scale * h| <= 4 * 9 * k, * 3 * rank < 2^23)"""
    m, n, k, rank, adapters = sizes
    print("case: exact sums", sizes, run, flush=True)
    g = torch.Generator("cuda").manual_seed(15)
    x, down, up = (torch.randint(-3, 4, s, generator=g, device="cuda").to(torch.bfloat16) for s in ((m, k), (adapters, rank, k), (adapters, n, rank)))
    chosen = torch.randint(-1, adapters, ((m + run - 1) // run,), generator=g, device="cuda").repeat_interleave(run)[:m].to(index)
    out = torch.randint(-100, 100, (m, n), generator=g, device="cuda").float()
    w = R.Adapters(down, up, torch.tensor([1.0, 2.0, -1.0, 0.5, 4.0, 0.0, -2.0], device="cuda")[:adapters])
    want, _ = exact(x, w, chosen, out)
    ws = R.adapter_linear_workspace(m, w)
    ws.fill_(0xFF)
    R.adapter_linear(x, w, chosen, out, ws)
    assert torch.equal(out.double(), want)


@pytest.mark.gpu
def test_between_the_products_nothing_is_rounded_to_fewer_bits():
    """h = 1 + 2^-8 + 2^-16 + 2^-23 and -(1 + 2^-8), which cancel but for the last 8 of 24 bits.  (Terms of h lie 32 elements apart, so that they
    are added one after the other; each of its three parts then cancels, or is left, by itself.)"""
    m, n, k, rank, adapters = CANCELS
    print("case: cancelling", flush=True)
    down = torch.zeros(adapters, rank, k, dtype=torch.bfloat16, device="cuda")
    for i, v in enumerate((1.0, 2.0 ** -8, 2.0 ** -16, 2.0 ** -23)):
        down[0, 0, 32 * i] = v
        if i < 2:
            down[0, 1, 32 * i] = -v
    x, up = torch.ones(m, k, dtype=torch.bfloat16, device="cuda"), torch.ones(adapters, n, rank, dtype=torch.bfloat16, device="cuda")
    w, chosen = R.Adapters(down, up), torch.zeros(m, dtype=torch.int32, device="cuda")
    for size in (m, 5, 600):                      # (5, 600: groups of 16)
        out = torch.zeros(size, n, device="cuda")
        R.adapter_linear(x[:size], w, chosen[:size], out, R.adapter_linear_workspace(size, w))
        assert (out == 2.0 ** -16 + 2.0 ** -23).all()


@pytest.mark.gpu
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_infinities_stay_in_their_rows(out):
    m, n, k, rank, adapters = INFINITIES
    print("case: infinities", out, flush=True)
    x, w, chosen, kept, _ = check(m, n, k, rank, adapters, out, chosen=torch.arange(m, device="cuda") % 2, seed=16)
    x[2, 5] = float("inf")
    w.up[1, 30, :] = float("nan")
    got = kept.clone()
    R.adapter_linear(x, w, chosen.int(), got, R.adapter_linear_workspace(m, w))
    bad = torch.zeros(got.shape, dtype=torch.bool, device="cuda")
    bad[2], bad[1::2, 30] = True, True
    assert (~got[bad].isfinite()).all() and got[~bad].isfinite().all()


@pytest.mark.gpu
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_all_rows_of_one_adapter_and_none_at_all(out):
    m, n, k, rank, adapters = UNEVEN
    for a in (0, 5):
        check(m, n, k, rank, adapters, out, chosen=torch.full((m,), a, device="cuda"), seed=11)
    for none in (-1, adapters, 1 << 40):
        check(m, n, k, rank, adapters, out, chosen=torch.full((m,), none, device="cuda"), index=torch.int64, seed=12)
    # one row by itself, groups of 64 that are full and one more
    place = torch.arange(m, device="cuda")
    for chosen in (torch.where(place == 777, 3, -1), torch.where(place < 64, 0, torch.where(place < 129, 4, 2)), place // 65 % 7 - 1, place % 6):
        check(m, n, k, rank, adapters, out, chosen=chosen, seed=13)


@pytest.mark.gpu
def test_the_same_bits_twice_and_in_a_graph():
    m, n, k, rank, adapters = GRAPH
    print("case: graph", flush=True)
    for out_type in ("bf16", "f32"):
        x, w, chosen, kept, got = check(m, n, k, rank, adapters, out_type, 60, seed=18)
        ws, out, chosen = R.adapter_linear_workspace(m, w), kept[:, :n].clone(), chosen.int()
        R.adapter_linear(x, w, chosen, out, ws)
        assert torch.equal(out, got)
        graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            R.adapter_linear(x, w, chosen, out, ws)
        for seed in range(3):
            chosen.copy_(torch.randint(-1, adapters, (m,), generator=torch.Generator("cuda").manual_seed(seed), device="cuda"))
            out.copy_(kept[:, :n])
            R.adapter_linear(x, w, chosen, out, ws)
            want = out.clone()
            out.copy_(kept[:, :n])
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)
