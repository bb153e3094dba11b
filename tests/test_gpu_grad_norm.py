"""The norm of many gradients together and clipping by it, against the definition in 64 bits.

Bounds: squares and sums are formed in 64 bits, so the sum is off by at most total * 2^-52 of itself.  The norm is
rounded to fp32 (2^-24 of it); norm + 1e-6, the quotient and the product are rounded once each: a scaled gradient is off
by at most 4 * 2^-24 of itself (2 % more for what the first order leaves out), and by half a unit in the last place of
bf16 (2^-8 of it: eight significant bits) where it is rounded to that."""
import math

import numpy as np
import pytest
import torch

import paper_2605_06534_amd as R

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16]
IDS = ["f32", "bf16"]


def layout(numels, dtype, seed, gap, std=1.0):
    """Tensors one behind the other in one buffer, `gap` elements between them; the buffer begins with one of those."""
    g = torch.Generator().manual_seed(seed)
    flat = (torch.randn(sum(numels) + gap * (len(numels) + 1), generator=g) * std).to(dtype).cuda()
    at, views = gap, []
    for n in numels:
        views.append(flat[at:at + n])
        at += n + gap
    return flat, views


def true_norm(views):
    return math.sqrt(sum(float((v.double() ** 2).sum()) for v in views))


SETS = {
    "one": [1],
    "nothing": [0, 0],
    "few": [3, 0, 1, 17, 5],
    "around_a_share": [8191, 1, 8192, 8193, 16384],
    "many_small": [1 + i % 37 for i in range(3000)],
    "large": [5000000, 7, 3000001, 64, 0, 2999],
}


def expected(views, max_norm):
    norm = true_norm(views)
    factor = min(1.0, max_norm / (norm + 1e-6))
    return norm, [v.double().cpu().numpy() * factor for v in views]


def near(got, want, dtype, changed=True):
    off = np.abs(got.double().cpu().numpy() - want)
    bound = np.abs(want) * (1.02 * 4 * 2.0 ** -24 + (torch.finfo(dtype).eps / 2 if dtype == torch.bfloat16 else 0)) + 2.0 ** -134
    assert (off <= bound).all(), (off - bound).max()


@pytest.mark.parametrize("gap", [0, 1, 3, 16])
@pytest.mark.parametrize("name", SETS)
@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
def test_clip(dtype, name, gap):
    print("case: clip", dtype, name, gap, flush=True)
    numels = SETS[name]
    total = sum(numels)
    flat, views = layout(numels, dtype, 21, gap)
    kept = flat.clone()
    out, outs = layout(numels, dtype, 22, gap)
    untouched = out.clone()
    tab, out_tab, offsets = R.ptr_table(views), R.ptr_table(outs), R.offset_table(numels)
    ws, norm = R.grad_workspace(), torch.zeros(1, device="cuda")
    s = torch.zeros(1, dtype=torch.float64, device="cuda")
    norm64 = true_norm(views)
    for max_norm in (norm64 / 3, norm64 * 2 + 1, 0.0, float("inf")):
        ws.fill_(0xA5)
        R.grad_clip_norm(tab, offsets, total, dtype, out_tab, max_norm, norm, ws)
        _, want = expected(views, max_norm)
        assert abs(norm.item() - norm64) <= norm64 * (2.0 ** -24 + total * 2.0 ** -53)
        for o, w in zip(outs, want):
            near(o, w, dtype)
        assert torch.equal(flat, kept)                            # out of place: the gradients stay
        if max_norm > norm64:
            assert all(torch.equal(o, v) for o, v in zip(outs, views))
        # in two calls, as ranks do that add their sums up in between: the same bits
        two, twos = layout(numels, dtype, 22, gap)
        R.grad_sum_squares(tab, offsets, total, dtype, s, ws)
        assert abs(s.item() - norm64 ** 2) <= norm64 ** 2 * (total + 8) * 2.0 ** -52
        norm2 = torch.zeros(1, device="cuda")
        R.grad_clip(tab, offsets, total, dtype, R.ptr_table(twos), s, max_norm, norm2)
        assert norm2.item() == norm.item() and all(torch.equal(o, v) for o, v in zip(outs, twos))
        # in place
        inplace = flat.clone()
        at, same = gap, []
        for n in numels:
            same.append(inplace[at:at + n])
            at += n + gap
        t = R.ptr_table(same)
        R.grad_clip_norm(t, offsets, total, dtype, t, max_norm, None, ws)
        assert all(torch.equal(o, v) for o, v in zip(outs, same))
    # between the tensors nothing was written
    mask = torch.ones_like(out, dtype=torch.bool)
    at = gap
    for n in numels:
        mask[at:at + n] = False
        at += n + gap
    assert torch.equal(out[mask], untouched[mask])


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
def test_outputs_elsewhere_than_inputs(dtype):
    """Inputs and outputs that lie differently to the 16-byte vectors."""
    print("case: clip, other alignment", dtype, flush=True)
    numels = [1000, 33, 20001]
    _, views = layout(numels, dtype, 23, 1)
    _, outs = layout(numels, dtype, 24, 2)
    norm = torch.zeros(1, device="cuda")
    R.grad_clip_norm(R.ptr_table(views), R.offset_table(numels), sum(numels), dtype, R.ptr_table(outs), 1.0, norm, R.grad_workspace())
    for o, w in zip(outs, expected(views, 1.0)[1]):
        near(o, w, dtype)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
def test_extreme_sizes_of_values(dtype):
    """Squares beyond fp32's range on either side."""
    print("case: clip, extreme values", dtype, flush=True)
    for std in (1e30, 1e-30):
        _, views = layout([4000, 100], dtype, 25, 1, std)
        _, outs = layout([4000, 100], dtype, 26, 1)
        norm = torch.zeros(1, device="cuda")
        n64 = true_norm(views)
        R.grad_clip_norm(R.ptr_table(views), R.offset_table([4000, 100]), 4100, dtype, R.ptr_table(outs), n64 / 7, norm, R.grad_workspace())
        assert abs(norm.item() - n64) <= n64 * 1.01 * 2.0 ** -24
        for o, w in zip(outs, expected(views, n64 / 7)[1]):
            near(o, w, dtype)


def test_null_pointers_and_parts():
    """A replicated tensor that another rank counts: its sum is left out, its gradient is scaled all the same."""
    print("case: clip with tensors left out", flush=True)
    numels = [500, 70, 9000]
    _, views = layout(numels, torch.float32, 27, 1)
    offsets, ws = R.offset_table(numels), R.grad_workspace()
    tab = R.ptr_table(views)
    counted = tab.clone()
    counted[1] = 0
    s = torch.zeros(1, dtype=torch.float64, device="cuda")
    R.grad_sum_squares(counted, offsets, sum(numels), torch.float32, s, ws)
    part = true_norm([views[0], views[2]])
    assert abs(s.item() - part ** 2) <= part ** 2 * 1e-12
    s += float((views[1].double() ** 2).sum())        # the other rank's sum
    want = expected(views, 2.0)[1]
    R.grad_clip(tab, offsets, sum(numels), torch.float32, tab, s, 2.0)
    for v, w in zip(views, want):
        near(v, w, torch.float32)
    kept = [v.clone() for v in views]
    out_tab = tab.clone()
    out_tab[0] = 0
    R.grad_clip(tab, offsets, sum(numels), torch.float32, out_tab, s, 0.0)
    assert torch.equal(views[0], kept[0]) and (views[1] == 0).all() and (views[2] == 0).all()


def test_ranks_of_a_plan_count_every_gradient_once():
    """A plan says which rank sends, and so may count, a replicated tensor: the ranks' sums are the whole model's."""
    print("case: sums of the ranks of a plan", flush=True)
    from workloads import models
    ts = models.decoder(2, 256, 4, 4, 64, 512, 1000, fused=True)
    g = torch.Generator().manual_seed(28)
    whole = [torch.randn(t["rows"], t["cols"], generator=g).cuda() for t in ts]
    total, tp = 0.0, 2
    for rank in range(tp):
        plan = R.shard_plan(ts, 4, tp, rank)
        mine = R.shard_plan(ts, tp)                   # a rank holds what a receiver of the same degree would
        local = [torch.empty(plan.src_numel(t), dtype=torch.float32, device="cuda") for t in range(len(ts))]
        for t, (d, w) in enumerate(zip(ts, whole)):
            if d["rule"] == R.REPLICATED:
                part = w
            elif d["rule"] == R.SPLIT_COLS:
                part = w.chunk(tp, 1)[rank]
            else:
                part = torch.cat([s.chunk(tp, 0)[rank] for s in w.split(d["sections"] or [d["rows"]], 0)])
            local[t].copy_(part.reshape(-1))
            assert mine.local_numel(t, rank) == plan.src_numel(t)
        tab = R.ptr_table(local)
        for t in range(len(ts)):
            if not plan.tensor_is_read(t):
                tab[t] = 0
        s = torch.zeros(1, dtype=torch.float64, device="cuda")
        numels = [x.numel() for x in local]
        R.grad_sum_squares(tab, R.offset_table(numels), sum(numels), torch.float32, s, R.grad_workspace())
        total += s.item()
    want = true_norm(whole) ** 2
    assert abs(total - want) <= want * 1e-12


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
def test_norms_that_are_no_numbers(dtype):
    print("case: clip with infinities and NaN", dtype, flush=True)
    for bad, rest in ((float("inf"), 0.0), (float("nan"), float("nan"))):
        _, views = layout([300, 50], dtype, 29, 1)
        views[1][7] = bad
        _, outs = layout([300, 50], dtype, 30, 1)
        norm = torch.zeros(1, device="cuda")
        R.grad_clip_norm(R.ptr_table(views), R.offset_table([300, 50]), 350, dtype, R.ptr_table(outs), 1.0, norm, R.grad_workspace())
        assert torch.isnan(norm).item() if math.isnan(bad) else norm.item() == bad
        assert torch.isnan(outs[1][7]).item()         # inf * 0, or NaN
        others = torch.cat([outs[0], outs[1][:7], outs[1][8:]]).float()
        assert torch.isnan(others).all() if math.isnan(rest) else (others == 0).all()


def test_a_total_that_is_wrong_costs_nothing_but_speed():
    print("case: clip with another total", flush=True)
    numels = [70000, 3, 50001]
    _, views = layout(numels, torch.bfloat16, 31, 1)
    want = true_norm(views)
    for total in (0, 1, 50000, 1 << 40):
        s = torch.zeros(1, dtype=torch.float64, device="cuda")
        R.grad_sum_squares(R.ptr_table(views), R.offset_table(numels), total, torch.bfloat16, s, R.grad_workspace())
        assert abs(s.item() - want ** 2) <= want ** 2 * 1e-12


def test_in_a_graph():
    print("case: clip in a graph", flush=True)
    numels = [30000, 5, 40001]
    flat, views = layout(numels, torch.float32, 32, 1)
    _, outs = layout(numels, torch.float32, 33, 1)
    tab, out_tab, offsets, ws = R.ptr_table(views), R.ptr_table(outs), R.offset_table(numels), R.grad_workspace()
    norm = torch.zeros(1, device="cuda")

    def step():
        R.grad_clip_norm(tab, offsets, sum(numels), torch.float32, out_tab, 3.0, norm, ws)

    step()
    torch.cuda.synchronize()
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            step()
    torch.cuda.synchronize()
    for rep in range(4):
        flat.mul_(1.5)
        ws.fill_(rep)
        g.replay()
        torch.cuda.synchronize()
        got, n = [o.clone() for o in outs], norm.item()
        step()
        assert n == norm.item() and all(torch.equal(a, b) for a, b in zip(got, outs))
