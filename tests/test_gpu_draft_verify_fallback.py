"""Where a refused draft leaves nothing of the target, the sample is one of the target: over one part of a row and over many, over one step of
a part and over several (of more than 262144 columns), with samples in the first, a middle and the last of them.  Whole numbers, equal to
the definition's in 64 bits."""
import pytest
import torch

import paper_2605_06534_amd as R
from test_gpu_draft_verify import DTYPES, check, definition, run

pytestmark = pytest.mark.gpu

COLS = [1000, 4096, 4097, 12289, 40001, 262145, 300001]
NUMBERS = [0.0, 1e-6, 0.02, 0.3, 0.5, 0.77, 0.99, 1.0 - 2.0 ** -24]


def rows_of(n, cols, dtype, seed):
    z = torch.randn(n, cols, generator=torch.Generator("cuda").manual_seed(seed), device="cuda") * 2
    z[:, [0, cols // 2, cols - 1]] = -float("inf")               # columns of probability zero in the first, a middle and the last part
    return torch.softmax(z, 1).to(DTYPES[dtype])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", COLS)
def test_target_and_draft_alike(cols, dtype):
    """A drafted token of probability zero under both does not stay, and max(p - q, 0) is zero everywhere."""
    print("case: target and draft alike", cols, dtype, flush=True)
    requests = 2 * len(NUMBERS)
    lengths = torch.tensor([1 + r % 3 for r in range(requests)], device="cuda")
    offsets = torch.cat((torch.zeros(1, dtype=torch.int64, device="cuda"), lengths.cumsum(0)))
    n = int(offsets[-1])
    target = rows_of(n + requests, cols, dtype, 1)
    request = torch.repeat_interleave(torch.arange(requests, device="cuda"), lengths)
    draft = target[torch.arange(n, device="cuda") + request].clone()
    at = torch.tensor([0, cols // 2, cols - 1], device="cuda")
    drafted, u = at[torch.arange(n, device="cuda") % 3], torch.full((n + requests,), 0.5, device="cuda")
    last = offsets[1:] + torch.arange(requests, device="cuda")
    u[last] = torch.tensor(NUMBERS, device="cuda").repeat(2)
    # every other request's first token stays, where it has more than one
    for r in range(0, requests, 2):
        if lengths[r] > 1:
            drafted[offsets[r]] = cols // 3
            u[offsets[r] + r] = 0.0
    kept = check(target, draft, drafted, offsets, u)
    assert 0 in kept and 1 in kept
    tokens, _ = run(target, draft, drafted, offsets, u)
    if cols in (40001, 300001):                   # samples of the first 4096 columns, of the last ones, and between (elsewhere the last are one of probability zero)
        samples = tokens[offsets[:-1] + torch.arange(requests, device="cuda") + torch.tensor(kept, device="cuda")]
        assert (samples < 4096).any() and (samples >= (cols - 1) // 4096 * 4096).any() and ((samples >= 4096) & (samples < cols - 4096)).any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", COLS)
def test_all_that_there_is_refused(cols, dtype):
    """Drafts without probabilities: a row whose only weight is the refused token's, and one whose refused token is out of range."""
    print("case: all of it refused", cols, dtype, flush=True)
    places = [0, 1, cols // 3, cols // 2, cols - 2, cols - 1]
    target = torch.zeros(2 * len(places), cols, device="cuda")
    for r, at in enumerate(places):
        target[2 * r:2 * r + 2, at] = 0.5
    target = target.to(DTYPES[dtype])
    offsets = torch.arange(len(places) + 1, device="cuda")
    u = torch.full((2 * len(places),), 0.75, device="cuda")      # 0.75 < 0.5 does not hold
    for drafted in (torch.tensor(places, device="cuda"), torch.tensor([-1, cols, 1 << 40, -(1 << 40), cols + 1, -2], device="cuda")):
        assert check(target, None, drafted, offsets, u) == [0] * len(places)
        tokens, _ = run(target, None, drafted, offsets, u)
        assert tokens.view(-1, 2)[:, 0].tolist() == places


def test_beside_requests_of_other_kinds_and_in_a_graph():
    print("case: a mixture in a graph", flush=True)
    cols, lengths = 40001, [0, 1, 3, 1, 0, 2]
    offsets = torch.tensor([0, 0, 1, 4, 5, 5, 7], device="cuda")
    target = rows_of(13, cols, "f32", 5)
    draft = rows_of(7, cols, "f32", 6)
    draft[0], draft[4] = target[1], target[7]                    # requests 1 and 3: nothing is left
    drafted = torch.tensor([0, 17, 0, 900, cols - 1, 40000, 5], device="cuda")
    u = torch.rand(13, generator=torch.Generator("cuda").manual_seed(7), device="cuda")
    check(target, draft, drafted, offsets, u)
    tokens, accepted, ws = torch.empty(13, dtype=torch.int64, device="cuda"), torch.empty(6, dtype=torch.int32, device="cuda"), R.draft_verify_workspace(6, cols)
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        R.draft_verify(target, draft, drafted, offsets, u, tokens, accepted, ws)
    for seed in range(4):
        u.copy_(torch.rand(13, generator=torch.Generator("cuda").manual_seed(seed), device="cuda"))
        want = definition(target, draft, drafted, offsets, u)
        tokens.fill_(5), accepted.fill_(5)
        graph.replay()
        torch.cuda.synchronize()
        assert tokens.tolist() == want[0] and accepted.tolist() == want[1]
