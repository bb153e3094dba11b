"""Gradients of an embedding whose sums are exact: whole numbers with all sums below 2^24 and a power of two for the scale, so that
one token lost or added twice among thousands shows.  Rows whose tokens cross the ends of so many blocks of 32 sorted tokens."""
import pytest
import torch

import paper_2605_06534_amd as R

pytestmark = pytest.mark.gpu


def check(tokens, rows, cols, dy_dtype, grad_dtype, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    n, most = len(tokens), 3 if dy_dtype == torch.bfloat16 else 500
    dy = torch.randint(-most, most + 1, (n, cols + 1), generator=g, device="cuda").to(dy_dtype)[:, :cols]
    old = torch.randint(-99, 100, (rows, cols), generator=g, device="cuda").to(grad_dtype)
    tokens = tokens[torch.randperm(n, generator=g, device="cuda")]
    here = (tokens >= 0) & (tokens < rows)
    sums = torch.zeros(rows, cols, dtype=torch.float64, device="cuda").index_add_(0, tokens[here], dy[here].double())
    assert dy.abs().double().sum(0).max() < 1 << 24
    named = torch.zeros(rows, dtype=torch.bool, device="cuda")
    named[tokens[here]] = True
    ws = R.embedding_grad_workspace(rows, cols, n)
    for accumulate in (False, True):
        grad = old.clone()
        R.embedding_grad(dy, tokens, grad, ws, scale=0.5, accumulate=accumulate)
        # (below 2^24 the sum in fp32 is exact, halves included where old is added; then one rounding)
        want = (0.5 * sums + (old.double() if accumulate else 0)).float().to(grad_dtype)
        assert torch.equal(grad, want), (accumulate, (grad != want).nonzero()[:5].tolist())


@pytest.mark.parametrize("offset", [0, 1, 31])
@pytest.mark.parametrize("blocks", [1, 2, 3, 7, 8, 9, 15, 16, 17, 18, 33, 64, 65, 66, 130, 500])
def test_one_row_across_many_blocks(blocks, offset):
    """The run begins `offset` tokens into a block, or where one begins, and ends the same way or a token on."""
    print("case: exact gradient, one row", blocks, offset, flush=True)
    for cols, dt, gt in ((24, torch.bfloat16, torch.float32), (1030, torch.float32, torch.float32), (520, torch.bfloat16, torch.bfloat16),
                         (257, torch.float32, torch.bfloat16)):
        for more in (-1, 0, 1):
            length = 32 * blocks + more
            ids = torch.cat([torch.full((offset,), 1), torch.full((length,), 2), torch.arange(40) % 7 - 1, torch.full((3,), 77)])
            # (-1 and 77 are tokens of no row)
            check(ids.cuda(), 6, cols, dt, gt, 100 + blocks)


@pytest.mark.parametrize("n,rows,cols", [(5000, 3, 40), (16384, 50, 513), (16385, 50, 513), (60000, 900, 300), (70000, 2, 1500), (30000, 1, 2050),
                                         (140000, 17, 2100)])
@pytest.mark.parametrize("dt,gt", [(torch.bfloat16, torch.float32), (torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16)],
                         ids=["bf16_f32", "f32_f32", "bf16_bf16"])
def test_rows_with_many_tokens(n, rows, cols, dt, gt):
    """Long blocks too: sums of up to 140000 terms of 3 (of 500: fewer)."""
    print("case: exact gradient, many tokens", n, rows, cols, dt, gt, flush=True)
    if dt == torch.float32:
        n = min(n, 33000)                              # 33000 x 500 < 2^24
    g = torch.Generator("cuda").manual_seed(111)
    # most tokens name the first rows
    ids = (torch.rand(n, generator=g, device="cuda") ** 4 * (rows + 1)).long() - (torch.rand(n, generator=g, device="cuda") < 0.01).long() * 99999
    check(ids, rows, cols, dt, gt, 112)
