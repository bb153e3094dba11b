"""One workspace for batches of all lengths, made for the longest: on either side of where blocks of sorted tokens double, and of
where one workgroup sorts.  Gradients of small whole numbers, whose sums are exact."""
import pytest
import torch

import paper_2605_06534_amd as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols,lengths", [(500, 5120, (1, 33, 16384, 16385, 40000, 52428, 52429, 104857, 104858, 110000)),
                                               (3000, 520, (16384, 262144, 262145, 524288, 524289, 530000))])
def test_a_workspace_for_the_longest(rows, cols, lengths):
    print("case: one workspace", rows, cols, flush=True)
    g = torch.Generator("cuda").manual_seed(91)
    longest = max(lengths)
    dy = torch.randint(-3, 4, (longest, cols), generator=g, device="cuda").to(torch.bfloat16)
    tokens = torch.randint(0, rows + 5, (longest,), generator=g, device="cuda")
    buffer = torch.full((R.embedding_grad_workspace(rows, cols, longest).numel() + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    ws, behind = buffer[:-4096], buffer[-4096:]
    for n in lengths:
        want = torch.zeros(rows + 5, cols, device="cuda").index_add_(0, tokens[:n], dy[:n].float())[:rows]
        for space in (ws, R.embedding_grad_workspace(rows, cols, n)):
            grad = torch.full((rows, cols), 9.0, device="cuda")
            R.embedding_grad(dy[:n], tokens[:n], grad, space)
            assert torch.equal(grad, want), n
        assert (behind == 0xA5).all()
