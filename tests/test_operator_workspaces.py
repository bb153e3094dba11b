"""The workspace of a gradient or a product never shrinks where one of its sizes grows: a program that keeps one for its
largest call has enough for all."""
import ctypes
import random

import pytest

from paper_2605_06534_amd import binding


def need(name, *sizes):
    v = ctypes.c_size_t()
    assert getattr(binding._lib, name)(*sizes, ctypes.byref(v)) == binding.OK
    return v.value


STEPS = {
    "rows": [1, 500, 19008, 19009, 1 << 18, (1 << 18) + 1, 1 << 22, 1 << 30],
    "cols": [1, 8, 9, 96, 511, 512, 513, 1024, 1025, 4096, 5119, 5120, 5121, 5632, 5640, 8192, 70001, 1 << 24],
    "tokens": [0, 1, 31, 32, 33, 64, 65, 1000, 4097, 16383, 16384, 16385, 32769, 40000, 52428, 52429, 52430, 65536, 104858, 262144,
               524288, 524289, 530000, 1 << 20, 3355444, 6710887, 1 << 23, 1 << 26, (1 << 31) - 1],
}


@pytest.mark.parametrize("grows", STEPS)
def test_gradient_workspaces_never_shrink(grows):
    for rows in STEPS["rows"]:
        for cols in STEPS["cols"]:
            for tokens in STEPS["tokens"]:
                at = dict(rows=rows, cols=cols, tokens=tokens)
                if at[grows] != STEPS[grows][0]:
                    continue
                sizes = [need("rose_embedding_grad_workspace_bytes", *dict(at, **{grows: step}).values()) for step in STEPS[grows]]
                assert sizes == sorted(sizes), (at, grows, sizes)


def test_gradient_workspaces_between_the_steps():
    rng = random.Random(7)
    for _ in range(20000):
        large = [int(2 ** rng.uniform(0, 23)), int(2 ** rng.uniform(0, 14)), int(2 ** rng.uniform(0, 20))]
        small = [max(1, int(v * rng.uniform(0.3, 1))) if rng.random() < 0.7 else v for v in large]
        assert need("rose_embedding_grad_workspace_bytes", *small) <= need("rose_embedding_grad_workspace_bytes", *large), (small, large)


def test_product_workspaces_never_shrink():
    rng = random.Random(8)
    for _ in range(5000):
        large = [int(2 ** rng.uniform(0, 15)), int(2 ** rng.uniform(0, 15)), int(2 ** rng.uniform(0, 15))]
        small = [max(1, int(v * rng.uniform(0.3, 1))) if rng.random() < 0.7 else v for v in large]
        assert need("rose_mx4_linear_workspace_bytes", *small) <= need("rose_mx4_linear_workspace_bytes", *large), (small, large)
