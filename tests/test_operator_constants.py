"""The binding's constants of the operators are the header's, and sums too long for a product's offsets are refused."""
import os
import re

from paper_2605_06534_amd import binding

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "rose_delta.h")


def test_constants_are_the_header_s():
    text = open(HEADER).read()
    value = dict(re.findall(r"#define\s+(ROSE_\w+)\s+(\d+)\b", text))
    assert int(value["ROSE_GRAD_WORKSPACE_BYTES"]) == binding.GRAD_WORKSPACE_BYTES
    assert int(value["ROSE_MX4_BLOCK"]) == binding.MX4_BLOCK
    types = dict(re.findall(r"(ROSE_DTYPE_\w+)\s*=\s*(\d+)", text))
    assert {k: int(v) for k, v in types.items()} == {"ROSE_DTYPE_BF16": binding.DTYPE_BF16, "ROSE_DTYPE_F32": binding.DTYPE_F32}


def test_sums_that_are_too_long_for_a_product():
    p = 1 << 20
    k = 1 << 24
    f = binding._lib.rose_mx4_matmul
    assert f(p, p, 1, p, p, 1, k, p, binding.DTYPE_F32, 1, None) == binding.ERR_UNSUPPORTED


def test_codes_and_scales_have_the_sizes_that_the_header_states():
    q = binding.Mx4(3, 33, device="cpu")              # a row of two blocks
    assert tuple(q.codes.shape) == (3, 2 * binding.MX4_BLOCK // 2) and tuple(q.scales.shape) == (3, 2)
