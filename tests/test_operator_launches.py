"""No launch of an operator asks for 2^32 threads or more in a dimension, which is more than a launch can have: shown on the
host, with a stand-in for the runtime's launch function that notes the sizes and starts nothing.  The addresses are never read."""
import json
import os
import subprocess
import sys

import pytest

from paper_2605_06534_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, UNSUPPORTED = binding.OK, binding.ERR_UNSUPPORTED
BF16, F32 = binding.DTYPE_BF16, binding.DTYPE_F32
P = 1 << 20                                         # an aligned address
MOST = (1 << 31) - 1                                # rows, columns and tokens that the operators take

RECORDER = """
#include <stddef.h>
typedef struct { unsigned x, y, z; } dims;
static unsigned long long noted[4096][3];
static int launches;
int hipLaunchKernel(const void *f, dims grid, dims block, void **args, size_t lds, void *stream) {
    if (launches < 4096) {
        noted[launches][0] = (unsigned long long)grid.x * block.x;
        noted[launches][1] = (unsigned long long)grid.y * block.y;
        noted[launches][2] = (unsigned long long)grid.z * block.z;
    }
    ++launches;
    return 0;
}
int hipGetLastError(void) { return 0; }
/* what a launch's sizes go through on their way there */
static dims next_grid, next_block;
static size_t next_lds;
static void *next_stream;
int __hipPushCallConfiguration(dims grid, dims block, size_t lds, void *stream) {
    next_grid = grid, next_block = block, next_lds = lds, next_stream = stream;
    return 0;
}
int __hipPopCallConfiguration(dims *grid, dims *block, size_t *lds, void **stream) {
    *grid = next_grid, *block = next_block, *lds = next_lds, *stream = next_stream;
    return 0;
}
int noted_launches(void) { return launches; }
void forget_launches(void) { launches = 0; }
unsigned long long noted_threads(int launch, int dimension) { return noted[launch][dimension]; }
"""

# The stand-in is loaded for everyone before the library is: its functions are the ones that the library finds.
SCRIPT = """
import ctypes, json, sys
recorder = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
recorder.noted_threads.restype = ctypes.c_ulonglong
sys.path.insert(0, sys.argv[2])
from paper_2605_06534_amd import binding
out = []
for name, args in json.loads(sys.stdin.read()):
    recorder.forget_launches()
    status = getattr(binding._lib, name)(*args)
    out.append((status, [[recorder.noted_threads(i, d) for d in range(3)] for i in range(recorder.noted_launches())]))
print("launches " + json.dumps(out))
"""


@pytest.fixture(scope="module")
def recorder(tmp_path_factory):
    folder = tmp_path_factory.mktemp("recorder")
    source, lib = folder / "recorder.c", folder / "recorder.so"
    source.write_text(RECORDER)
    subprocess.check_call(["gcc", "-shared", "-fPIC", "-O1", str(source), "-o", str(lib)])
    return str(lib)


def launched(recorder, calls):
    """[(status, threads of each launch)] of calls [(name, arguments)]"""
    done = subprocess.run([sys.executable, "-c", SCRIPT, recorder, ROOT], input=json.dumps(calls), capture_output=True, text=True, timeout=600)
    assert done.returncode == 0, done.stderr
    return json.loads([line for line in done.stdout.splitlines() if line.startswith("launches ")][-1][len("launches "):])


def fits(launches):
    return all(0 < threads < 1 << 32 for launch in launches for threads in launch)


def test_the_stand_in_sees_the_launches(recorder):
    (status, launches), = launched(recorder, [("rose_grad_sum_squares", (P, P, 3, 100, F32, P, P, binding.GRAD_WORKSPACE_BYTES, None))])
    assert status == OK and launches == [[256, 1, 1], [256, 1, 1]]


def test_clipping_with_any_total(recorder):
    calls = []
    for dtype in (BF16, F32):
        for total in (0, 1, 1 << 32, 1 << 36, 1 << 37, 1 << 40, (1 << 63) - 1):
            calls += [("rose_grad_sum_squares", (P, P, 3, total, dtype, P, P, binding.GRAD_WORKSPACE_BYTES, None)),
                      ("rose_grad_clip", (P, P, 3, total, dtype, P, P, 1.0, P, None)),
                      ("rose_grad_clip_norm", (P, P, 3, total, dtype, P, 1.0, P, P, binding.GRAD_WORKSPACE_BYTES, None))]
    for call, (status, launches) in zip(calls, launched(recorder, calls)):
        assert status == OK and launches and fits(launches), (call, launches)


@pytest.mark.parametrize("grad", [BF16, F32], ids=["bf16", "f32"])
def test_gradients_of_very_many_rows(recorder, grad):
    """Narrow gradients whose rows without tokens are more than one launch takes eight of a workgroup."""
    calls = [("rose_embedding_grad", (P, BF16, cols, P, 8, n, 0, 1.0, P, grad, rows, cols, stride, 0, P, 1 << 62, None))
             for rows in (1 << 20, (1 << 29) + 1, 600000000, 1 << 30, MOST) for cols, stride in ((1, 1), (1, 2), (7, 7), (9, 9))
             for n in (0, 1, 5, 20000, MOST)]
    for call, (status, launches) in zip(calls, launched(recorder, calls)):
        assert status == OK and launches and fits(launches), (call, launches)


def test_gradients_of_more_than_launches_hold_queue_nothing(recorder):
    """No memory holds these; what is refused is refused before the tokens are sorted."""
    calls = [("rose_embedding_grad", (P, BF16, cols, P, 8, n, 0, 1.0, P, F32, 10, cols, cols, accumulate, P, 1 << 62, None))
             for n, cols in ((MOST, MOST), (1 << 27, MOST), (MOST, 1 << 27)) for accumulate in (0, 1)]
    for call, (status, launches) in zip(calls, launched(recorder, calls)):
        assert status == UNSUPPORTED and not launches, (call, status, launches)


@pytest.mark.parametrize("out", [BF16, F32], ids=["bf16", "f32"])
def test_lookups_of_very_many_vectors(recorder, out):
    calls = [("rose_embedding_lookup", (P, BF16, 100, cols, cols, P, 4, n, 0, 1.0, P, out, cols, None))
             for n, cols in ((1, MOST), (1, 1), (MOST, 1), (MOST, 9), (MOST, 25), (1 << 30, 200), (1 << 24, 5120), (20000, MOST))]
    for call, (status, launches) in zip(calls, launched(recorder, calls)):
        assert status == OK and launches and fits(launches), (call, launches)
        _, (_, _, _, cols, _, _, _, n, *_) = call
        vectors = n * -(-cols // (8 if out == BF16 else 4))
        assert vectors <= 2 * sum(threads for threads, _, _ in launches) < 2 * vectors + 1024 * len(launches)     # one or two a thread


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_4_bit_matrices_of_very_many_vectors(recorder, dtype):
    sizes = [(1, 1), (MOST, 1), (MOST, 33), (1 << 29, 33), (1 << 30, 64), (5, MOST), (1 << 24, 28000)]
    calls = [("rose_mx4_quantize", (P, dtype, rows, cols, cols, P, P, None)) for rows, cols in sizes]
    calls += [("rose_mx4_dequantize", (P, P, rows, cols, P, dtype, cols, None)) for rows, cols in sizes]
    for call, (status, launches), (rows, cols) in zip(calls, launched(recorder, calls), sizes * 2):
        assert status == OK and launches and fits(launches), (call, launches)
        vectors = rows * -(-cols // 32) * (4 if dtype == BF16 else 8)
        assert vectors <= 2 * sum(threads for threads, _, _ in launches) < vectors + 1024 * len(launches)     # two a thread


def test_products_with_very_many_rows_of_weights(recorder):
    calls = [("rose_mx4_matmul", (P, P, m, P, P, n, k, P, out, n, None))
             for m in (1, 16, 17, 40, 64) for n in (1, 6143, 1 << 30, MOST) for k in (32, 4096) for out in (BF16, F32)]
    calls += [("rose_mx4_linear", (P, BF16, m, 33, P, P, n, 33, P, BF16, n, P, 1 << 40, None)) for m in (1, 8) for n in (1 << 30, MOST)]
    calls += [("rose_mx4_matmul", (P, P, 65, P, P, MOST - 255, 64, P, BF16, MOST, None)), ("rose_mx4_matmul", (P, P, MOST, P, P, MOST, 0, P, F32, MOST, None))]
    for call, (status, launches) in zip(calls, launched(recorder, calls)):
        assert status == OK and launches and fits(launches), (call, status, launches)


def test_products_of_more_tiles_than_a_launch_holds_queue_nothing(recorder):
    """No memory holds these; what is refused is refused before the activations are quantised."""
    calls = [("rose_mx4_linear", (P, F32, m, 64, P, P, n, 64, P, BF16, n, P, 1 << 50, None)) for m, n in ((MOST, MOST), (MOST, 65), (1 << 20, 1 << 20))]
    calls += [("rose_mx4_matmul", (P, P, m, P, P, n, 64, P, BF16, n, None)) for m, n in ((MOST, MOST), (65, MOST), (1 << 20, 1 << 20))]
    for call, (status, launches) in zip(calls, launched(recorder, calls)):
        assert status == UNSUPPORTED and not launches, (call, status, launches)


def test_activations_are_not_quantised_again_for_very_many_rows_of_weights(recorder):
    """Five to eight rows: by the product itself up to where that costs more than a launch, once for all beyond."""
    alone = [(8, 1024, 1024), (8, 32768, 1024), (8, 16384, 2048), (5, 32768, 33), (4, 151936, 2048), (1, 1 << 20, 8192)]
    before = [(8, 32769, 1024), (8, 32769, 33), (8, 16400, 2048), (5, 151936, 2048), (8, 1024, 2049), (9, 1024, 1024)]
    calls = [("rose_mx4_linear", (P, BF16, m, k, P, P, n, k, P, BF16, n, P, 1 << 40, None)) for m, n, k in alone + before]
    for (status, launches), size, want in zip(launched(recorder, calls), alone + before, [1] * len(alone) + [2] * len(before)):
        assert status == OK and len(launches) == want, (size, launches)


def test_no_tensors_need_no_table(recorder):
    """An empty table's address is null; the offsets still say that there is nothing."""
    W = binding.GRAD_WORKSPACE_BYTES
    calls = [("rose_grad_sum_squares", (None, P, 0, 0, F32, P, P, W, None)), ("rose_grad_clip", (None, P, 0, 0, F32, None, P, 1.0, P, None)),
             ("rose_grad_clip_norm", (None, P, 0, 0, BF16, None, 1.0, P, P, W, None))]
    assert all(status == OK and launches for status, launches in launched(recorder, calls))
