"""What the operators at the two ends of a synchronisation refuse, through the C ABI and on the host alone: the addresses
here are never read, since a refused call queues nothing."""
import ctypes

import pytest
import torch

import paper_2605_06534_amd as R
from paper_2605_06534_amd import binding

OK, ARG, SHAPE, ALIGN, UNSUPPORTED = (binding.OK, binding.ERR_ARG, binding.ERR_SHAPE, binding.ERR_ALIGN, binding.ERR_UNSUPPORTED)
P = 1 << 20                                         # an aligned address
BF16, F32 = binding.DTYPE_BF16, binding.DTYPE_F32
BIG = 1 << 31


def refused(name, good, changes):
    """Each change of one or more arguments of a call that would be fine makes the status it names."""
    f = getattr(binding._lib, name)
    for change, status in changes:
        args = dict(good, **change)
        assert f(*args.values()) == status, (name, change)


def test_lookup_refusals():
    good = dict(table=P, tt=BF16, rows=10, cols=8, ts=8, tokens=P, tb=8, n=4, first=0, scale=1.0, out=P, ot=BF16, os=8, stream=None)
    refused("rose_embedding_lookup", good, [
        (dict(table=None), ARG), (dict(tokens=None), ARG), (dict(out=None), ARG), (dict(tt=2), ARG), (dict(ot=-1), ARG),
        (dict(rows=-1), ARG), (dict(cols=-8), ARG), (dict(n=-1), ARG), (dict(ts=7), ARG), (dict(os=7), ARG), (dict(tb=2), ARG),
        (dict(first=-1), ARG), (dict(table=P + 1), ALIGN), (dict(tokens=P + 4), ALIGN), (dict(tb=4, tokens=P + 2), ALIGN),
        (dict(ot=F32, out=P + 2), ALIGN), (dict(tt=F32, table=P + 2), ALIGN), (dict(rows=BIG), UNSUPPORTED), (dict(n=BIG), UNSUPPORTED),
        (dict(cols=BIG, ts=BIG, os=BIG), UNSUPPORTED), (dict(n=0, tokens=None, out=None), OK)])


def test_embedding_grad_refusals():
    need = ctypes.c_size_t()
    size = binding._lib.rose_embedding_grad_workspace_bytes
    assert size(10, 8, 4, ctypes.byref(need)) == OK and need.value >= 32
    assert size(10, 8, 4, None) == ARG and size(-1, 8, 4, ctypes.byref(need)) == ARG and size(10, 8, -4, ctypes.byref(need)) == ARG
    assert size(BIG, 8, 4, ctypes.byref(need)) == UNSUPPORTED
    assert size(10, 8, 4, ctypes.byref(need)) == OK
    good = dict(dy=P, dt=BF16, ds=8, tokens=P, tb=8, n=4, first=0, scale=1.0, grad=P, gt=F32, rows=10, cols=8, gs=8, acc=0, ws=P,
                wsb=need.value, stream=None)
    refused("rose_embedding_grad", good, [
        (dict(dy=None), ARG), (dict(tokens=None), ARG), (dict(grad=None), ARG), (dict(ws=None), ARG), (dict(wsb=need.value - 1), ARG),
        (dict(ds=7), ARG), (dict(gs=7), ARG), (dict(dt=3), ARG), (dict(gt=3), ARG), (dict(tb=1), ARG), (dict(first=-2), ARG),
        (dict(n=-1), ARG), (dict(rows=-1), ARG), (dict(cols=-1), ARG), (dict(dy=P + 1), ALIGN), (dict(grad=P + 2), ALIGN),
        (dict(ws=P + 128), ALIGN), (dict(n=BIG), UNSUPPORTED), (dict(rows=BIG), UNSUPPORTED)])


def test_gradient_norm_refusals():
    W = binding.GRAD_WORKSPACE_BYTES
    table = dict(grads=P, offsets=P, n=3, total=100, dtype=F32)
    bad_table = [(dict(grads=None), ARG), (dict(offsets=None), ARG), (dict(n=-1), ARG), (dict(total=-1), ARG), (dict(dtype=5), ARG),
                 (dict(grads=P + 4), ALIGN), (dict(offsets=P + 4), ALIGN)]
    refused("rose_grad_sum_squares", dict(table, sum=P, ws=P, wsb=W, stream=None), bad_table + [
        (dict(sum=None), ARG), (dict(sum=P + 4), ALIGN), (dict(ws=None), ARG), (dict(wsb=W - 1), ARG), (dict(ws=P + 8), ALIGN)])
    refused("rose_grad_clip", dict(table, outs=P, sum=P, max_norm=1.0, norm=None, stream=None), bad_table + [
        (dict(outs=None), ARG), (dict(sum=None), ARG), (dict(max_norm=-1.0), ARG), (dict(max_norm=float("nan")), ARG),
        (dict(outs=P + 4), ALIGN), (dict(norm=P + 2), ALIGN)])
    refused("rose_grad_clip_norm", dict(table, outs=P, max_norm=1.0, norm=P, ws=P, wsb=W, stream=None), bad_table + [
        (dict(outs=None), ARG), (dict(max_norm=-0.5), ARG), (dict(ws=None), ARG), (dict(wsb=0), ARG), (dict(ws=P + 64), ALIGN),
        (dict(norm=P + 1), ALIGN)])


def test_mx4_refusals():
    refused("rose_mx4_quantize", dict(x=P, dtype=BF16, rows=4, cols=40, stride=40, codes=P, scales=P, stream=None), [
        (dict(x=None), ARG), (dict(codes=None), ARG), (dict(scales=None), ARG), (dict(dtype=2), ARG), (dict(rows=-1), ARG),
        (dict(stride=39), ARG), (dict(x=P + 1), ALIGN), (dict(codes=P + 8), ALIGN), (dict(rows=BIG), UNSUPPORTED),
        (dict(rows=0, x=None, codes=None, scales=None), OK)])
    refused("rose_mx4_dequantize", dict(codes=P, scales=P, rows=4, cols=40, out=P, dtype=F32, stride=40, stream=None), [
        (dict(codes=None), ARG), (dict(scales=None), ARG), (dict(out=None), ARG), (dict(dtype=9), ARG), (dict(cols=-1), ARG),
        (dict(stride=8), ARG), (dict(out=P + 2), ALIGN), (dict(codes=P + 4), ALIGN)])
    refused("rose_mx4_matmul", dict(ac=P, as_=P, m=4, wc=P, ws=P, n=8, k=64, out=P, ot=BF16, os=8, stream=None), [
        (dict(ac=None), ARG), (dict(as_=None), ARG), (dict(wc=None), ARG), (dict(ws=None), ARG), (dict(out=None), ARG), (dict(m=-1), ARG),
        (dict(n=-1), ARG), (dict(k=-1), ARG), (dict(os=7), ARG), (dict(ot=2), ARG), (dict(ac=P + 1), ALIGN), (dict(wc=P + 8), ALIGN),
        (dict(out=P + 1), ALIGN), (dict(k=BIG), UNSUPPORTED), (dict(m=0, ac=None, as_=None, out=None), OK)])
    need = ctypes.c_size_t()
    assert binding._lib.rose_mx4_linear_workspace_bytes(100, 8, 64, None) == ARG
    assert binding._lib.rose_mx4_linear_workspace_bytes(-1, 8, 64, ctypes.byref(need)) == ARG
    assert binding._lib.rose_mx4_linear_workspace_bytes(100, 8, 64, ctypes.byref(need)) == OK and need.value > 0
    refused("rose_mx4_linear", dict(x=P, xt=BF16, m=100, xs=64, wc=P, ws=P, n=8, k=64, out=P, ot=BF16, os=8, work=P, wb=need.value, stream=None), [
        (dict(x=None), ARG), (dict(wc=None), ARG), (dict(ws=None), ARG), (dict(out=None), ARG), (dict(xt=7), ARG), (dict(ot=7), ARG),
        (dict(xs=63), ARG), (dict(os=7), ARG), (dict(m=-1), ARG), (dict(work=None), ARG), (dict(wb=need.value - 1), ARG),
        (dict(x=P + 1), ALIGN), (dict(wc=P + 1), ALIGN), (dict(work=P + 16), ALIGN), (dict(n=BIG, os=BIG), UNSUPPORTED)])


def test_binding_refuses_what_the_library_cannot_see():
    """Shapes, devices and strides that only the tensors know."""
    cpu = torch.zeros(4, 8)
    with pytest.raises(R.RoseError) as e:
        R.embedding_lookup(cpu, torch.zeros(3, dtype=torch.int64), torch.zeros(3, 8))
    assert e.value.status == SHAPE
    with pytest.raises(R.RoseError) as e:
        R.Mx4(4, 40, torch.zeros(4, 16, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8))
    assert e.value.status == SHAPE
    with pytest.raises(R.RoseError) as e:
        R.grad_sum_squares(torch.zeros(3, dtype=torch.int64), torch.zeros(3, dtype=torch.int64), 5, torch.float32,
                           torch.zeros(1, dtype=torch.float64), torch.zeros(8))
    assert e.value.status == SHAPE
    assert R.offset_table([3, 0, 5], device="cpu").tolist() == [0, 3, 3, 8]


@pytest.mark.gpu
def test_binding_refuses_shapes_that_do_not_fit():
    print("case: shapes that do not fit", flush=True)
    t, ids = torch.zeros(4, 8, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    q = R.Mx4(4, 8)
    ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    for call in (lambda: R.embedding_lookup(t, ids, torch.zeros(2, 8, device="cuda")),
                 lambda: R.embedding_lookup(t, ids, torch.zeros(3, 7, device="cuda")),
                 lambda: R.embedding_lookup(t.t(), ids, torch.zeros(3, 4, device="cuda")),
                 lambda: R.embedding_lookup(t, ids.float(), torch.zeros(3, 8, device="cuda")),
                 lambda: R.embedding_lookup(t, ids.repeat(2)[::2], torch.zeros(3, 8, device="cuda")),
                 lambda: R.embedding_lookup(t.half(), ids, torch.zeros(3, 8, device="cuda")),
                 lambda: R.embedding_grad(torch.zeros(2, 8, device="cuda"), ids, t, ws),
                 lambda: R.embedding_grad(torch.zeros(3, 9, device="cuda"), ids, t, ws),
                 lambda: R.mx4_quantize(torch.zeros(4, 9, device="cuda"), q),
                 lambda: R.mx4_dequantize(q, torch.zeros(5, 8, device="cuda")),
                 lambda: R.mx4_matmul(R.Mx4(2, 8), q, torch.zeros(2, 5, device="cuda")),
                 lambda: R.mx4_matmul(R.Mx4(2, 40), q, torch.zeros(2, 4, device="cuda")),
                 lambda: R.mx4_linear(torch.zeros(2, 9, device="cuda"), q, torch.zeros(2, 4, device="cuda"), ws),
                 # a broadcast input: its rows lie on top of each other
                 lambda: R.embedding_grad(torch.zeros(1, 8, device="cuda").expand(3, 8), ids, t, ws)):
        with pytest.raises(R.RoseError) as e:
            call()
        assert e.value.status in (SHAPE, ARG)
