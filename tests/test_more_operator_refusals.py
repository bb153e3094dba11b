"""What the operators between hidden states and tokens refuse, what they launch, and what their workspaces need: through the C ABI and on the
host alone, since a refused call queues nothing and a stand-in notes the launches of the others."""
import ctypes
import os
import random
import re

import pytest
import torch

import paper_2605_06534_amd as R
from paper_2605_06534_amd import binding
from test_operator_launches import fits, launched, recorder  # noqa: F401  (recorder: a fixture)
from test_operator_refusals import refused

OK, ARG, SHAPE, ALIGN, UNSUPPORTED = (binding.OK, binding.ERR_ARG, binding.ERR_SHAPE, binding.ERR_ALIGN, binding.ERR_UNSUPPORTED)
P = 1 << 20                                         # an aligned address
BF16, F32 = binding.DTYPE_BF16, binding.DTYPE_F32
BIG, MOST = 1 << 31, (1 << 31) - 1
NAN = float("nan")


def need(name, *sizes):
    v = ctypes.c_size_t()
    assert getattr(binding._lib, name)(*sizes, ctypes.byref(v)) == OK
    return v.value


def test_norm_refusals():
    good = dict(x=P, xt=BF16, rows=4, cols=8, xs=8, w=P, b=P, wt=BF16, eps=1e-5, center=1, out=P, ot=F32, os=8, mean=P, rstd=P, stream=None)
    refused("rose_layer_norm", good, [
        (dict(x=None), ARG), (dict(w=None), ARG), (dict(out=None), ARG), (dict(xt=2), ARG), (dict(wt=2), ARG), (dict(ot=-1), ARG), (dict(rows=-1), ARG),
        (dict(cols=-8), ARG), (dict(cols=0), ARG), (dict(xs=7), ARG), (dict(os=7), ARG), (dict(eps=-1e-9), ARG), (dict(eps=NAN), ARG),
        (dict(center=0), ARG), (dict(x=P + 1), ALIGN), (dict(w=P + 1), ALIGN), (dict(b=P + 1), ALIGN), (dict(out=P + 2), ALIGN),
        (dict(mean=P + 2), ALIGN), (dict(rstd=P + 1), ALIGN), (dict(rows=BIG), UNSUPPORTED), (dict(cols=BIG, xs=BIG, os=BIG), UNSUPPORTED),
        (dict(rows=0, x=None, out=None), OK)])
    size = binding._lib.rose_layer_norm_grad_workspace_bytes
    v = ctypes.c_size_t()
    assert size(4, 8, None) == ARG and size(-1, 8, ctypes.byref(v)) == ARG and size(BIG, 8, ctypes.byref(v)) == UNSUPPORTED
    good = dict(dy=P, dt=BF16, ds=8, x=P, xt=F32, xs=8, rows=4, cols=8, w=P, wt=F32, mean=P, rstd=P, dx=P, gs=8, dw=P, db=P, acc=0, ws=P,
                wb=need("rose_layer_norm_grad_workspace_bytes", 4, 8), stream=None)
    refused("rose_layer_norm_grad", good, [
        (dict(dy=None), ARG), (dict(x=None), ARG), (dict(w=None), ARG), (dict(rstd=None), ARG), (dict(dx=None), ARG), (dict(ws=None), ARG),
        (dict(wb=good["wb"] - 1), ARG), (dict(dt=3), ARG), (dict(xt=3), ARG), (dict(wt=-1), ARG), (dict(cols=0), ARG), (dict(rows=-1), ARG),
        (dict(ds=7), ARG), (dict(xs=7), ARG), (dict(gs=7), ARG), (dict(dy=P + 1), ALIGN), (dict(dx=P + 2), ALIGN), (dict(dw=P + 2), ALIGN),
        (dict(db=P + 1), ALIGN), (dict(mean=P + 2), ALIGN), (dict(rstd=P + 2), ALIGN), (dict(ws=P + 16), ALIGN), (dict(rows=BIG), UNSUPPORTED)])


def test_distill_refusals():
    entries = dict(z=P, zt=BF16, rows=4, cols=50, zs=50, ids=P, ib=8, teacher=P, top=3, t=1.0)
    bad = [(dict(z=None), ARG), (dict(zt=2), ARG), (dict(rows=-1), ARG), (dict(cols=0), ARG), (dict(cols=-1), ARG), (dict(zs=49), ARG), (dict(ids=None), ARG),
           (dict(teacher=None), ARG), (dict(ib=2), ARG), (dict(top=-1), ARG), (dict(t=0.0), ARG), (dict(t=-1.0), ARG), (dict(t=NAN), ARG),
           (dict(t=float("inf")), ARG), (dict(z=P + 1), ALIGN), (dict(ids=P + 4), ALIGN), (dict(teacher=P + 2), ALIGN), (dict(rows=1 << 22), UNSUPPORTED),
           (dict(cols=BIG, zs=BIG), UNSUPPORTED), (dict(top=binding.DISTILL_MOST_TOP + 1), UNSUPPORTED)]
    work = dict(ws=P, wb=need("rose_distill_workspace_bytes", 4, 50), stream=None)
    bad_work = [(dict(ws=None), ARG), (dict(wb=work["wb"] - 1), ARG), (dict(ws=P + 8), ALIGN)]
    assert binding._lib.rose_distill_workspace_bytes(4, 50, None) == ARG
    refused("rose_distill_loss", dict(entries, loss=P, lse=P, **work), bad + bad_work + [
        (dict(loss=None), ARG), (dict(lse=None), ARG), (dict(loss=P + 1), ALIGN), (dict(lse=P + 2), ALIGN),
        (dict(rows=0, z=None, ids=None, teacher=None, loss=None, lse=None), OK)])
    refused("rose_distill_grad", dict(entries, lse=P, d_loss=P, d=P, ds=50, stream=None), bad + [
        (dict(lse=None), ARG), (dict(d_loss=None), ARG), (dict(d=None), ARG), (dict(ds=49), ARG), (dict(d=P + 1), ALIGN), (dict(d_loss=P + 2), ALIGN)])
    refused("rose_distill_loss_grad", dict(entries, d_loss=P, loss=P, lse=P, d=P, ds=50, **work), bad + bad_work + [
        (dict(d_loss=None), ARG), (dict(loss=None), ARG), (dict(lse=None), ARG), (dict(d=None), ARG), (dict(ds=49), ARG), (dict(d=P + 1), ALIGN)])


def test_verify_refusals():
    good = dict(p=P, ps=50, q=P, qs=50, dtype=F32, cols=50, drafted=P, tb=8, n=6, offsets=P, requests=2, u=P, tokens=P, accepted=P, ws=P,
                wb=need("rose_draft_verify_workspace_bytes", 2, 50), stream=None)
    assert binding._lib.rose_draft_verify_workspace_bytes(2, 50, None) == ARG
    refused("rose_draft_verify", good, [
        (dict(p=None), ARG), (dict(drafted=None), ARG), (dict(offsets=None), ARG), (dict(u=None), ARG), (dict(tokens=None), ARG), (dict(accepted=None), ARG),
        (dict(dtype=2), ARG), (dict(tb=2), ARG), (dict(n=-1), ARG), (dict(requests=-1), ARG), (dict(cols=0), ARG), (dict(ps=49), ARG), (dict(qs=49), ARG),
        (dict(ws=None), ARG), (dict(wb=good["wb"] - 1), ARG), (dict(p=P + 2), ALIGN), (dict(q=P + 2), ALIGN), (dict(drafted=P + 4), ALIGN),
        (dict(offsets=P + 4), ALIGN), (dict(u=P + 2), ALIGN), (dict(tokens=P + 4), ALIGN), (dict(accepted=P + 2), ALIGN), (dict(ws=P + 128), ALIGN),
        (dict(n=BIG), UNSUPPORTED), (dict(requests=1 << 18, wb=1 << 40), UNSUPPORTED), (dict(cols=BIG, ps=BIG, qs=BIG), UNSUPPORTED)])


def test_adapter_refusals():
    good = dict(x=P, m=5, k=40, xs=40, down=P, up=P, scales=P, adapters=3, rank=4, chosen=P, cb=4, out=P, ot=BF16, n=30, os=30, ws=P,
                wb=need("rose_adapter_linear_workspace_bytes", 5, 30, 40, 3, 4), stream=None)
    assert binding._lib.rose_adapter_linear_workspace_bytes(5, 30, 40, 3, 4, None) == ARG
    refused("rose_adapter_linear", good, [
        (dict(x=None), ARG), (dict(down=None), ARG), (dict(up=None), ARG), (dict(chosen=None), ARG), (dict(out=None), ARG), (dict(ot=2), ARG), (dict(cb=1), ARG),
        (dict(m=-1), ARG), (dict(n=-1), ARG), (dict(k=-1), ARG), (dict(adapters=-1), ARG), (dict(rank=-1), ARG), (dict(xs=39), ARG), (dict(os=29), ARG),
        (dict(ws=None), ARG), (dict(wb=good["wb"] - 1), ARG), (dict(x=P + 1), ALIGN), (dict(down=P + 1), ALIGN), (dict(up=P + 1), ALIGN),
        (dict(scales=P + 2), ALIGN), (dict(chosen=P + 2), ALIGN), (dict(out=P + 1), ALIGN), (dict(ws=P + 64), ALIGN), (dict(m=1 << 29), UNSUPPORTED),
        (dict(k=BIG, xs=BIG), UNSUPPORTED), (dict(n=BIG, os=BIG), UNSUPPORTED), (dict(adapters=binding.MOST_ADAPTERS + 1), UNSUPPORTED),
        (dict(rank=binding.MOST_RANK + 1), UNSUPPORTED), (dict(m=1 << 28, n=1 << 20, os=1 << 20), UNSUPPORTED),
        (dict(m=0, x=None, chosen=None, out=None), OK)])


def test_constants_are_the_header_s():
    header = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "rose_delta.h")
    value = dict(re.findall(r"#define\s+(ROSE_\w+)\s+(\d+)\b", open(header).read()))
    assert int(value["ROSE_DISTILL_MOST_TOP"]) == binding.DISTILL_MOST_TOP
    assert int(value["ROSE_MOST_ADAPTERS"]) == binding.MOST_ADAPTERS and int(value["ROSE_MOST_RANK"]) == binding.MOST_RANK


def test_workspaces_never_shrink():
    rng = random.Random(3)
    for _ in range(20000):
        for name, bits in (("rose_layer_norm_grad_workspace_bytes", (24, 20)), ("rose_distill_workspace_bytes", (21, 20)),
                           ("rose_draft_verify_workspace_bytes", (17, 24)), ("rose_adapter_linear_workspace_bytes", (20, 15, 15, 12, 10))):
            large = [int(2 ** rng.uniform(0, b)) for b in bits]
            small = [max(1, int(v * rng.uniform(0.3, 1))) if rng.random() < 0.7 else v for v in large]
            assert need(name, *small) <= need(name, *large), (name, small, large)


def test_launches_of_very_many(recorder):  # noqa: F811
    W = 1 << 62
    calls = [("rose_layer_norm", (P, xt, rows, cols, cols, P, None, F32, 1e-5, 1, P, ot, cols, P, P, None))
             for rows, cols in ((1, 1), (1, MOST), (MOST, 1), (MOST, 100), ((1 << 22) - 2, 60000), ((1 << 22) - 2, 5120), (70000, 64), (3, 16385))
             for xt, ot in ((BF16, BF16), (F32, BF16))]
    calls += [("rose_layer_norm_grad", (P, dt, cols, P, BF16, cols, rows, cols, P, BF16, P, P, P, cols, P, P, 0, P, W, None))
              for rows, cols in ((0, 5), (1, 1), (1, MOST), (MOST, 1), (MOST, 100), (MOST, MOST), (1 << 20, 5120), (70000, 64), (3, 16385)) for dt in (BF16, F32)]
    rows_cols = ((1, 1), (1, MOST), ((1 << 22) - 1, 1), ((1 << 22) - 1, 152064), ((1 << 22) - 1, MOST), (512, 152064), (513, 40000), (600, 20000))
    calls += [("rose_distill_loss", (P, dt, rows, cols, cols, P, 8, P, 5, 1.0, P, P, P, W, None)) for rows, cols in rows_cols for dt in (BF16, F32)]
    calls += [("rose_distill_loss_grad", (P, dt, rows, cols, cols, P, 8, P, top, 1.0, P, P, P, P, cols, P, W, None))
              for rows, cols in rows_cols for dt in (BF16, F32) for top in (5, 1024)]
    calls += [("rose_distill_grad", (P, dt, rows, cols, cols, P, 8, P, 5, 1.0, P, P, P, cols, None)) for rows, cols in rows_cols for dt in (BF16, F32)]
    calls += [("rose_draft_verify", (P, cols, P, cols, BF16, cols, P, 4, n, P, requests, P, P, P, P, W, None))
              for requests, cols in ((1, 1), (1, MOST), ((1 << 18) - 1, 1 << 20), ((1 << 18) - 1, MOST)) for n in (0, 1000)]
    calls += [("rose_adapter_linear", (P, m, k, k, P, P, None, adapters, rank, P, 4, P, dt, n, n, P, W, None))
              for m, n, k, adapters, rank in ((1, 1, 1, 1, 1), (1, MOST, MOST, 1, 1024), (512, MOST, 8, 65536, 1024), (513, 4096, 4096, 65536, 64), (1 << 20, 4096, 4096, 65536, 1024),
                                              ((1 << 21) - 1, 4096, 4096, 65536, 512), ((1 << 28), 128, 4096, 1, 32), (1 << 22, 4096, 4096, 100, 128), (300, 1 << 27, 1, 1, 1))
              for dt in (BF16, F32)]
    for call, (status, launches) in zip(calls, launched(recorder, calls)):
        assert status == OK and launches and fits(launches), (call, status, launches)


def test_binding_refuses_what_the_library_cannot_see():
    x, w, f = torch.zeros(4, 8), torch.zeros(8), torch.zeros(4)
    ids = torch.zeros(4, 3, dtype=torch.int64)
    for call in (lambda: R.layer_norm(x, w, x), lambda: R.layer_norm_grad(x, x, w, f, x, w, w), lambda: R.distill_loss(x, ids, torch.zeros(4, 3), f, f, f),
                 lambda: R.draft_verify(x, None, ids[0], ids[0], f, ids[0], f, f),
                 lambda: R.Adapters(torch.zeros(2, 3, 8), torch.zeros(2, 5, 3)),
                 lambda: R.Adapters(torch.zeros(2, 3, 8, dtype=torch.bfloat16), torch.zeros(2, 5, 4, dtype=torch.bfloat16)),
                 lambda: R.Adapters(torch.zeros(2, 3, 8, dtype=torch.bfloat16), torch.zeros(2, 5, 3, dtype=torch.bfloat16), torch.zeros(3))):
        with pytest.raises(R.RoseError) as e:
            call()
        assert e.value.status == SHAPE


@pytest.mark.gpu
def test_binding_refuses_shapes_that_do_not_fit():
    print("case: shapes that do not fit", flush=True)
    g = dict(device="cuda")
    x, w, f, ws = torch.zeros(4, 8, **g), torch.zeros(8, **g), torch.zeros(4, **g), torch.empty(1 << 20, dtype=torch.uint8, **g)
    ids, t = torch.zeros(4, 3, dtype=torch.int64, **g), torch.zeros(4, 3, **g)
    tokens, offsets, u, accepted = torch.zeros(3, dtype=torch.int64, **g), torch.tensor([0, 3], **g), torch.zeros(4, **g), torch.zeros(1, dtype=torch.int32, **g)
    out4 = torch.zeros(4, dtype=torch.int64, **g)
    a = R.Adapters(torch.zeros(2, 3, 8, dtype=torch.bfloat16, **g), torch.zeros(2, 5, 3, dtype=torch.bfloat16, **g))
    xb, o, chosen = x.bfloat16(), torch.zeros(4, 5, **g), torch.zeros(4, dtype=torch.int32, **g)
    for call in (lambda: R.layer_norm(x, w[:7], x), lambda: R.layer_norm(x, w, x[:3]), lambda: R.layer_norm(x, w, x, bias=w.bfloat16()),
                 lambda: R.layer_norm(x, w, x, bias=w, center=False), lambda: R.layer_norm(x, w, x, mean=f[:3]), lambda: R.layer_norm(x, w, x, rstd=f.double()),
                 lambda: R.layer_norm(x, w.half(), x), lambda: R.layer_norm(x.t(), w, x), lambda: R.layer_norm(x, w.cpu(), x),
                 lambda: R.layer_norm(x[:1].expand(4, 8), w, x),
                 lambda: R.layer_norm_grad(x, x, w, f, x.bfloat16(), w, ws), lambda: R.layer_norm_grad(x, x, w, f, x, w.bfloat16(), ws),
                 lambda: R.layer_norm_grad(x, x, w, f, x, w, ws[:64]), lambda: R.layer_norm_grad(x, x[:3], w, f, x, w, ws),
                 lambda: R.layer_norm_grad(x, x, w, f, x, w, ws.cpu()), lambda: R.layer_norm_grad(x, x, w, f, x, w, ws, dbias=f),
                 lambda: R.distill_loss(x, ids, t[:, :2], f, f, ws), lambda: R.distill_loss(x, ids.float(), t, f, f, ws), lambda: R.distill_loss(x, ids[:3], t[:3], f, f, ws),
                 lambda: R.distill_loss(x, ids, t.bfloat16(), f, f, ws), lambda: R.distill_loss(x, ids, t, f, f[:3], ws), lambda: R.distill_loss(x, ids, t, f, f, ws[:9]),
                 lambda: R.distill_loss(x, ids.t().contiguous().t(), t, f, f, ws), lambda: R.distill_grad(x, ids, t, f, f, x.bfloat16()),
                 lambda: R.distill_grad(x, ids, t, f, f, x[:, :7]), lambda: R.distill_loss_grad(x, ids, t, f, f, f, x[:3], ws), lambda: R.distill_loss(x, ids, t, f, f, ws, temperature=0.0),
                 lambda: R.draft_verify(x[:3], None, tokens, offsets, u, out4, accepted, ws), lambda: R.draft_verify(x, x, tokens, offsets, u, out4, accepted, ws),
                 lambda: R.draft_verify(x, xb[:3], tokens, offsets, u, out4, accepted, ws), lambda: R.draft_verify(x, None, tokens, offsets.int(), u, out4, accepted, ws),
                 lambda: R.draft_verify(x, None, tokens, offsets, u[:3], out4, accepted, ws), lambda: R.draft_verify(x, None, tokens, offsets, u, out4.int(), accepted, ws),
                 lambda: R.draft_verify(x, None, tokens, offsets, u, out4, accepted.long(), ws), lambda: R.draft_verify(x, None, tokens, offsets, u, out4, accepted, ws[:0]),
                 lambda: R.adapter_linear(x, a, chosen, o, ws), lambda: R.adapter_linear(xb[:, :7], a, chosen, o, ws), lambda: R.adapter_linear(xb, a, chosen[:3], o, ws),
                 lambda: R.adapter_linear(xb, a, chosen.float(), o, ws), lambda: R.adapter_linear(xb, a, chosen, o[:, :4], ws), lambda: R.adapter_linear(xb, a, chosen, o, ws[:8]),
                 lambda: R.adapter_linear(xb, a, chosen, o.half(), ws)):
        with pytest.raises(R.RoseError) as e:
            call()
        assert e.value.status in (SHAPE, ARG)
    R.adapter_linear(xb, a, chosen, o, ws)
    R.draft_verify(x, None, tokens, offsets, u, out4, accepted, ws)
    torch.cuda.synchronize()
