"""Layer norms of rows and their gradients against the formulas in 64 bits.

Bounds, with u = 2^-24 and sums of n terms formed as at most n / 64 + 24 additions one after the other (each loses u of what has been
summed so far): a mean is off by d u mean|x|, d = n / 64 + 25; a mean of squares of deviations by (d + 4) u of itself and twice the
mean's error times the mean deviation, its root's inverse by half of that and 3 u.  An output's own operations lose 4 u of each term, and
its rounding half of the type's eps.  Sums over rows are bounded as additions one after the other: rows * u * sum |dy xhat|."""
import pytest
import torch

import paper_2605_06534_amd as R

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TINY = 2.0 ** -134
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
TYPES = [("bf16", "bf16", "bf16"), ("f32", "f32", "f32"), ("bf16", "f32", "bf16"), ("f32", "bf16", "f32")]


def matrix(rows, cols, pad, dtype, seed, std=1.0, shift=0.0, offset=0):
    g = torch.Generator("cuda").manual_seed(seed)
    flat = (torch.randn(offset + rows * (cols + pad) + 8, generator=g, device="cuda") * std + shift).to(dtype)
    return flat[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]


def depth(n):
    return n / 64 + 25


def half(dtype):
    return torch.finfo(dtype).eps / 2


def forward(x, w, b, eps, center):
    """(out, mean, rstd), all in 64 bits, and bounds for what fp32 sums make of them"""
    x, n, d = x.double(), x.shape[1], depth(x.shape[1])
    mean = x.mean(1) if center else torch.zeros(len(x), dtype=torch.float64, device="cuda")
    e_mean = d * U * x.abs().mean(1) + U * mean.abs() if center else torch.zeros_like(mean)
    dev = x - mean[:, None]
    var = (dev * dev).mean(1)
    # sum (dev + e)^2 / n - var = 2 e mean(dev) + e^2, and mean(dev) is zero but for the rounding of dev
    e_dev = U * dev.abs() + e_mean[:, None]
    e_var = (d + 4) * U * var + e_mean ** 2 + 2 * U * (dev * dev).mean(1)
    rstd = (var + eps) ** -0.5
    e_rstd = rstd * (0.6 * e_var / (var + eps) + 4 * U)
    xhat = dev * rstd[:, None]
    w, b = w.double(), 0.0 if b is None else b.double()
    out = xhat * w + b
    e_out = (w.abs() * (e_dev * rstd[:, None] + dev.abs() * e_rstd[:, None] + 3 * U * xhat.abs()) + 3 * U * (out.abs() + (xhat * w).abs()))
    return (out, mean, rstd), (e_out, e_mean, e_rstd)


def check_forward(rows, cols, types, center, bias, pad=0, offset=0, seed=1, shift=0.3, out_pad=0, eps=1e-5):
    print("case: norm", rows, cols, types, center, bias, pad, offset, flush=True)
    xt, yt, wt = (DTYPES[t] for t in types)
    x = matrix(rows, cols, pad, xt, seed, 1.5, shift, offset)
    w, b = matrix(1, cols, 0, wt, seed + 1, 0.2, 1.0)[0], matrix(1, cols, 0, wt, seed + 2)[0] if bias else None
    whole = torch.full((rows, cols + out_pad), 7.0, dtype=yt, device="cuda")
    out, mean, rstd = whole[:, :cols], torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    R.layer_norm(x, w, out, bias=b, mean=mean, rstd=rstd, eps=eps, center=center)
    want, bound = forward(x, w, b, eps, center)
    assert (whole[:, cols:] == 7).all()
    off = (out.double() - want[0]).abs()
    assert (off <= bound[0] * (1 + half(yt)) + half(yt) * want[0].abs() + TINY).all(), (off - bound[0]).max()
    assert ((mean.double() - want[1]).abs() <= bound[1] + U * want[1].abs() + TINY).all()
    assert ((rstd.double() - want[2]).abs() <= bound[2] + U * want[2]).all()
    return x, w, b, out, mean, rstd


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("cols", [1, 2, 3, 4, 7, 8, 9, 15, 48, 63, 64, 65, 128, 130, 255, 513, 1000, 1024, 1030, 2047, 2056, 4096, 4099, 5120, 8191, 8200])
def test_forward(cols, types):
    for rows, center, bias, pad, offset in ((1, True, True, 0, 0), (5, False, False, 3, 1), (70, True, False, 8, 0)):
        check_forward(rows, cols, types, center, bias, pad, offset, out_pad=pad)


@pytest.mark.parametrize("rows,cols", [(3000, 640), (5000, 1025), (9001, 130), (4100, 2056), (4099, 5120), (8200, 4099), (20000, 48), (300, 16400), (7, 70001)])
def test_forward_of_many(rows, cols):
    for types, center in ((TYPES[0], True), (TYPES[1], False), (TYPES[2], False)):
        check_forward(rows, cols, types, center, center, seed=7, out_pad=1)


def test_rows_that_are_constant_or_far_from_zero():
    """No deviation at all: rstd is that of eps alone, and the output the bias."""
    print("case: constant rows", flush=True)
    x = torch.tensor([[0.0], [3.0], [-1e30], [2.0 ** -130]], device="cuda").expand(4, 640).contiguous()
    w, b, out = torch.ones(640, device="cuda"), torch.full((640,), 0.25, device="cuda"), torch.empty(4, 640, device="cuda")
    mean, rstd = torch.empty(4, device="cuda"), torch.empty(4, device="cuda")
    R.layer_norm(x[:2], w, out[:2], bias=b, mean=mean[:2], rstd=rstd[:2], eps=0.25)
    assert (out[:2] == 0.25).all() and (rstd[:2] == 2).all() and mean[:2].tolist() == [0.0, 3.0]
    # 640 = 5 * 128 equal values: partial sums are exact or off by u each, the deviation a few u of the value
    check_forward(9, 640, TYPES[1], True, True, shift=1000.0)
    check_forward(9, 5120, TYPES[1], True, True, shift=-300.0)
    R.layer_norm(x[3:], w, out[3:], center=False, eps=0.0, rstd=rstd[3:])          # squares that underflow: infinite, and 0 times that is no number
    assert rstd[3].isinf()


def test_numbers_that_are_none_stay_in_their_rows():
    print("case: NaN", flush=True)
    x = matrix(6, 1000, 0, torch.float32, 3)
    x[1, 17], x[3, 999], x[4, 0] = float("nan"), float("inf"), float("-inf")
    w, out, rstd = torch.ones(1000, device="cuda"), torch.empty(6, 1000, device="cuda"), torch.empty(6, device="cuda")
    R.layer_norm(x, w, out, rstd=rstd)
    assert out[[1, 3, 4]].isnan().any(1).all() and out[[0, 2, 5]].isfinite().all()
    R.layer_norm(x, w, out, rstd=rstd, center=False)
    assert out[1].isnan().all() and rstd[[3, 4]].eq(0).all() and out[[0, 2, 5]].isfinite().all()


@pytest.mark.parametrize("cols", [5, 640, 5120, 8193, 70000])
def test_in_place(cols):
    print("case: in place", cols, flush=True)
    for dtype in DTYPES.values():
        x, w = matrix(300, cols, 3, dtype, 4), matrix(1, cols, 0, dtype, 5)[0]
        out = torch.empty_like(x)
        R.layer_norm(x, w, out)
        R.layer_norm(x, w, x)
        assert torch.equal(x, out)


def backward(dy, x, w, mean, rstd):
    dy, x, w, rstd = dy.double(), x.double(), w.double(), rstd.double()[:, None]
    dev = x - mean.double()[:, None] if mean is not None else x
    xhat, g, n, d = dev * rstd, dy * w, x.shape[1], depth(x.shape[1])
    c1 = g.mean(1, keepdim=True) if mean is not None else torch.zeros_like(rstd)
    c2 = (g * xhat).mean(1, keepdim=True)
    dx = rstd * (g - c1 - xhat * c2)
    e_xhat = 2 * U * xhat.abs()
    e_c1 = (d + 2) * U * g.abs().mean(1, keepdim=True)
    e_c2 = (d + 5) * U * (g * xhat).abs().mean(1, keepdim=True)
    e_dx = rstd * (4 * U * (g.abs() + c1.abs() + (xhat * c2).abs()) + e_c1 + xhat.abs() * e_c2 + e_xhat * c2.abs())
    size_w, size_b = (dy * xhat).abs().sum(0), dy.abs().sum(0)
    return (dx, (dy * xhat).sum(0), dy.sum(0)), (e_dx, (len(x) + 4) * U * size_w, (len(x) + 2) * U * size_b)


def check_backward(rows, cols, types, center, pad=0, offset=0, accumulate=False, seed=11, dx_pad=0):
    print("case: gradient of a norm", rows, cols, types, center, pad, offset, accumulate, flush=True)
    xt, yt, wt = (DTYPES[t] for t in types)
    x, dy = matrix(rows, cols, pad, xt, seed, 1.5, 0.3, offset), matrix(rows, cols, pad, yt, seed + 1, 0.1, 0.02, offset)
    w = matrix(1, cols, 0, wt, seed + 2, 0.2, 1.0)[0]
    _, mean, rstd = (v.float() for v in forward(x, w, None, 1e-5, center)[0])
    mean = mean if center else None
    whole = torch.full((rows, cols + dx_pad), 7.0, dtype=xt, device="cuda")
    dx, dw, db = whole[:, :cols], matrix(1, cols, 0, torch.float32, seed + 3)[0].clone(), matrix(1, cols, 0, torch.float32, seed + 4)[0].clone()
    old_w, old_b = dw.double() * accumulate, db.double() * accumulate
    ws = R.layer_norm_grad_workspace(rows, cols)
    ws.fill_(0xFF)
    R.layer_norm_grad(dy, x, w, rstd, dx, dw, ws, mean=mean, dbias=db, accumulate=accumulate)
    want, bound = backward(dy, x, w, mean, rstd)
    assert (whole[:, cols:] == 7).all()
    assert ((dx.double() - want[0]).abs() <= bound[0] * (1 + half(xt)) + half(xt) * want[0].abs() + TINY).all()
    assert ((dw.double() - want[1] - old_w).abs() <= bound[1] + 2 * U * (old_w + want[1]).abs() + TINY).all()
    assert ((db.double() - want[2] - old_b).abs() <= bound[2] + 2 * U * (old_b + want[2]).abs() + TINY).all()


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("cols", [1, 3, 4, 7, 8, 9, 48, 64, 65, 130, 255, 513, 1000, 1030, 2047, 2056, 4096, 4099, 5120, 8191, 8200])
def test_backward(cols, types):
    for rows, center, pad, offset, accumulate in ((1, True, 0, 0, False), (5, False, 3, 1, True), (70, True, 8, 0, False)):
        check_backward(rows, cols, types, center, pad, offset, accumulate, dx_pad=pad)


@pytest.mark.parametrize("rows,cols", [(3000, 640), (5000, 1025), (9001, 130), (4100, 2056), (2099, 5120), (2200, 4099), (20000, 48), (300, 16400), (7, 70001)])
def test_backward_of_many(rows, cols):
    for types, center in ((TYPES[0], True), (TYPES[1], False), (TYPES[3], True)):
        check_backward(rows, cols, types, center, seed=13, dx_pad=1)


@pytest.mark.parametrize("rows,cols", [(1, 8), (257, 72), (4096, 640), (70000, 40), (5000, 2048), (2500, 5125)])
def test_sums_over_rows_that_are_exact(rows, cols):
    """Whole numbers: a row that is lost or counted twice shows."""
    print("case: exact sums", rows, cols, flush=True)
    g = torch.Generator("cuda").manual_seed(5)
    x = torch.randint(-8, 9, (rows, cols), generator=g, device="cuda").to(torch.bfloat16)
    dy = torch.randint(-8, 9, (rows, cols), generator=g, device="cuda").to(torch.bfloat16)
    rstd, mean = torch.full((rows,), 0.5, device="cuda"), torch.randint(-2, 3, (rows,), generator=g, device="cuda").float()
    w, dx, ws = torch.ones(cols, device="cuda"), torch.empty_like(x), R.layer_norm_grad_workspace(rows, cols)
    dw, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    R.layer_norm_grad(dy, x, w, rstd, dx, dw, ws, mean=mean, dbias=db)
    assert torch.equal(dw.double(), (dy.double() * (x.double() - mean[:, None]) * 0.5).sum(0)) and torch.equal(db.double(), dy.double().sum(0))


def test_what_is_not_wanted_is_left_out():
    print("case: without gradients of the parameters", flush=True)
    x, dy, w = matrix(40, 640, 0, torch.float32, 21), matrix(40, 640, 0, torch.float32, 22), matrix(1, 640, 0, torch.float32, 23)[0]
    rstd, ws = torch.rand(40, device="cuda") + 0.5, R.layer_norm_grad_workspace(40, 640)
    dx, dw, db = (torch.empty(s, device="cuda") for s in ((40, 640), 640, 640))
    R.layer_norm_grad(dy, x, w, rstd, dx, dw, ws, dbias=db)
    other, only = torch.empty_like(dx), torch.empty_like(dw)
    R.layer_norm_grad(dy, x, w, rstd, other, None, ws)
    assert torch.equal(other, dx)
    R.layer_norm_grad(dy, x, w, rstd, other, only, ws)
    assert torch.equal(other, dx) and torch.equal(only, dw)
    R.layer_norm_grad(dy[:0], x[:0], w, rstd[:0], dx[:0], dw, ws, accumulate=True)          # no rows: left alone, or zeros
    assert torch.equal(only, dw)
    R.layer_norm_grad(dy[:0], x[:0], w, rstd[:0], dx[:0], dw, ws, dbias=db)
    assert (dw == 0).all() and (db == 0).all()
    R.layer_norm(x[:0], w, dx[:0])


@pytest.mark.parametrize("cols", [5, 640, 5120, 8193, 70000])
def test_gradient_in_place(cols):
    print("case: gradient in place", cols, flush=True)
    for dtype in DTYPES.values():
        x, dy, w = matrix(150, cols, 3, dtype, 24), matrix(150, cols, 3, dtype, 25), matrix(1, cols, 0, dtype, 26)[0]
        rstd, ws, dw, other = torch.rand(150, device="cuda") + 0.5, R.layer_norm_grad_workspace(150, cols), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
        dx = torch.empty_like(x)
        R.layer_norm_grad(dy, x, w, rstd, dx, dw, ws, mean=rstd)
        for target in (0, 1):
            a, b = x.clone(memory_format=torch.preserve_format), dy.clone(memory_format=torch.preserve_format)
            into = (a, b)[target]
            R.layer_norm_grad(b, a, w, rstd, into, other, ws, mean=rstd)
            assert torch.equal(into, dx) and torch.equal(other, dw)


def test_gradients_against_differences():
    """The gradient of sum(c * norm(x)) by central differences of the definition in 64 bits: their own error is h^2 times a third derivative
    and eps64 / h, both far below the bound for fp32."""
    print("case: differences", flush=True)
    rows, cols, h = 3, 37, 1e-4
    x, c, w, b = (matrix(r, cols, 0, torch.float32, 31 + i) for i, r in enumerate((rows, rows, 1, 1)))
    for center in (True, False):
        (_, mean, rstd), _ = forward(x, w[0], None, 1e-5, center)

        def loss(x, w, b):
            d = x - x.mean(1, keepdim=True) if center else x
            return (c.double() * (d * ((d * d).mean(1, keepdim=True) + 1e-5) ** -0.5 * w + b)).sum().item()

        dx, dw, db, ws = torch.empty_like(x), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda"), R.layer_norm_grad_workspace(rows, cols)
        R.layer_norm_grad(c, x, w[0], rstd.float(), dx, dw, ws, mean=mean.float() if center else None, dbias=db)
        args = [x.double(), w.double(), b.double()]
        for k, got in enumerate((dx, dw[None], db[None])):
            for i in range(got.shape[0]):
                for j in range(0, cols, 5):
                    ends = []
                    for s in (h, -h):
                        moved = [a.clone() for a in args]
                        moved[k][i, j] += s
                        ends.append(loss(*moved))
                    # rstd <= 1 / 0.3 of 37 normal values, so third derivatives are below 1e3 * |c|: 1e-5; fp32: 2^-24 * 100 terms
                    assert abs((ends[0] - ends[1]) / (2 * h) - got[i, j].item()) < 1e-5 * 3 + 2.0 ** -24 * 200


def test_the_same_bits_twice_and_in_a_graph():
    print("case: graph", flush=True)
    rows, cols = 1500, 1000
    x, dy, w = matrix(rows, cols, 0, torch.bfloat16, 41), matrix(rows, cols, 0, torch.bfloat16, 42), matrix(1, cols, 0, torch.bfloat16, 43)[0]
    y, mean, rstd, dx = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(x)
    dw, db, ws = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda"), R.layer_norm_grad_workspace(rows, cols)

    def step():
        R.layer_norm(x, w, y, mean=mean, rstd=rstd)
        R.layer_norm_grad(dy, x, w, rstd, dx, dw, ws, mean=mean, dbias=db)

    step()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for seed in range(3):
        x.copy_(matrix(rows, cols, 0, torch.bfloat16, 50 + seed))
        step()
        want = [t.clone() for t in (y, mean, rstd, dx, dw, db)]
        for t in (y, mean, rstd, dx, dw, db):
            t.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (y, mean, rstd, dx, dw, db)))
