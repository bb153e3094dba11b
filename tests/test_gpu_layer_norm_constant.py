"""Centred norms of rows without deviation, whatever their size and length: the mean is the value, rstd that of eps alone, the output the bias.

A plain fp32 sum of n equal values gives a mean that is off by a few units, and with it deviations that are not there: their squares overflow at
1e30 and are of eps's size at 1e4.  Exact here, since a mean m = v (1 + e), |e| <= d u (u = 2^-24, d = n / 64 + 25), leaves deviations v - m that
are exact and all equal; their mean is right but for d u of itself, so that what has to be added to m is off by v (d u)^2, less than half a unit
of v for n below 180,000."""
import pytest
import torch

import paper_2605_06534_amd as R

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
VALUES = [-1e30, 3.3e33, 12345.678, -10000.1, 1.0 / 3, 1e-30, 255.9]
COLS = [1, 3, 7, 9, 48, 65, 130, 255, 333, 641, 1000, 1030, 2047, 3001, 4099, 5121, 8191, 16400, 33333, 70001]


@pytest.mark.gpu
@pytest.mark.parametrize("y", DTYPES)
@pytest.mark.parametrize("x", DTYPES)
@pytest.mark.parametrize("cols", COLS)
def test_rows_of_one_value(cols, x, y):
    print("case: rows of one value", cols, x, y, flush=True)
    values = torch.tensor(VALUES, device="cuda").to(DTYPES[x])
    rows = values[:, None].expand(len(VALUES), cols).contiguous()
    w, b = torch.full((cols,), 3.0, device="cuda"), torch.full((cols,), 0.25, device="cuda")
    out, mean, rstd = torch.empty(rows.shape, dtype=DTYPES[y], device="cuda"), torch.empty(len(VALUES), device="cuda"), torch.empty(len(VALUES), device="cuda")
    R.layer_norm(rows, w, out, bias=b, mean=mean, rstd=rstd, eps=0.25)
    assert torch.equal(mean, values.float())
    assert (rstd == 2).all() and (out == 0.25).all()


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [333, 5121, 70001])
def test_infinities_and_what_is_no_number_keep_their_mean(cols):
    print("case: infinite means", cols, flush=True)
    x = torch.ones(4, cols, device="cuda")
    x[0, cols // 2], x[1, 0], x[2, cols - 1] = float("inf"), float("-inf"), float("nan")
    w, out, mean, rstd = torch.ones(cols, device="cuda"), torch.empty_like(x), torch.empty(4, device="cuda"), torch.empty(4, device="cuda")
    R.layer_norm(x, w, out, mean=mean, rstd=rstd, eps=0.25)
    assert mean[0] == float("inf") and mean[1] == float("-inf") and mean[2].isnan() and mean[3] == 1
    assert rstd[:3].isnan().all() and out[:3].isnan().all() and rstd[3] == 2 and (out[3] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [333, 5121, 16400, 70001])
def test_rows_whose_values_are_few_units_apart(cols):
    """Values v + k unit, k of 0 to 8, v = 2^20 (units of 2^-3): the mean is off by its rounding, half a unit of v, the squares about it too large by
    the square of that (and never too small), an output's deviation off by as much as the mean.  (What is left of fp32 sums of deviations
    below 9 units: 300 additions of 2^-24, a part in 10^4.)"""
    print("case: few units apart", cols, flush=True)
    k = torch.randint(0, 9, (6, cols), generator=torch.Generator("cuda").manual_seed(3), device="cuda")
    x = (2.0 ** 20 + k.double() / 8).float()
    w, out, mean, rstd = torch.ones(cols, device="cuda"), torch.empty_like(x), torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
    R.layer_norm(x, w, out, mean=mean, rstd=rstd, eps=0.0)
    d = x.double() - x.double().mean(1, keepdim=True)
    var = (d * d).mean(1)
    half, more = 2.0 ** -4, 9 / 8 * 1e-4
    assert ((mean.double() - x.double().mean(1)).abs() <= half + more).all()
    assert ((rstd.double() >= (var + (half + more) ** 2) ** -0.5 * (1 - 1e-4)) & (rstd.double() <= var ** -0.5 * (1 + 1e-4))).all()
    assert ((out.double() / rstd.double()[:, None] - d).abs() <= half + more).all()
