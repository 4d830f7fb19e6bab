"""The check of many rows at once sees what it is for: outputs that are off, and outputs that are no numbers (no GPU needed)."""

import math

import pytest
import torch

from quant_check import check_finite_rows
from quant_util import gen, held_torch, rows


def batch():
    g = gen(3)
    k, v = held_torch(rows(40, 1, 64, g)), held_torch(rows(40, 1, 64, g))
    cut = lambda a: {name: x[:, 0][None] for name, x in a.items()}
    q, seen = torch.randn(3, 64, generator=g).bfloat16(), torch.tensor([40, 7, 0])
    value = lambda a: a["lo"][..., None] + a["step"][..., None] * a["codes"]
    logit = (q.double() @ value(cut(k))[0].T) * 64 ** -0.5
    logit = torch.where(torch.arange(40) < seen[:, None], logit, -math.inf)
    lse = torch.logsumexp(logit, -1)
    weights = torch.nan_to_num(torch.exp(logit - lse[:, None]))
    return (weights @ value(cut(v))[0]).bfloat16(), lse.float(), q, cut(k), cut(v), seen, 64 ** -0.5


def test_right_rows_pass():
    check_finite_rows(*batch())


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("row", [0, 1, 2])
def test_an_output_that_is_no_number_fails_though_its_lse_is_right(row, value):
    out, *rest = batch()
    out[row, 5] = value
    with pytest.raises(AssertionError):
        check_finite_rows(out, *rest)


@pytest.mark.parametrize("row", [0, 1, 2])
def test_an_output_or_an_lse_that_is_off_fails(row):
    out, lse, *rest = batch()
    wrong = out.clone()
    wrong[row, 9] += 0.5
    with pytest.raises(AssertionError):
        check_finite_rows(wrong, lse, *rest)
    for bad in (0.25, float("nan")):
        off = lse.clone()
        off[row] = off[row] + bad if math.isfinite(off[row]) else bad
        with pytest.raises(AssertionError):
            check_finite_rows(out, off, *rest)
