"""The check of many rows at once with what it cannot see by itself asked first: no output may be NaN or infinite."""

import torch

from quant_util import check_attend_torch


def check_finite_rows(out, lse, q, k, v, seen, scale):
    """``quant_util.check_attend_torch`` on rows whose outputs have to be numbers.  Its comparison, far = error > bound, is false for
    an error that is no number.  Errors and bounds are numbers where the inputs and outputs are: they are sums and products in 64
    bits of fp32 and bf16 numbers, of which none here is above 2^40."""
    for x in (q, *k.values(), *v.values()):
        assert torch.isfinite(x).all() and (x.abs() < 2.0 ** 40).all()
    assert torch.isfinite(out).all(), (~torch.isfinite(out)).any(-1).nonzero()[:5].tolist()
    assert torch.isfinite(lse[seen > 0]).all()
    check_attend_torch(out, lse, q, k, v, seen, scale)
