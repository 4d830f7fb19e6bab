"""The batches of many kinds once more, with outputs that have to be numbers: unused bytes of the pools are NaN rows, so a row of V
that is not there and counts all the same shows as NaN in an output whose lse is right."""

import pytest

import test_gpu_quant_attend as many
from quant_check import check_finite_rows

pytestmark = pytest.mark.gpu

BATCHES = many.test_batches_of_many_kinds_against_torch_in_64_bits
CASES = next(m for m in BATCHES.pytestmark if m.name == "parametrize").args[1]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_outputs_of_batches_of_many_kinds_are_numbers(case, monkeypatch):
    calls = []
    monkeypatch.setattr(many, "check_attend_torch", lambda *a: (calls.append(1), check_finite_rows(*a)))
    BATCHES(*case)
    assert calls


@pytest.mark.parametrize("case", [
    (2, 1, 1000, 64, 16, 10, 200, 1), (3, 1, 1024, 128, 32, 1, 300, 3), (2, 1, 333, 128, 64, 100, 900, 16), (2, 1024, 1, 64, 16, 1, 150, 2), (1, 512, 2, 128, 64, 40, 70, 1),
    (2, 31, 33, 64, 32, 60, 400, 1),
], ids=str)
def test_groups_and_heads_up_to_the_most(case, monkeypatch):
    monkeypatch.setattr(many, "check_attend_torch", check_finite_rows)
    BATCHES(*case)
