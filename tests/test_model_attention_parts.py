"""Forward passes whose keys are split over workgroups and joined, with one block of rows
and with several, against 64 bits: parts that a row does not see, lengths that end inside
a part, and values that are no numbers in some parts."""
from __future__ import annotations

import pytest
import torch

from ._attention import check, reference
from .test_model_attention import BF16, F16, F32, _ints, make, mas, run_and_check  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("Tq,Tk,Hq,Hk,D", [(100, 2000, 2, 1, 64), (45, 1500, 3, 1, 128), (40, 1100, 4, 2, 40), (33, 3000, 1, 1, 96), (1, 5000, 3, 1, 128)])
def test_rows_over_split_keys(mas, dtype, Tq, Tk, Hq, Hk, D):
    q, k, v, _ = make(3, Tq, Tk, Hq, Hk, D, dtype, Tk)
    t_q, t_k = _ints([Tq, Tq, max(Tq // 2, 1)]), _ints([Tk, 700, 517])
    run_and_check(mas, q, k, v, None, "causal", t_q=t_q, t_k=t_k, causal=True, slope=torch.full((Hq,), 0.05, device="cuda"))
    run_and_check(mas, q, k, v, None, "all", t_q=t_q, t_k=t_k, cap=15.0)
    docs = _ints([[0, 10, Tk - 60, Tk], [0, 300, 600, 700], [0, 0, 0, 517]])
    run_and_check(mas, q, k, v, None, "documents", t_q=t_q, t_k=t_k, causal=True, doc_start=docs, prefix=_ints([[3, 70, 2], [9, 300, 0], [0, 0, 512]]))


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("Tq", [1, 60])
def test_values_that_are_no_numbers_in_a_part(mas, dtype, Tq):
    Tk, D, at = 2500, 64, 2470
    q, k, v, _ = make(2, Tq, Tk, 2, 1, D, dtype, 7)
    print(f"[gpu-case] parts, no numbers Tq={Tq} {dtype}", flush=True)
    want = reference(q, k, v, causal=True)["out"]
    for bad in (float("nan"), float("inf"), -float("inf")):
        # Past every row's place, and in the last part where rows from `at` on see it.
        k2, v2 = k.clone(), v.clone()
        v2[:, at, :, 5] = bad
        out = mas.mas_attention(q, k2, v2, causal=True)
        sees = torch.arange(Tq) + Tk - Tq >= at
        hit = out[:, sees.cuda(), :, 5]
        assert bool(hit.isnan().all()) if bad != bad else bool((hit == bad).all())
        value = want[0].clone()
        out[:, sees.cuda(), :, 5] = 0
        value[:, sees, :, 5] = 0
        check(out, (value, want[1]), f"around {bad}")
        k2[:, 2000:], v2[:, 2000:] = bad, bad
        out = mas.mas_attention(q, k2, v2, causal=True, t_k=_ints([2000, 2000]), t_q=_ints([Tq, Tq]))
        check(out, reference(q, k, v, causal=True, t_k=_ints([2000, 2000]), t_q=_ints([Tq, Tq]))["out"], f"padding {bad}")
