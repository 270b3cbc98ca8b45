"""Caps far above the scores, in every type: capped attention is then nearly the
uncapped one, and its error may not grow with the cap; and caps next to nothing."""
from __future__ import annotations

import pytest
import torch

from ._attention import check, reference
from .test_model_attention import BF16, F16, F32, _ints, make, mas  # noqa: F401

pytestmark = pytest.mark.gpu

CAPS = [257.0, 1e4, 1e5, 1e6, 1e7, 1e12, 3e38]


def compare(mas, q, k, v, g, label, **args):
    """Values of the capped problem in 64 bits; bounds of the uncapped one, which know of
    no cap, twice: a capped score is no larger than its uncapped one and tanh' at most 1,
    tanh from its series or as 1 + 2 r for |x| >= 1/4 errs by 2^-20 of itself at most, as
    much as the bounds allow for a score, and p differs from the uncapped p by less than
    a hundredth here (scores up to 6: 6^3 / (3 cap^2) < 0.002)."""
    print(f"[gpu-case] {label} q{tuple(q.shape)} k{tuple(k.shape)} {q.dtype} cap={args['cap']}", flush=True)
    want = reference(q, k, v, g, **args)
    loose = reference(q, k, v, g, **dict(args, cap=0.0))
    bound = lambda n: (want[n][0], 2 * loose[n][1])
    lse = torch.full((q.shape[0], q.shape[2], q.shape[1]), 7.0, device="cuda")
    out = mas.mas_attention(q, k, v, lse_out=lse, **args)
    check(out, bound("out"), label + " out")
    check(lse, bound("lse"), label + " lse")
    if g is not None:
        for n, x in zip(("dq", "dk", "dv"), mas.mas_attention_backward(g, q, k, v, out, lse, **args)):
            check(x, bound(n), f"{label} {n}")


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("cap", CAPS)
def test_large_caps(mas, dtype, cap):
    lens = _ints([100, 0, 1])
    compare(mas, *make(3, 100, 100, 4, 2, 64, dtype, 1), "few rows", t_q=lens, t_k=lens, causal=True, cap=cap)
    slope = torch.tensor([0.5, 0.25, 0.1], device="cuda")
    compare(mas, *make(2, 40, 40, 3, 1, 72, dtype, 2), "distances", slope=slope, cap=cap)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("cap", [300.0, 1e6])
def test_large_caps_of_steps_and_of_many_rows(mas, dtype, cap):
    """Keys split and joined, and batches whose ordinary caps go to shared tiles."""
    q, k, v, _ = make(2, 1, 2100, 8, 2, 64, dtype, 3)
    compare(mas, q, k, v, None, "step", t_k=_ints([2100, 700]), causal=True, cap=cap)
    q, k, v, g = make(140, 130, 130, 2, 2, 40, dtype, 4)
    compare(mas, q, k, v, g, "many rows", causal=True, cap=cap)
    ws = torch.empty(mas.mas_attention_workspace_bytes(q, k, backward=True), dtype=torch.uint8, device="cuda")
    lse = torch.empty((140, 2, 130), device="cuda")
    out = mas.mas_attention(q, k, v, causal=True, cap=cap, lse_out=lse, workspace=ws)
    assert torch.equal(out, mas.mas_attention(q, k, v, causal=True, cap=cap))


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_infinities_and_large_caps(mas, dtype):
    """Values that later queries alone see leave earlier ones as they are."""
    q, k, v, _ = make(1, 90, 90, 2, 2, 64, dtype, 5)
    want = mas.mas_attention(q, k, v, causal=True, cap=1e6)
    v2 = v.clone()
    v2[:, 70:] = float("inf")
    got = mas.mas_attention(q, k, v2, causal=True, cap=1e6)
    # The second pass over such rows takes its keys in another order: fp32 sums, and one
    # rounding of p and of the result each.
    ref = reference(q, k, v, causal=True, cap=1e6), reference(q, k, v, causal=True)
    check(got[:, :70], (ref[0]["out"][0][:, :70], 2 * ref[1]["out"][1][:, :70]), "before infinity")
    assert bool(want.isfinite().all()) and bool((got[:, 70:] == float("inf")).all())


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("cap", [1e-40, 1e-38, 1e-30, 1e-3])
def test_small_caps(mas, dtype, cap):
    """Scores next to equal: means of the values seen."""
    q, k, v, g = make(2, 50, 50, 2, 1, 32, dtype, 6)
    want = reference(q, k, v, g, causal=True, cap=cap)
    lse = torch.empty((2, 2, 50), device="cuda")
    out = mas.mas_attention(q, k, v, causal=True, cap=cap, lse_out=lse)
    check(out, want["out"], "out")
    check(lse, want["lse"], "lse")
    grads = mas.mas_attention_backward(g, q, k, v, out, lse, causal=True, cap=cap)
    check(grads[2], want["dv"], "dv")
    assert all(bool(x.isfinite().all()) for x in grads)
