"""Padding and eps = 0 in mas_qk_norm_rope and its backward pass: a token past its
item's length has no norm, and counts in no weight's gradient."""
from __future__ import annotations

import pytest
import torch

from .test_model_qk import F16, F32, BF16, make, mas, run_and_check  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("D,R", [(7, 6), (64, 64), (64, 20), (100, 50), (130, 0)])
def test_eps_zero_with_padding(mas, dtype, D, R):
    """Heads of whole pieces and others, items that are all padding among them."""
    lens = torch.tensor([9, 4, 0, 1], dtype=torch.int32, device="cuda")
    st = make(4, 9, 3, 2, D, R, dtype, D + R)
    got = run_and_check(mas, st, R, "eps zero", t_x=lens, eps=0.0)
    assert all(bool(x.isfinite().all()) for x in got)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_eps_zero_with_padding_off_boundaries(mas, dtype):
    """64 channels that start off 16-byte boundaries go channel by channel too."""
    gen = torch.Generator().manual_seed(3)
    lens = torch.tensor([9, 4, 0, 1], dtype=torch.int32, device="cuda")
    wide = torch.randn((4, 9, 5, 67), generator=gen).to(dtype).cuda()
    st = dict(make(4, 9, 3, 2, 64, 64, dtype, 1), q=wide[:, :, :3, 1:65], k=wide[:, :, 3:, 1:65])
    got = run_and_check(mas, st, 64, "off boundaries", t_x=lens, eps=0.0)
    assert all(bool(x.isfinite().all()) for x in got)
