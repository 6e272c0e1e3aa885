"""A scale of zero gives every visible key the same weight; a query that is not finite still shows
(0 * NaN and 0 * inf are NaN)."""

import math

import pytest
import torch

from tests.chunk_util import Batch, attend, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kw", [dict(), dict(dtype=torch.float32), dict(fp8=True)], ids=["bf16", "f32", "fp8"])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_scale_zero(kw, value):
    for hint in (0, 1):
        for splits in (1, 3):
            bt = Batch([(40, 200), (1, 90)], seed=46, **kw)
            clean = attend(bt, scale=0.0, hint=hint, splits=splits)
            check(bt, clean, scale=0.0)
            bt.q[7, 3, 11] = value
            got = attend(bt, scale=0.0, hint=hint, splits=splits)
            assert torch.isnan(got[7, 3]).all()
            got[7, 3] = clean[7, 3]
            assert torch.equal(got, clean)
