"""Non-finite queries, keys and values in calls that split the keys: what a row sees shows in it,
whatever the number of splits and whichever kernel joins them."""

import math

import pytest
import torch

from paper_2605_01910_amd import santa as S
from tests.chunk_util import SCALE, Batch, attend

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
NAN = float("nan")
TYPES = {"bf16": dict(), "f32": dict(dtype=F32), "fp8": dict(fp8=True)}
# hint 0: 128-row tiles; 1: 32-row tiles, joined by the last split (groups of up to four); 2: by a launch
HINTS = (0, 1, 2)


def set_row(bt, cache, b, pos, value):
    at = torch.tensor([pos], device=bt.q.device)
    row = bt.rows(cache, b, at)
    bt.put(cache, b, at, torch.full_like(row, 0x7f if bt.fp8 else value))


@pytest.mark.parametrize("splits", [0, 1, 3, 64, 200])
@pytest.mark.parametrize("kind", sorted(TYPES))
def test_a_nan_query_stays_in_its_row(kind, splits):
    for lens, at in (([(40, 2900), (2, 700)], (7, 3)), ([(1, 3000)], (0, 3))):
        for hint in HINTS:
            bt = Batch(lens, seed=43, **TYPES[kind])
            clean = attend(bt, hint=hint, splits=splits)
            bt.q[at[0], at[1], 11] = NAN
            got = attend(bt, hint=hint, splits=splits)
            assert torch.isnan(got[at]).all()
            got[at] = clean[at]
            assert torch.equal(got, clean)


@pytest.mark.parametrize("L", [65, 129])
@pytest.mark.parametrize("kind", sorted(TYPES))
def test_a_nan_key_alone_in_its_split(kind, L):
    """The newest key, the only one of the last of three splits (of 32 or 64 keys)."""
    for hint in HINTS:
        bt = Batch([(1, L), (1, L - 20)], seed=44, **TYPES[kind])
        set_row(bt, bt.k, 0, L - 1, NAN)
        for window in (None, (1, 0), (L - 1, 2)):
            got = attend(bt, window, hint=hint, splits=3)
            assert torch.isnan(got[0]).all() and torch.isfinite(got[1]).all()


def far_split(kind, **kw):
    """One token over 640 keys, the first half of them with scores e^-500 below the others'."""
    bt = Batch([(1, 640)], seed=45, **TYPES[kind], **kw)
    one, minus = (0x50, 0xd0) if bt.fp8 else (6.0, -6.0)
    p = torch.arange(640, device="cuda")
    rows = bt.rows(bt.k, 0, p)
    rows[:] = one
    rows[:320] = minus
    bt.put(bt.k, 0, p, rows)
    if bt.fp8:
        bt.k_scale.fill_(0.75)
    bt.q.fill_(4.0)
    return bt


@pytest.mark.parametrize("splits", [1, 2, 5, 20])
@pytest.mark.parametrize("kind", sorted(TYPES))
def test_nan_keys_and_values_far_below_the_maximum(kind, splits):
    """A NaN score counts though its split's other scores vanish beside the maximum; a NaN value that
    the row sees shows though its weight rounds to zero, and an infinite one gives inf or NaN."""
    for hint in HINTS:
        bt = far_split(kind)
        assert torch.isfinite(attend(bt, hint=hint, splits=splits)).all()
        set_row(bt, bt.k, 0, 100, NAN)
        assert torch.isnan(attend(bt, hint=hint, splits=splits)).all()
        for value in (NAN, math.inf):
            bt = far_split(kind)
            at = torch.tensor([100], device="cuda")
            row = bt.rows(bt.v, 0, at)
            row[:, :, 9] = 0x7f if bt.fp8 else value
            bt.put(bt.v, 0, at, row)
            got = attend(bt, hint=hint, splits=splits)
            assert not torch.isfinite(got[..., 9]).any()
            got[..., 9] = 0
            assert torch.isfinite(got).all()
