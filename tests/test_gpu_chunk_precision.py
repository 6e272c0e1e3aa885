"""Few rows per sequence (drafted and single tokens, windows) in 16-bit and FP8 caches: the weights
are as good as the 32-bit scores, so that the output's own rounding is all but the whole error."""

import math

import pytest
import torch

from paper_2605_01910_amd import santa as S
from tests.chunk_util import SCALE, Batch, answer, attend

pytestmark = pytest.mark.gpu
H = 2.0 ** -8   # half a step of bfloat16, relative to the value


def close(bt, got, window):
    """chunk_util.answer's bound with 2^-14 in the place of a weight's rounding to bfloat16: a weight is
    held in two parts, the second at most 1.5 * 2^-7 of it and rounded by at most H of that."""
    want, tol = answer(bt, window)
    weights = magnitude(bt, window) * (H - 2.0 ** -14)
    over = (got.double() - want).abs() - (tol - weights)
    assert over.max() <= 0, over.max().item()


def magnitude(bt, window):
    """sum_j p_j |v_j| in float64: the answer over |v|."""
    kept = bt.v
    bt.v = bt.v & 0x7f if bt.fp8 else bt.v.abs()
    out = answer(bt, window)[0]
    bt.v = kept
    return out


LENS = [(1, 1), (3, 300), (1, 4000), (8, 2500), (5, 5), (1, 65)]


@pytest.mark.parametrize("window", [None, (500, 4)], ids=str)
@pytest.mark.parametrize("kw", [dict(), dict(layout="paged", Hq=4, Hkv=1), dict(layout="hnd", Hq=3, Hkv=3),
                                dict(fp8=True, layout="paged"), dict(fp8=True)],
                         ids=["bf16", "bf16_paged", "bf16_hnd_g1", "fp8_paged", "fp8"])
def test_few_rows(kw, window):
    bt = Batch(LENS, seed=53, filler=0.0, **kw)
    for hint in (1, 8):
        for splits in (0, 1, 5):
            close(bt, attend(bt, window, hint=hint, splits=splits), window)


@pytest.mark.parametrize("kw", [dict(), dict(fp8=True, layout="paged"), dict(Hq=8, Hkv=1)], ids=["bf16", "fp8", "g8"])
def test_decode_window(kw):
    bt = Batch([(1, 1), (1, 70), (1, 3000), (1, 900)], seed=54, filler=0.0, **kw)
    for window in ((1, 0), (64, 4), (1000, 16)):
        kv, sh, win = bt.kv(), bt.shape(), S.window_of(*window)
        out = torch.full_like(bt.q, 7.0)
        S.santa_decode_window(bt.q, kv, sh, win, SCALE, out, S.alloc_attend_workspace(sh, kv, None, win))
        close(bt, out, window)


def test_infinite_values_of_every_weight():
    """Both parts of a weight are positive: a value of +inf gives +inf whatever its weight, in tiles
    that every row sees."""
    for fill in (math.inf, -math.inf):
        bt = Batch([(2, 640)], seed=55)
        for pos in range(0, 600, 7):
            bt.v[0, pos, :, pos // 7] = fill
        for hint in (0, 1):
            for splits in (1, 4):
                got = attend(bt, hint=hint, splits=splits)
                assert torch.all(got[..., :86] == fill) and torch.isfinite(got[..., 86:]).all()
