"""Mean squares of the chunk attention's errors, row by row.  A key that is dropped or counted twice
among hundreds moves a 16-bit output by less than the worst case of all roundings together, but by
far more than they come to on average."""

import math

import pytest
import torch

from tests.chunk_util import SCALE, Batch, attend

H = 2.0 ** -8   # half a step of bfloat16, relative to the value
SOFT = SCALE / 4  # of scores that leave every key a share: what one key brings is not hidden by a few large ones


def squares(bt, window=None, scale=SOFT):
    """Per row, in float64: the answer [T, Hq, 128] and a bound of the mean square of its errors.

    A value is rounded by at most H of itself, evenly over that range, so on average by H / sqrt(3):
    with weights p_j the output's own rounding gives o^2 H^2 / 3 and the weights' (independent of
    each other) sum_j p_j^2 v_j^2 H^2 / 3.  A rounding can stay at H for all 128 features of a row,
    since a weight is rounded once for all of them: three times that; and once more for what 128
    features leave to chance."""
    out = torch.zeros((bt.T, bt.Hq, 128), dtype=torch.float64, device=bt.q.device)
    most = torch.zeros((bt.T, bt.Hq), dtype=torch.float64, device=bt.q.device)
    for b, (c, L) in enumerate(bt.lens):
        if not c:
            continue
        k, v = bt.values(bt.k, b, L), bt.values(bt.v, b, L)
        p, j = torch.arange(L - c, L, device=k.device)[:, None], torch.arange(L, device=k.device)[None]
        seen = j <= p
        if window:
            seen = seen & ((j > p - window[0]) | (j < window[1]))
        at = bt.starts[b]
        for h in range(bt.Hq):
            s = (bt.q[at:at + c, h].double() @ k[:, h // bt.G].T * scale).masked_fill(~seen, -math.inf)
            w = s.softmax(-1)
            o = w @ v[:, h // bt.G]
            out[at:at + c, h] = o
            most[at:at + c, h] = 4 * H * H / 3 * ((w * w) @ (v[:, h // bt.G] ** 2).mean(-1) + (o * o).mean(-1))
    return out, most


LENS = [(3, 300), (1, 4000), (150, 1500), (33, 33), (9, 2500), (1, 700)]


@pytest.mark.gpu
@pytest.mark.parametrize("window", [None, (500, 4), (1000, 40)], ids=str)
@pytest.mark.parametrize("kw", [dict(), dict(layout="paged", Hq=8, Hkv=1), dict(layout="hnd", Hq=3, Hkv=3),
                                dict(fp8=True, layout="paged"), dict(fp8=True, Hq=8, Hkv=1)],
                         ids=["bf16", "bf16_paged_g8", "bf16_hnd_g1", "fp8_paged", "fp8_g8"])
def test_mean_squares(kw, window):
    bt = Batch(LENS, seed=47, **kw)
    want, most = squares(bt, window)
    for hint in (0, 1, 32 // bt.G):
        for splits in (0, 1, 5):
            err = ((attend(bt, window, SOFT, hint=hint, splits=splits).double() - want) ** 2).mean(-1)
            assert (err <= most).all(), (err / most).max().item()


def test_the_bound_finds_a_dropped_key():
    """One key left out of the answer itself: nearly every row's mean square passes the bound."""
    for L in (300, 900):
        bt = Batch([(3, L)], seed=48, device="cpu")
        bt.q[:, :, :1] = 1.0
        want, most = squares(bt)
        bt.k[0, 50] = 0
        bt.k[0, 50, :, :1] = -1e5       # its score: e^-2000 of the others'
        dropped, _ = squares(bt)
        assert (((dropped - want) ** 2).mean(-1) > most).double().mean() > 0.9
