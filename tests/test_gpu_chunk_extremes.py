"""Values near the largest of their type, and sequences without keys in split calls."""

import pytest
import torch

from paper_2605_01910_amd import santa as S
from tests.chunk_util import SCALE, Batch, attend, check

pytestmark = pytest.mark.gpu
F32 = torch.float32


@pytest.mark.parametrize("kw", [dict(), dict(dtype=F32)], ids=["bf16", "f32"])
@pytest.mark.parametrize("rise", [1.0, 5.0, 60.0])
def test_values_near_the_largest(kw, rise):
    """One value of 2e38 whose key scores `rise` above the earlier keys': no weight passes 1 on the way,
    so no sum that the output does not call for overflows."""
    for L in (70, 200, 1500):
        for hint in (0, 1):
            for splits in (0, 1, 3):
                bt = Batch([(1, L)], seed=57, **kw)
                bt.q[:] = 0
                bt.q[..., 0] = 8.0
                p = torch.arange(L, device="cuda")
                k, v = bt.rows(bt.k, 0, p), bt.rows(bt.v, 0, p)
                k[:] = 0
                k[L - 3, :, 0] = rise / (8.0 * SCALE)
                v[L - 3, :, 7] = 2e38
                v[L - 2, :, 9] = -2e38
                bt.put(bt.k, 0, p, k)
                bt.put(bt.v, 0, p, v)
                got = attend(bt, hint=hint, splits=splits)
                assert torch.isfinite(got).all()
                check(bt, got)


@pytest.mark.parametrize("kw", [dict(), dict(dtype=F32), dict(fp8=True), dict(layout="paged", Hq=8, Hkv=1)],
                         ids=["bf16", "f32", "fp8", "g8"])
@pytest.mark.parametrize("splits", [0, 1, 3, 64, 200])
def test_sequences_without_keys(kw, splits):
    """ctx_len 0 beside others: rows of zeros, whichever kernel joins the splits."""
    bt = Batch([(1, 900), (1, 1), (1, 70)], seed=58, **kw)
    bt.ctx[1] = 0
    kv, sh = bt.kv(), bt.shape()
    for window in (None, (100, 4)):
        win = S.window_of(*window) if window else None
        with S.options("auto", splits):
            ws = S.alloc_attend_workspace(sh, kv, None, win)
            out = torch.full_like(bt.q, 7.0)
            S.santa_attend_chunk(bt.q, kv, sh, None, win, SCALE, out, ws)
        torch.cuda.synchronize()
        assert torch.all(out[1] == 0)
        rest = Batch([(1, 900), (1, 1), (1, 70)], seed=58, **kw)
        out[1] = attend(rest, window, splits=splits)[1]
        check(rest, out, window)
