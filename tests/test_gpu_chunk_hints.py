"""Hints that are too small by far: tiles that the grid was not made for are taken unsplit by its
workgroups, however the grid's own tiles are split and joined, in workspaces of the hint's size."""

import pytest
import torch

from paper_2605_01910_amd import santa as S
from tests.chunk_util import SCALE, Batch, check

pytestmark = pytest.mark.gpu
TYPES = {"bf16": dict(), "f32": dict(dtype=torch.float32), "fp8_paged": dict(fp8=True, layout="paged"),
         "paged_g8": dict(layout="paged", Hq=8, Hkv=1)}


@pytest.mark.parametrize("splits", [0, 1, 2, 5, 64])
@pytest.mark.parametrize("kind", sorted(TYPES))
def test_small_hints(kind, splits):
    bt = Batch([(300, 900), (0, 7), (1, 1500), (70, 333), (2, 1200)], pad=700, seed=51, **TYPES[kind])
    kv, sh = bt.kv(), bt.shape()
    for window in (None, (200, 4)):
        win = S.window_of(*window) if window else None
        for hint in (1, 2, 32 // bt.G + 1, 100):
            with S.options("auto", splits):
                n = S.santa_attend_workspace_size(sh, kv, bt.chunk(hint), win)
                room = torch.full((n + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
                ws = room[(-room.data_ptr()) % 256:][:n]
                behind = room[ws.data_ptr() - room.data_ptr() + n:]
                S.santa_workspace_init(ws)
                for _ in range(2):
                    out = torch.full_like(bt.q, 7.0)
                    S.santa_attend_chunk(bt.q, kv, sh, bt.chunk(hint), win, SCALE, out, ws)
                    check(bt, out, window)
            assert torch.all(behind == 0x5a)
            S.check_workspace(ws)
