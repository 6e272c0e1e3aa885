"""Batches whose tiles are more than a launch has workgroups."""

import ctypes

import pytest
import torch

from paper_2605_01910_amd import santa as S
from tests.chunk_util import SCALE, Batch, check

pytestmark = pytest.mark.gpu
ref = ctypes.byref


@pytest.mark.parametrize("rows,Hq,Hkv,hint", [(2 ** 25, 128, 128, 0), (2 ** 25, 64, 8, 0), (2 ** 25, 64, 64, 2 ** 20)])
def test_rows_behind_the_last_sequence(rows, Hq, Hkv, hint):
    """2^25 rows, nearly all of them behind the last sequence: they are not read and their outputs are
    left alone, so the buffers of this test end where the sequences do."""
    bt = Batch([(130, 200), (1, 64)], Hq=Hq, Hkv=Hkv, seed=56)
    kv, sh, ch = bt.kv(), bt.shape(), S.chunk_of(bt.q_start, rows, hint)
    ws, out = S.alloc_attend_workspace(sh, kv, ch), torch.full_like(bt.q, 7.0)
    torch.cuda.synchronize()
    assert S.load().santa_attend_chunk(bt.q.data_ptr(), ref(kv), ref(sh), ref(ch), None, SCALE, out.data_ptr(),
                                       ws.data_ptr(), ws.numel(), None) == S.SANTA_OK
    torch.cuda.synchronize()
    check(bt, out)
