"""The calls that README.md shows run as they stand, one block after the other."""

import os
import re

import pytest
import torch

from paper_2605_01910_amd import santa as S
from tests.chunk_util import SCALE, Batch, check
from tests.test_gpu_rope import new_rows

README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


@pytest.mark.gpu
def test_new_tokens_example():
    """A prompt's chunk, then a decode step: q1, k1, v1 are its rows, and ctx_len has moved on."""
    code = [c for c in re.findall(r"```python\n(.*?)```", open(README).read(), re.S) if "S.santa_" in c]
    assert code
    bt = Batch([(40, 300), (7, 90)], layout="paged", seed=49, n=400)
    one = Batch([(1, 301), (1, 91)], layout="paged", seed=50, n=400)
    (q, k, v), (q1, k1, v1) = new_rows(bt, True), new_rows(one, True)
    one.k, one.v, one.table = bt.k, bt.v, bt.table
    names = dict(k_pages=bt.k, v_pages=bt.v, block_table=bt.table, ctx_len=bt.ctx, n_k=bt.n, q=q, k=k, v=v,
                 num_kv_heads=bt.Hkv, batch=bt.B, q_start=bt.q_start, num_tokens=bt.T, max_tokens=40,
                 q_rot=bt.q, out=torch.full_like(bt.q, 7.0), scale=SCALE,
                 q1=q1, k1=k1, v1=v1, q1_rot=one.q, out1=torch.full_like(one.q, 7.0))
    exec(code[0], names)
    check(bt, names["out"])
    if len(code) > 1:
        bt.ctx += 1
        exec(code[1], names)
        check(one, names["out1"], (names["win"].window, names["win"].sinks))
    assert isinstance(names["plan"], S.santa_rope_t)
