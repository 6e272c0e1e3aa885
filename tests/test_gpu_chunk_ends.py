"""Chunks whose rows do not begin at 0 (a view into longer prefix sums), ends past the buffers and
falling ones: the rotary store and the attention agree on which row holds which token."""

import pytest
import torch

from paper_2605_01910_amd import santa as S
from tests.chunk_util import SCALE, Batch
from tests.test_gpu_rope import F32, RAGGED, THETA, new_rows

pytestmark = pytest.mark.gpu
KINDS = {"bf16": dict(), "paged": dict(layout="paged"), "f32": dict(dtype=F32, layout="hnd"),
         "fp8": dict(fp8=True, layout="paged"),
         "four_tokens_a_workgroup": dict(lens=[(1, 1), (2050, 2100), (0, 9), (2049, 2060)], Hq=2, Hkv=1)}


def store(bt, q, k, v, q_start):
    """Outputs and caches after santa_rope_append of rows q, k, v on copies of bt's caches."""
    kept = bt.k, bt.v
    bt.k, bt.v = ((x.contiguous().clone()) for x in kept)
    out = torch.full_like(q, 7.0)
    S.santa_rope_append(q, k, v, bt.kv(), bt.shape(), S.chunk_of(q_start, q.shape[0]),
                        S.rope_plan(128, False, THETA), out)
    torch.cuda.synchronize()
    got, (bt.k, bt.v) = (out, bt.k, bt.v), kept
    return got


def attention(bt, q, q_start, hint):
    kv, sh, ch = bt.kv(), bt.shape(), S.chunk_of(q_start, q.shape[0], hint)
    out = torch.full_like(q, 7.0)
    S.santa_attend_chunk(q, kv, sh, ch, None, SCALE, out, S.alloc_attend_workspace(sh, kv, ch))
    torch.cuda.synchronize()
    return out


def same(a, b):
    return torch.equal(torch.nan_to_num(a.float(), 9), torch.nan_to_num(b.float(), 9))


def batch(kind, **more):
    kw = dict(KINDS[kind], **more)
    return Batch(kw.pop("lens", RAGGED), **kw)


@pytest.mark.parametrize("lead", [1, 4, 37])
@pytest.mark.parametrize("kind", sorted(KINDS))
def test_rows_before_the_first_sequence(kind, lead):
    """q_start[0] > 0: the rows before it hold no token.  They are not stored, their outputs are left
    as they were, and all else is as in the call on the rows from there on."""
    bt = batch(kind, pad=lead + 5, seed=40)
    q, k, v = new_rows(bt, False)
    want = store(bt, q[lead:].contiguous(), k[lead:], v[lead:], bt.q_start)
    got = store(bt, q, k, v, bt.q_start + lead)
    assert torch.all(got[0][:lead] == 7.0) and torch.equal(got[0][lead:], want[0])
    assert same(got[1], want[1]) and same(got[2], want[2])
    for hint in (0, 1):
        a = attention(bt, q[lead:].contiguous(), bt.q_start, hint)
        b = attention(bt, q, bt.q_start + lead, hint)
        assert torch.all(b[:lead] == 7.0) and torch.equal(b[lead:], a)


@pytest.mark.parametrize("kind", sorted(KINDS))
def test_ends_past_the_buffers(kind):
    """An end past num_tokens counts as num_tokens, in the store as in the attention."""
    bt = batch(kind, seed=41)
    q, k, v = new_rows(bt, False)
    ends = bt.q_start.clone()
    ends[bt.starts.index(bt.T):] = bt.T + 990
    want, got = store(bt, q, k, v, bt.q_start), store(bt, q, k, v, ends)
    assert all(same(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("kind", sorted(KINDS))
def test_falling_ends(kind):
    """A sequence whose end lies before its start has no tokens; the rows that no sequence holds are
    not stored and their outputs are left as they were."""
    kw = {x: y for x, y in KINDS[kind].items() if x != "lens"}
    bt = Batch([(5, 60), (4, 40), (3, 50)], seed=42, **kw)
    q, k, v = new_rows(bt, False)
    falling = torch.tensor([0, 5, 2, 2], dtype=torch.int32, device="cuda")
    none = torch.tensor([0, 5, 5, 5], dtype=torch.int32, device="cuda")
    want, got = store(bt, q, k, v, none), store(bt, q, k, v, falling)
    assert torch.all(got[0][5:] == 7.0)
    assert all(same(a, b) for a, b in zip(got, want))
