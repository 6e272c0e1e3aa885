"""santa_attend_chunk and santa_decode_window against float64: element types, head groups, cache
layouts, ragged chunks from none to long, windows with sinks, and hidden keys and values that must
not show (tests/chunk_util.py derives the bounds)."""

import pytest
import torch

from paper_2605_01910_amd import santa as S
from tests.chunk_util import SCALE, Batch, attend, check

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32

RAGGED = [(1, 1), (0, 5), (3, 70), (33, 33), (1, 513), (17, 200), (0, 0), (129, 300)]
CASES = {
    "one_token": dict(lens=[(1, 1)]),
    "one_token_long": dict(lens=[(1, 2049)]),
    "whole_prompt": dict(lens=[(257, 257)]),
    "ragged": dict(lens=RAGGED, pad=3),
    "ragged_hnd": dict(lens=RAGGED, layout="hnd", pad=1),
    "ragged_paged": dict(lens=RAGGED, layout="paged", pad=5),
    "ragged_paged_1": dict(lens=RAGGED, layout="paged", page=1),
    "ragged_paged_64": dict(lens=RAGGED, layout="paged", page=64),
    "ragged_paged_8": dict(lens=RAGGED, layout="paged", page=8),
    "page_past_context": dict(lens=RAGGED, layout="paged", page=2048),
    "padded_rows": dict(lens=RAGGED, gap=8),
    "padded_pages": dict(lens=RAGGED, layout="paged", gap=8, Hq=5, Hkv=5),
    "group_1": dict(lens=RAGGED, Hq=3, Hkv=3),
    "group_2": dict(lens=RAGGED, Hq=6, Hkv=3, layout="hnd"),
    "group_8": dict(lens=RAGGED, Hq=8, Hkv=1, layout="paged"),
    "f32": dict(lens=RAGGED, dtype=F32, pad=2),
    "f32_paged_group_1": dict(lens=RAGGED, dtype=F32, Hq=2, Hkv=2, layout="paged"),
    "f32_group_8": dict(lens=RAGGED, dtype=F32, Hq=8, Hkv=1, layout="hnd", gap=4),
    "fp8": dict(lens=RAGGED, fp8=True),
    "fp8_paged": dict(lens=RAGGED, fp8=True, layout="paged", Hq=16, Hkv=2, pad=9),
    "fp8_hnd_group_1": dict(lens=RAGGED, fp8=True, layout="hnd", Hq=2, Hkv=2, gap=16),
    # past one load of 64 table entries, and past the one fetched ahead
    "long_paged": dict(lens=[(70, 3000), (1, 2500), (9, 1100)], layout="paged"),
    "long_paged_f32": dict(lens=[(70, 2300)], layout="paged", dtype=F32, Hq=2, Hkv=1),
    "long_paged_fp8": dict(lens=[(70, 3000), (2, 2500)], layout="paged", fp8=True),
    "many_sequences": dict(lens=[(i % 4, 3 + i) for i in range(150)], layout="paged"),
}
WINDOWS = [None, (1, 0), (40, 4), (64, 100), (1000, 1)]


@pytest.mark.parametrize("window", WINDOWS, ids=str)
@pytest.mark.parametrize("case", sorted(CASES))
def test_chunk(case, window):
    """Both kernels (by the hint), unsplit and split; hints that are too small (1 for the few-row
    kernel, 9 to 33 tokens for full tiles) leave tiles that the grid was not made for."""
    bt = Batch(seed=len(case), **CASES[case])
    for hint in (0, 1, 32 // bt.G + 1):
        for splits in (0, 3):
            check(bt, attend(bt, window, hint=hint, splits=splits), window)


@pytest.mark.parametrize("splits", [1, 2, 7, 64, 256])
@pytest.mark.parametrize("hint", [0, 2])
def test_splits(splits, hint):
    bt = Batch([(2, 3000), (1, 5), (5, 1500)], seed=3)
    for window in (None, (700, 4)):
        check(bt, attend(bt, window, hint=hint, splits=splits), window)


@pytest.mark.parametrize("kw", [dict(), dict(dtype=F32), dict(fp8=True)], ids=["bf16", "f32", "fp8"])
@pytest.mark.parametrize("layout", ["nhd", "paged"])
def test_decode_window(kw, layout):
    """The single-token call, also without ctx_len, and with windows longer than the context."""
    lens = [(1, 1), (1, 64), (1, 65), (1, 700), (1, 4000)]
    for Hq, Hkv in ((8, 1), (4, 2), (3, 3)):
        bt = Batch(lens, Hq=Hq, Hkv=Hkv, layout=layout, seed=5, **kw)
        for window in ((1, 0), (64, 4), (257, 16), (5000, 3), (2 ** 31 - 1, 2 ** 31 - 1)):
            win, kv, sh = S.window_of(*window), bt.kv(), bt.shape()
            ws = S.alloc_attend_workspace(sh, kv, None, win)
            out = torch.full_like(bt.q, 7.0)
            S.santa_decode_window(bt.q, kv, sh, win, SCALE, out, ws)
            check(bt, out, window)
    if layout == "nhd":
        bt = Batch([(1, 333)] * 3, seed=6, **kw)
        kv, sh, win = bt.kv(), bt.shape(), S.window_of(100, 4)
        kv.ctx_len = None
        out = torch.full_like(bt.q, 7.0)
        S.santa_decode_window(bt.q, kv, sh, win, SCALE, out, S.alloc_attend_workspace(sh, kv, None, win))
        check(bt, out, (100, 4))


@pytest.mark.parametrize("kw", [dict(), dict(dtype=F32)], ids=["bf16", "f32"])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_hidden_values_reach_no_row(kw, value):
    """A non-finite value row shows in exactly the rows that see it, a non-finite key hidden from a
    row does not show there: in a chunk's own later tokens, and before a window."""
    for window in (None, (30, 2)):
        for hint in (0, 1):
            bt = Batch([(40, 200), (3, 100)], seed=9, **kw)
            dev = bt.q.device
            v = bt.rows(bt.v, 0, torch.tensor([170, 185], device=dev))
            v[:, :, 5:9] = value
            bt.put(bt.v, 0, torch.tensor([170, 185], device=dev), v)
            check(bt, attend(bt, window, hint=hint), window)
    # keys: the last token's key is hidden from all but the last row
    for hint in (0, 1):
        bt = Batch([(9, 64)], seed=10, **kw)
        clean = attend(bt, hint=hint)
        k = bt.rows(bt.k, 0, torch.tensor([63], device=bt.q.device))
        bt.put(bt.k, 0, torch.tensor([63], device=bt.q.device), torch.full_like(k, value))
        assert torch.equal(attend(bt, hint=hint)[:8], clean[:8])


@pytest.mark.parametrize("layout", ["nhd", "paged"])
def test_hidden_fp8_nan(layout):
    """The NaN code in a value row: in the rows that see it, with and without a window."""
    for window in (None, (30, 2)):
        for hint in (0, 1):
            bt = Batch([(40, 200), (3, 100)], seed=23, fp8=True, layout=layout)
            at = torch.tensor([170, 185], device=bt.q.device)
            v = bt.rows(bt.v, 0, at)
            v[:, :, 5], v[:, :, 9] = 0x7f, 0xff
            bt.put(bt.v, 0, at, v)
            check(bt, attend(bt, window, hint=hint), window)


def test_nonfinite_values_in_a_split_call():
    for value in (float("inf"), float("nan")):
        bt = Batch([(40, 900), (2, 700)], seed=24)
        at = torch.tensor([880, 899], device=bt.q.device)
        v = bt.rows(bt.v, 0, at)
        v[:, :, 100:] = value
        bt.put(bt.v, 0, at, v)
        for hint in (0, 1):
            check(bt, attend(bt, hint=hint, splits=5))


def test_a_nan_query_stays_in_its_row():
    for hint in (0, 1):
        bt = Batch([(40, 200)], seed=25)
        clean = attend(bt, hint=hint)
        bt.q[7, 3, 11] = float("nan")
        got = attend(bt, hint=hint)
        assert torch.isnan(got[7, 3]).all()
        got[7, 3] = clean[7, 3]
        assert torch.equal(got, clean)


def test_window_reads_no_hidden_page():
    """Pages between the sinks and the window are another sequence's by now: a page of NaN."""
    bt = Batch([(1, 1000), (4, 2000)], layout="paged", seed=11)
    want = attend(bt, (100, 4))
    filler = bt.table[0, -1].item()
    bt.table[0, 1:56] = filler          # window (900, 1000)
    bt.table[1, 1:118] = filler         # window of the first of four tokens: (1896, 1997)
    assert torch.equal(attend(bt, (100, 4)), want)
    assert torch.isfinite(want).all()


@pytest.mark.parametrize("scale", [0.0, -0.05, 1.5])
@pytest.mark.parametrize("kw", [dict(), dict(dtype=F32), dict(fp8=True)], ids=["bf16", "f32", "fp8"])
def test_scales(scale, kw):
    bt = Batch([(5, 90), (40, 300)], seed=12, **kw)
    for hint in (0, 1):
        check(bt, attend(bt, scale=scale, hint=hint), scale=scale)


@pytest.mark.parametrize("hint", [0, 1])
def test_context_shorter_than_chunk(hint):
    """Tokens before position 0 see nothing and give zero rows; a context past n_k counts as n_k."""
    bt = Batch([(5, 60), (4, 40)], seed=13)
    whole = attend(bt, hint=hint)
    bt.ctx[0] = 3          # two of five tokens stand before position 0
    bt.lens = [(5, 3), (4, 40)]
    got = attend(bt, hint=hint)
    assert torch.all(got[:2] == 0) and torch.equal(got[5:9], whole[5:9])
    one = Batch([(3, 3)], seed=14)
    one.k[0, :3], one.v[0, :3] = bt.k[0, :3], bt.v[0, :3]
    one.q[:] = bt.q[2:5]
    check(one, got[2:5])
    bt.ctx[0] = 0
    assert torch.all(attend(bt, hint=hint)[:5] == 0)
    bt.ctx[0], bt.ctx[1] = 10 ** 9, 40
    same = attend(bt, hint=hint)
    bt.ctx[0] = bt.n
    assert torch.equal(attend(bt, hint=hint), same)


def test_offsets_past_32_bits():
    """A pool of more than 2^31 elements, the sequence in its last pages."""
    bt = Batch([(20, 300), (1, 900)], Hq=8, Hkv=8, layout="paged", pages=135000, seed=15)
    assert bt.k.shape[0] * bt.k.stride(0) > 2 ** 31 and bt.table.min() > 130000
    for hint in (0, 1):
        for window in (None, (100, 4)):
            check(bt, attend(bt, window, hint=hint), window)


def test_much_padding():
    """Far more rows than tokens: a batch captured for a larger one."""
    for kw in (dict(), dict(layout="paged", fp8=True)):
        bt = Batch([(1, 900), (5, 700), (0, 3), (40, 300)], pad=1500, seed=33, **kw)
        for hint in (0, 1, 5, 40, 100):
            for splits in (0, 3):
                check(bt, attend(bt, (200, 4), hint=hint, splits=splits), (200, 4))


def test_the_same_call_twice_is_equal():
    bt = Batch([(300, 900), (1, 5000)], seed=16)
    for hint in (0, 1):
        assert torch.equal(attend(bt, hint=hint), attend(bt, hint=hint))


def test_captured_calls_share_a_workspace():
    """Two captured graphs on one workspace, another stream, replays between eager calls."""
    a, b = Batch([(7, 500), (1, 2000)], seed=17), Batch([(1, 3000)] * 2, seed=18, layout="paged")
    wants = [attend(a), attend(b, (800, 4), hint=1)]
    kv, sh, ch = a.kv(), a.shape(), a.chunk()
    kvb, shb, chb, win = b.kv(), b.shape(), b.chunk(1), S.window_of(800, 4)
    n = max(S.santa_attend_workspace_size(sh, kv, ch), S.santa_attend_workspace_size(shb, kvb, chb, win))
    ws = torch.empty(n + 256, dtype=torch.uint8, device="cuda")
    ws = ws[(-ws.data_ptr()) % 256:][:n]
    S.santa_workspace_init(ws)
    outs = [torch.zeros_like(a.q), torch.zeros_like(b.q)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            if i == 0:
                S.santa_attend_chunk(a.q, kv, sh, ch, None, SCALE, outs[0], ws)
            else:
                S.santa_attend_chunk(b.q, kvb, shb, chb, win, SCALE, outs[1], ws)
        graphs.append(g)
    for _ in range(3):
        for o in outs:
            o.zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, wants))
        # an eager decode step on the same workspace between the replays
        d = torch.zeros_like(b.q)
        with torch.cuda.stream(side):
            S.santa_attend_chunk(b.q, kvb, shb, chb, win, SCALE, d, ws)
        torch.cuda.synchronize()
        assert torch.equal(d, wants[1])


def test_workspace_shared_with_the_decode_calls():
    """A dense decode step and a window step in turn on one workspace; the dense step over the
    whole context equals the chunk call's single token within both bounds."""
    bt = Batch([(1, 700), (1, 3000)], Hq=8, Hkv=2, seed=19)
    kv, sh = bt.kv(), bt.shape()
    n = max(S.santa_workspace_size(sh, kv, 1, S.SANTA_KIND_DENSE), S.santa_attend_workspace_size(sh, kv))
    ws = torch.empty(n + 256, dtype=torch.uint8, device="cuda")
    ws = ws[(-ws.data_ptr()) % 256:][:n]
    S.santa_workspace_init(ws)
    first = None
    for _ in range(3):
        dense, chunk = torch.full_like(bt.q, 7.0), torch.full_like(bt.q, 7.0)
        S.santa_decode_dense(bt.q, kv, sh, SCALE, dense, ws)
        S.santa_attend_chunk(bt.q, kv, sh, None, None, SCALE, chunk, ws)
        S.check_workspace(ws)
        check(bt, chunk)
        check(bt, dense)
        assert first is None or torch.equal(first, chunk)
        first = chunk


def test_streams_and_the_call_timer():
    """Calls on two streams at once, each with its own workspace; the events of santa_time_next_call
    span a call's one or two kernels."""
    bt = Batch([(1, 3000), (200, 900)], seed=26)
    want = attend(bt)
    kv, sh, ch = bt.kv(), bt.shape(), bt.chunk()
    streams = [torch.cuda.Stream() for _ in range(2)]
    ws = [S.alloc_attend_workspace(sh, kv, ch) for _ in streams]
    outs = [torch.zeros_like(bt.q) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, w, o in zip(streams, ws, outs):
            S.santa_attend_chunk(bt.q, kv, sh, ch, None, SCALE, o, w, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    for splits in (1, 4):
        with S.options("auto", splits):
            w = S.alloc_attend_workspace(sh, kv, ch)
            e = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
            for x in e:
                x.record()
            torch.cuda.synchronize()
            S.santa_time_next_call(*e)
            S.santa_attend_chunk(bt.q, kv, sh, ch, None, SCALE, outs[0], w)
            torch.cuda.synchronize()
            assert 0 < e[0].elapsed_time(e[1]) < 100


def test_without_context_lengths():
    """No ctx_len: every sequence has n_k keys."""
    bt = Batch([(5, 300), (0, 300), (40, 300)], seed=27)
    kv, sh, ch = bt.kv(), bt.shape(), bt.chunk()
    kv.ctx_len = None
    out = torch.full_like(bt.q, 7.0)
    S.santa_attend_chunk(bt.q, kv, sh, ch, None, SCALE, out, S.alloc_attend_workspace(sh, kv, ch))
    check(bt, out)


def test_ends_outside_the_buffers():
    """q_start entries past num_tokens count as num_tokens, falling ones as none: no call names a
    row outside its buffers, and the sequences before them are as ever."""
    bt = Batch([(5, 60), (4, 40), (3, 50)], seed=28)
    want = attend(bt)
    bt.q_start[3] = 1000
    assert torch.equal(attend(bt), want)
    bt.q_start[:] = torch.tensor([0, 5, 2, 2], dtype=torch.int32)
    got = attend(bt)
    assert torch.equal(got[:5], want[:5]) and torch.all(got[5:] == 7.0)


def test_calls_leave_the_counters_at_zero():
    """A call whose last split joins the others (one token, few heads) counts them in the workspace's
    shared head and clears the count: calls of other shapes and kinds find it as they need it."""
    head = 256 + 4096 * (2 * 32 + 2 * 8 * 64) * 4
    one, two = Batch([(1, 4000), (1, 900)], seed=31), Batch([(1, 2500)] * 3, Hq=2, Hkv=1, seed=32, layout="paged")
    n = max(S.santa_attend_workspace_size(x.shape(), x.kv()) for x in (one, two))
    n = max(n, S.santa_workspace_size(one.shape(), one.kv(), 1, S.SANTA_KIND_DENSE))
    ws = torch.empty(n + 256, dtype=torch.uint8, device="cuda")
    ws = ws[(-ws.data_ptr()) % 256:][:n]
    S.santa_workspace_init(ws)
    for _ in range(3):
        for bt, win in ((one, None), (two, S.window_of(600, 4))):
            out = torch.full_like(bt.q, 7.0)
            S.santa_attend_chunk(bt.q, bt.kv(), bt.shape(), None, win, SCALE, out, ws)
            check(bt, out, (600, 4) if win else None)
            assert not ws[:head].any()
    S.santa_decode_dense(one.q, one.kv(), one.shape(), SCALE, out := torch.full_like(one.q, 7.0), ws)
    check(one, out)
    S.santa_attend_chunk(one.q, one.kv(), one.shape(), None, None, SCALE, out, ws)
    check(one, out)


def test_argument_checks():
    bt = Batch([(2, 40)], seed=20)
    kv, sh, ch = bt.kv(), bt.shape(), bt.chunk()
    ws, out = S.alloc_attend_workspace(sh, kv, ch), torch.empty_like(bt.q)
    with pytest.raises(ValueError):
        S.santa_attend_chunk(bt.q[:, :4], kv, sh, ch, None, SCALE, out, ws)
    with pytest.raises(ValueError):
        S.santa_attend_chunk(bt.q[:1], kv, sh, ch, None, SCALE, out, ws)
    with pytest.raises(TypeError):
        S.santa_attend_chunk(bt.q.float(), kv, sh, ch, None, SCALE, out, ws)
    with pytest.raises(TypeError):
        S.santa_attend_chunk(bt.q.cpu(), kv, sh, ch, None, SCALE, out, ws)
    with pytest.raises(ValueError):
        S.santa_attend_chunk(bt.q.transpose(0, 1).contiguous().transpose(0, 1), kv, sh, ch, None, SCALE, out, ws)
    with pytest.raises(S.SantaError):
        S.santa_attend_chunk(bt.q, kv, sh, ch, None, SCALE, out, ws[:256])
    with pytest.raises(ValueError):
        S.santa_attend_chunk(bt.q, kv, sh, ch, None, SCALE, out, torch.zeros(ws.numel(), dtype=torch.uint8))
    with pytest.raises(TypeError):
        S.chunk_of(bt.q_start.cpu(), bt.T)
    with pytest.raises(TypeError):
        S.chunk_of(bt.q_start.long(), bt.T)


def test_launch_path_options_are_ignored():
    """The decode steps' path options change nothing here, FP8 caches included."""
    for kw in (dict(), dict(fp8=True)):
        bt = Batch([(40, 90), (1, 300)], seed=29, **kw)
        want = attend(bt)
        kv, sh, ch = bt.kv(), bt.shape(), bt.chunk()
        for path in ("one", "two", "multi", "rows"):
            with S.options(path):
                out = torch.full_like(bt.q, 7.0)
                S.santa_attend_chunk(bt.q, kv, sh, ch, None, SCALE, out, S.alloc_attend_workspace(sh, kv, ch))
                assert torch.equal(out, want)


@pytest.mark.parametrize("kw", [dict(), dict(layout="paged"), dict(fp8=True)], ids=["nhd", "paged", "fp8"])
def test_shared_prefix_and_equal_rows(kw):
    """Two sequences over the same cache rows (a batch stride of 0, or the same pages): equal queries
    give equal outputs, whatever their place in the batch."""
    bt = Batch([(6, 700), (6, 700)], seed=30, **kw)
    if bt.layout == "paged":
        bt.table[1] = bt.table[0]
    else:
        bt.k, bt.v = bt.k[:1].expand(2, -1, -1, -1), bt.v[:1].expand(2, -1, -1, -1)
    if bt.fp8:
        bt.k_scale[1], bt.v_scale[1] = bt.k_scale[0], bt.v_scale[0]
    bt.q[6:] = bt.q[:6]
    for hint in (0, 1):
        got = attend(bt, (300, 4), hint=hint)
        assert torch.equal(got[:6], got[6:])
        check(bt, got, (300, 4))
