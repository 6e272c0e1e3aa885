"""santa_rope_append where a workgroup takes four tokens (4096 rows and more, fewer than 32 heads in
all), against float64: every element type and layout, sequences that begin and end inside a group of
four, rows behind the last one, and more rows than a launch of one workgroup per token has threads."""

import pytest
import torch

from paper_2605_01910_amd import santa as S
from tests.chunk_util import HALF, Batch
from tests.test_gpu_rope import F32, THETA, bound, new_rows, positions_of, rotated

pytestmark = pytest.mark.gpu

LENS = [(1, 1), (1102, 1210), (0, 5), (3, 70), (2, 2), (1999, 1999), (1, 900), (1000, 1003)]   # 4108 tokens
CASES = {
    "bf16": dict(pad=3),
    "bf16_paged": dict(layout="paged", pad=1, Hq=16, Hkv=4),
    "bf16_hnd": dict(layout="hnd", gap=8, Hq=4, Hkv=4),
    "f32_paged": dict(dtype=F32, layout="paged", pad=2, Hq=3, Hkv=3),
    "f32": dict(dtype=F32, Hq=2, Hkv=1, pad=5),
    "fp8": dict(fp8=True, pad=2, Hq=8, Hkv=1),
    "fp8_paged": dict(fp8=True, layout="paged", pad=6, Hq=16, Hkv=2),
}


@pytest.mark.parametrize("R,interleaved", [(128, False), (128, True), (32, False)])
@pytest.mark.parametrize("queries", [True, False])
@pytest.mark.parametrize("case", sorted(CASES))
def test_four_tokens_a_workgroup(case, queries, R, interleaved):
    bt = Batch(LENS, seed=R, **CASES[case])
    assert bt.T > 4096 and bt.Hq + 2 * bt.Hkv < 32
    q, k, v = new_rows(bt, fused=queries)
    before = [x.clone() for x in (bt.k, bt.v)]
    out = torch.full((bt.T, bt.Hq, 128), 7.0, dtype=bt.dtype, device="cuda")
    S.santa_rope_append(q if queries else None, k, v, bt.kv(), bt.shape(), bt.chunk(),
                        S.rope_plan(R, interleaved, THETA), out if queries else None)
    torch.cuda.synchronize()
    _, pos = positions_of(bt)
    used = bt.starts[-1]
    if queries:
        assert torch.all(out[used:] == 7.0)
        over = (out.double() - rotated(q, pos, R, interleaved)).abs() - bound(q, bt.dtype, R)
        assert over[:used].amax() <= 0
        assert torch.equal(out[:used, :, R:], q[:used, :, R:])
    kr = rotated(k, pos, R, interleaved)
    for b, (c, L) in enumerate(bt.lens):
        at, p = bt.starts[b], torch.arange(L - c, L, device="cuda")
        gk, gv = bt.rows(bt.k, b, p), bt.rows(bt.v, b, p)
        if bt.fp8:
            for got, x, scale, slack in ((gk, kr, bt.k_scale, bound(k, F32, R)), (gv, v.double(), bt.v_scale, None)):
                s = scale[b].double()[:, None]
                want = (x[at:at + c] / s).clamp(-448, 448)
                # half a step of e4m3: 2^-4 of the value, 2^-10 among subnormals
                tol = want.abs() * 2.0 ** -4 + 2.0 ** -10 + (0 if slack is None else slack[at:at + c] / s)
                assert ((got.view(torch.float8_e4m3fn).double() - want).abs() <= tol).all()
        else:
            assert torch.equal(gv, v[at:at + c])
            assert ((gk.double() - kr[at:at + c]).abs() <= bound(k, bt.dtype, R)[at:at + c]).all()
        bt.put(bt.k, b, p, bt.rows(before[0], b, p))
        bt.put(bt.v, b, p, bt.rows(before[1], b, p))
    for cache, old in ((bt.k, before[0]), (bt.v, before[1])):   # nothing else of the cache changed
        assert torch.equal(torch.nan_to_num(cache.float(), 9), torch.nan_to_num(old.float(), 9))


def test_more_rows_than_a_launch_has_threads():
    """2^24 rows and more of 32 heads: one workgroup of 256 threads per row would pass 32 bits."""
    T = 2 ** 24 + 1
    bt = Batch([(4, 50)], Hq=16, Hkv=16, seed=52)
    rows = torch.empty(T, 16, 128, dtype=bt.dtype, device="cuda")
    rows[-4:] = new_rows(bt, False)[1]
    ends = torch.tensor([T - 4, T], dtype=torch.int32, device="cuda")
    before = bt.v.clone()
    S.santa_rope_append(None, rows, rows, bt.kv(), bt.shape(), S.chunk_of(ends, T), None, None)
    torch.cuda.synchronize()
    assert torch.equal(bt.k[0, 46:], rows[-4:]) and torch.equal(bt.v[0, 46:], rows[-4:])
    assert torch.equal(bt.v[0, :46], before[0, :46])
    del rows
    torch.cuda.empty_cache()
