"""Host side of santa_rope_append, santa_attend_chunk and santa_decode_window: what they refuse
before any launch, the workspace size, and the rotary plan (no GPU)."""

import ctypes
import math

import pytest

from paper_2605_01910_amd import santa as S

INV, UNS, WS = S.SANTA_ERR_INVALID_ARG, S.SANTA_ERR_UNSUPPORTED, S.SANTA_ERR_WORKSPACE
ref = ctypes.byref


def shape(B=2, Hq=8, Hkv=2, d=128, dtype=0):
    return S.santa_shape_t(B, Hq, Hkv, d, dtype)


def kv(n=4096, **kw):
    x = S.santa_kv_t(16, 16, n * 256, 256, 128, None, None, 0, 0, n)
    for k, v in kw.items():
        setattr(x, k, v)
    return x


def chunk(tokens=10, q_start=16, most=0):
    return S.santa_chunk_t(q_start, tokens, most)


def window(w=64, s=4):
    return S.santa_window_t(w, s)


def attend(sh=None, kv_=None, ch=None, win=None, q=16, out=16, ws=256, n=1 << 40, scale=0.1):
    return S.load().santa_attend_chunk(q, ref(kv_ or kv()), ref(sh or shape()), ref(ch or chunk()),
                                       None if win is None else ref(win), scale, out, ws, n, None)


@pytest.mark.parametrize("kw,status", [
    (dict(sh=shape(d=64)), UNS), (dict(sh=shape(Hq=6, Hkv=2)), UNS), (dict(sh=shape(B=0)), INV),
    (dict(sh=shape(dtype=3)), INV), (dict(kv_=kv(n_k=0)), INV), (dict(kv_=kv(k=None)), INV),
    (dict(kv_=kv(k=8)), UNS), (dict(kv_=kv(stride_n=129)), UNS), (dict(kv_=kv(stride_b=-8)), INV),
    (dict(kv_=kv(kv_dtype=1)), INV), (dict(kv_=kv(kv_dtype=1, k_scale=16, v_scale=16), sh=shape(dtype=1)), UNS),
    (dict(kv_=kv(k_new=16, v_new=16)), UNS), (dict(kv_=kv(block_table=16, page_size=12, max_pages=999)), UNS),
    (dict(kv_=kv(block_table=16, page_size=16, max_pages=9)), INV),
    (dict(ch=chunk(0)), INV), (dict(ch=chunk(-1)), INV), (dict(ch=chunk(most=-1)), INV),
    (dict(ch=chunk(3, None)), INV), (dict(win=window(0)), INV), (dict(win=window(5, -1)), INV),
    (dict(q=None), INV), (dict(out=None), INV), (dict(q=8), UNS), (dict(out=8), UNS),
    (dict(scale=float("nan")), INV), (dict(scale=float("inf")), INV),
    (dict(ws=None), WS), (dict(ws=64), WS), (dict(n=1000), WS),
    (dict(sh=shape(B=2 ** 30, Hq=8, Hkv=8), ch=chunk(2 ** 31 - 1)), UNS),
])
def test_attend_refuses(kw, status):
    assert attend(**kw) == status
    assert S.load().santa_last_error()


def test_window_call_needs_a_window():
    st = S.load().santa_decode_window(16, ref(kv()), ref(shape()), None, 0.1, 16, 256, 1 << 40, None)
    assert st == INV


def test_workspace_size():
    L = S.load()

    def size(sh=None, kv_=None, ch=None, win=None):
        return L.santa_attend_workspace_size(ref(sh or shape()), ref(kv_ or kv()), None if ch is None else ref(ch),
                                             None if win is None else ref(win))

    assert size() > 0 and size(ch=chunk(), win=window()) > 0
    assert size(sh=shape(d=64)) == 0 and size(ch=chunk(0)) == 0 and size(win=window(0)) == 0
    assert size(kv_=kv(n_k=0)) == 0 and L.santa_attend_workspace_size(ref(shape()), None, None, None) == 0
    # a long context over few tokens is split, and a split call needs room for its parts
    assert size(kv_=kv(n=65536)) > size(kv_=kv(n=64))
    with S.options("auto", 1):
        assert size(kv_=kv(n=65536)) == size(kv_=kv(n=64))


def rope_append(rows=None, kv_=None, sh=None, ch=None, rope="plan", q_out=16):
    r = S.santa_rows_t(16, 16, 16, 8 * 128, 256, 256, None)
    for k, v in (rows or {}).items():
        setattr(r, k, v)
    plan = S.rope_plan() if rope == "plan" else rope
    return S.load().santa_rope_append(ref(r), ref(kv_ or kv()), ref(sh or shape()), ref(ch or chunk()),
                                      None if plan is None else ref(plan), q_out, None)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=dict(k=None)), INV), (dict(rows=dict(v=None)), INV), (dict(rows=dict(q=None)), INV),
    (dict(q_out=None), INV), (dict(rope=None), INV), (dict(rows=dict(k=8)), UNS), (dict(rows=dict(q=8)), UNS),
    (dict(q_out=8), UNS), (dict(rows=dict(k_stride=128)), INV), (dict(rows=dict(v_stride=260)), UNS),
    (dict(rows=dict(q_stride=8 * 128 + 8)), INV), (dict(rope=S.santa_rope_t()), INV),
    (dict(sh=shape(d=64)), UNS), (dict(ch=chunk(0)), INV), (dict(ch=chunk(3, None)), INV),
    (dict(kv_=kv(k_new=16, v_new=16)), INV), (dict(kv_=kv(kv_dtype=1)), INV), (dict(kv_=kv(v=None)), INV),
    (dict(kv_=kv(block_table=16, page_size=3, max_pages=9)), UNS),
])
def test_rope_append_refuses(kw, status):
    # (q_out is 16, the same address as q: allowed while q is contiguous)
    assert rope_append(**kw) == status
    assert S.load().santa_last_error()


@pytest.mark.parametrize("kw", [
    dict(rotary_dim=0), dict(rotary_dim=24), dict(rotary_dim=144), dict(theta=1.0), dict(theta=float("nan")),
    dict(theta=float("inf")), dict(scaling="linear", factor=0.0), dict(scaling="base", factor=-2.0),
    dict(scaling="bands", factor=8.0), dict(scaling="bands", factor=8.0, original_len=8192, low=4.0, high=4.0),
    dict(scaling="ramp", factor=8.0, original_len=8192, low=0.0), dict(gain=float("nan")),
    dict(scaling="ramp", factor=8.0, original_len=8192, low=1.0, high=float("inf")),
])
def test_rope_plan_refuses(kw):
    with pytest.raises(S.SantaError):
        S.rope_plan(**kw)


def test_rope_plan_names_scalings():
    with pytest.raises(ValueError):
        S.rope_plan(scaling="other")


@pytest.mark.parametrize("R", [16, 32, 96, 128])
@pytest.mark.parametrize("scaling", ["none", "linear", "base", "bands", "ramp"])
def test_rope_plan_frequencies(R, scaling):
    """step = 2^64 frac(f_i / 2 pi) from the definition, within the double's own rounding."""
    theta, factor, N, lo, hi = 500000.0, 8.0, 8192.0, 1.0, 4.0
    plan = S.rope_plan(R, True, theta, scaling, factor, N, lo, hi)
    assert plan.rotary_dim == R and plan.interleaved == 1
    gain = 0.1 * math.log(8) + 1 if scaling == "ramp" else 1.0
    assert plan.gain == pytest.approx(gain, rel=2 ** -23)
    for i in range(R // 2):
        f = theta ** (-2 * i / R)
        if scaling == "linear":
            f /= factor
        elif scaling == "base":
            f = (theta * factor ** (R / (R - 2))) ** (-2 * i / R)
        elif scaling == "bands":
            turns = N * f / (2 * math.pi)
            s = (turns - lo) / (hi - lo)
            f = f if turns >= hi else f / factor if turns <= lo else (1 - s) * f / factor + s * f
        elif scaling == "ramp":
            at = lambda t: R * math.log(N / (2 * math.pi * t)) / (2 * math.log(theta))  # noqa: E731
            a, b = max(0, math.floor(at(hi))), min(R - 1, math.ceil(at(lo)))
            m = min(1, max(0, (i - a) / max(b - a, 0.001)))
            f = f / factor * m + f * (1 - m)
        # both sides take a power, a logarithm and a few products in doubles
        assert plan.step[i] / 2.0 ** 64 == pytest.approx(f / (2 * math.pi) % 1.0, rel=2e-14)
    assert all(plan.step[i] == 0 for i in range(R // 2, 64))


def test_rope_plan_gain_is_kept():
    assert S.rope_plan(gain=0.5).gain == 0.5
    assert S.rope_plan(scaling="ramp", factor=0.5, original_len=4096, low=1, high=32).gain == 1.0
