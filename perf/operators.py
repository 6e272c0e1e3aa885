"""Performance cases of the operators around the decode step: rotary positions with the
store into the KV cache, attention of a chunk of new tokens over the cache, and attention
with a sliding window and sinks.

A case is one call for one attention layer.  The head layouts, cache layouts, element types
and context lengths are those of the repository's configurations (``workload/gen.py``) and
decode cases: 32 query heads over 8 KV heads with head_dim 128 at up to 64k keys, groups of 1
to 8, contiguous and 16-token-page caches, bfloat16, float32 and FP8 E4M3.

Keys of a case:

    op        rope | chunk | window
    B, Hq, Hkv
    n_lo, n   context lengths after the call's tokens, one per sequence, in [n_lo, n]
    c_lo, c   new tokens per sequence, in [c_lo, c]
    pad       rows behind the last sequence (a batch padded for a captured graph)
    dtype     bf16 | f32 (rows, outputs and, without fp8, the cache)
    kv        "" | "fp8" (E4M3 codes with per-(sequence, KV head) scales)
    layout    nhd | hnd | paged (16-token pages, shuffled table)
    window, sinks   window: keys a token sees besides the first `sinks` (0: all of them)
    rotary, interleaved, scaling    rope: rotated features, pair layout, long-context scaling
    fused     rope: q, k and v are parts of one projection's rows

``own`` False computes the plain form: elementary operations in 32 bits (angles in 64).
"""

from __future__ import annotations

import math
import random

import torch

own = False

D = 128
PAGE = 16
SCALE = 1.0 / math.sqrt(D)
THETA, FACTOR, ORIGINAL = 500000.0, 8.0, 8192
BAND_LOW, BAND_HIGH = 1.0, 4.0       # scaling "bands"
TURNS_SLOW, TURNS_FAST = 1.0, 32.0   # scaling "ramp"


def _case(op, B, n, c=1, n_lo=None, c_lo=None, Hq=32, Hkv=8, dtype="bf16", kv="", layout="nhd", pad=0,
          window=0, sinks=0, rotary=D, interleaved=False, scaling="none", fused=False):
    return {"op": op, "B": B, "Hq": Hq, "Hkv": Hkv, "n_lo": n if n_lo is None else n_lo, "n": n,
            "c_lo": c if c_lo is None else c_lo, "c": c, "pad": pad, "dtype": dtype, "kv": kv,
            "layout": layout, "window": window, "sinks": sinks, "rotary": rotary,
            "interleaved": interleaved, "scaling": scaling, "fused": fused}


def listed():
    named = {
        # one user's next token: the smallest call, on the critical path of every layer
        "rope_b1_token": _case("rope", 1, 32768),
        # a serving batch's next tokens into an FP8 paged cache, long-context frequencies
        "rope_b64_fp8_paged": _case("rope", 64, 16384, n_lo=1024, kv="fp8", layout="paged",
                                    interleaved=True, scaling="bands"),
        # three prompts arrive together, straight from the fused projection
        "rope_prompts_paged": _case("rope", 3, 8192, 8192, n_lo=2000, c_lo=2000, layout="paged",
                                    scaling="ramp", fused=True),
        # numerics and bring-up: one float32 head, an odd chunk
        "chunk_f32_one_head": _case("chunk", 1, 1024, 77, Hq=1, Hkv=1, dtype="f32"),
        # verification of five drafted tokens for eight users on medium contexts
        "chunk_b8_5_tokens": _case("chunk", 8, 12345, 5, n_lo=9000, layout="paged"),
        # one step of a chunked prefill near the end of a long prompt
        "chunk_512_at_32k": _case("chunk", 1, 32768, 512, layout="paged"),
        # a mixed batch: prompts' chunks beside single tokens, groups of eight, FP8, padded
        "chunk_mixed_fp8_paged": _case("chunk", 12, 4000, 700, n_lo=1, c_lo=1, Hq=64, kv="fp8",
                                       layout="paged", pad=37),
        # a whole prompt at once: the largest
        "chunk_prompt_8k": _case("chunk", 1, 8192, 8192),
        # a windowed layer in one user's decode step
        "window_b1_32k": _case("window", 1, 32768, window=1024, sinks=4),
        # the same layer for a ragged serving batch, wider window
        "window_b64_paged": _case("window", 64, 65536, n_lo=4096, layout="paged", window=4096, sinks=4),
        # groups of eight over an FP8 head-major cache
        "window_b16_g8_fp8": _case("window", 16, 20011, n_lo=700, Hq=64, kv="fp8", layout="hnd",
                                   window=2048, sinks=16),
        # a chunk of a long prompt through a windowed layer
        "window_chunk_2k": _case("window", 1, 16384, 2048, layout="paged", window=1024, sinks=4),
    }
    return [dict(c, name=k) for k, c in named.items()]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """Another call of the same ranges: 1 to 64 sequences of 64 to 65536 keys, 1 to 8192 new tokens
    each, groups of 1 to 8, every cache layout and element type, windows of 64 to 8192 keys."""
    op = rng.choice(["rope", "chunk", "window"])
    dtype, kv = rng.choice([("bf16", ""), ("bf16", ""), ("bf16", ""), ("f32", ""), ("bf16", "fp8")])
    layout = rng.choice(["nhd", "hnd", "paged", "paged"])
    Hkv = rng.choice([1, 2, 4, 8, 8])
    G = rng.choice([1, 2, 4, 4, 4, 8])
    n = _log_int(rng, 64, 65536 if dtype == "bf16" else 8192)    # float32 is the numerics type
    c = 1 if rng.random() < 0.4 else _log_int(rng, 2, min(n, 8192))
    B = _log_int(rng, 1, 64)
    window = sinks = 0
    if op == "window":
        window, sinks = _log_int(rng, 64, 8192), rng.choice([0, 1, 4, 16, 64])
    # at most the cost of the largest listed cases: cache rows, new rows, scores of the padded batch
    rows = 4_000_000 if op == "rope" else 16_000_000
    B = max(1, min(B, rows // (n * Hkv * (2 if dtype == "f32" else 1)), 20000 // c))
    keys = min(n, window + sinks + c - 1) if window else n
    if op != "rope":
        c = max(1, min(c, 2_000_000_000 // (B * G * Hkv * keys)))
    n_lo = n if rng.random() < 0.3 else max(c, int(n * rng.uniform(0.05, 0.9)))
    c_lo = c if rng.random() < 0.5 else max(1, int(c * rng.uniform(0.05, 0.9)))
    case = _case(op, B, n, c, min(n_lo, n), c_lo, G * Hkv, Hkv, dtype, kv, layout,
                 pad=rng.choice([0, 0, 5, 37]), window=window, sinks=sinks)
    if op == "rope":
        case["rotary"] = rng.choice([128, 128, 64, 32, 96])
        case["interleaved"] = rng.random() < 0.5
        case["scaling"] = rng.choice(["none", "linear", "base", "bands", "ramp"])
        case["fused"] = rng.random() < 0.5
    return case


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _lengths(case):
    """(new tokens, context length) of every sequence: a property of the case."""
    r = random.Random(1000003 * case["n"] + 1009 * case["c"] + 31 * case["n_lo"] + case["B"])
    out = []
    for _ in range(case["B"]):
        c = r.randint(case["c_lo"], case["c"])
        out.append((c, max(c, r.randint(case["n_lo"], case["n"]))))
    return out


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    B, Hq, Hkv, n = case["B"], case["Hq"], case["Hkv"], case["n"]
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    lens = _lengths(case)
    T = sum(c for c, _ in lens) + case["pad"]

    def normal(*shape):
        return torch.randn(*shape, device="cuda", dtype=dt, generator=g)

    s = {"case": case, "T": T}
    starts = [0]
    for c, _ in lens:
        starts.append(starts[-1] + c)
    s["q_start"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    s["ctx"] = torch.tensor([L for _, L in lens], dtype=torch.int32, device="cuda")
    # the cache: Gaussian rows, three in a hundred keys with larger norms
    if case["layout"] == "paged":
        need = [-(-L // PAGE) for _, L in lens]
        pages = sum(need) + 3
        order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
        s["table"] = torch.zeros(B, -(-n // PAGE), dtype=torch.int32, device="cuda")
        at = 0
        for b, m in enumerate(need):
            s["table"][b, :m] = order[at:at + m]
            at += m
        shape = (pages, Hkv, PAGE, D)
    else:
        shape = (B, n, Hkv, D) if case["layout"] == "nhd" else (B, Hkv, n, D)
    k, v = normal(*shape), normal(*shape)
    k *= torch.where(torch.rand(*shape[:3], 1, device="cuda", generator=g) < 0.03, 3.0, 1.0).to(dt)
    if case["kv"] == "fp8":
        s["k_scale"] = 0.01 + 0.01 * torch.rand(B, Hkv, device="cuda", generator=g)
        s["v_scale"] = 0.01 + 0.01 * torch.rand(B, Hkv, device="cuda", generator=g)
        k = (k.float() * 60).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        v = (v.float() * 60).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    s["k"], s["v"] = k, v
    s["out"] = torch.zeros(T, Hq, D, dtype=dt, device="cuda")
    if case["op"] == "rope":
        if case["fused"]:
            rows = normal(T, (Hq + 2 * Hkv) * D)
            parts = rows.split([Hq * D, Hkv * D, Hkv * D], dim=1)
            s["q"], s["k_new"], s["v_new"] = (p.unflatten(1, (-1, D)) for p in parts)
        else:
            s["q"], s["k_new"], s["v_new"] = normal(T, Hq, D), normal(T, Hkv, D), normal(T, Hkv, D)
    else:
        s["q"] = normal(T, Hq, D)
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a serving program keeps beside its buffers: descriptors, the rotary plan, a workspace."""
    from paper_2605_01910_amd import santa as S

    case = s["case"]
    if case["layout"] == "paged":
        kv = S.kv_paged(s["k"], s["v"], s["table"], s["ctx"], case["n"])
    else:
        kv = S.kv_contiguous(s["k"], s["v"], s["ctx"], case["layout"])
    if case["kv"] == "fp8":
        S.set_fp8_cache(kv, s["k_scale"], s["v_scale"])
    s["kv"], s["shape"] = kv, S.shape_of(s["q"], case["Hkv"])
    s["shape"].batch = case["B"]
    one = case["c"] == 1 and case["pad"] == 0
    s["chunk"] = S.chunk_of(None if one else s["q_start"], s["T"], case["c"])
    s["one"] = one
    if case["op"] == "rope":
        s["rope"] = S.rope_plan(case["rotary"], case["interleaved"], THETA, case["scaling"], FACTOR,
                                ORIGINAL, BAND_LOW if case["scaling"] == "bands" else TURNS_SLOW,
                                BAND_HIGH if case["scaling"] == "bands" else TURNS_FAST)
    else:
        s["win"] = S.window_of(case["window"], case["sinks"]) if case["window"] else None
        s["ws"] = S.alloc_attend_workspace(s["shape"], kv, s["chunk"], s["win"])


# ---------------------------------------------------------------------------
# the calls
# ---------------------------------------------------------------------------

def run(s):
    case = s["case"]
    if own:
        from paper_2605_01910_amd import santa as S

        if case["op"] == "rope":
            S.santa_rope_append(s["q"], s["k_new"], s["v_new"], s["kv"], s["shape"], s["chunk"], s["rope"],
                                s["out"])
        elif case["op"] == "window" and s["one"]:
            S.santa_decode_window(s["q"], s["kv"], s["shape"], s["win"], SCALE, s["out"], s["ws"])
        else:
            S.santa_attend_chunk(s["q"], s["kv"], s["shape"], s["chunk"], s["win"], SCALE, s["out"], s["ws"])
    elif case["op"] == "rope":
        _plain_rope(s)
    else:
        _plain_attend(s)
    if case["op"] != "rope":
        return s["out"]
    if case["kv"] == "fp8":
        return s["out"], s["k"].view(torch.float8_e4m3fn), s["v"].view(torch.float8_e4m3fn)
    return s["out"], s["k"], s["v"]


def _tokens(s):
    """Sequence, index in the sequence's chunk and cache position of every row, and whether it holds a
    token (rows behind the last sequence do not)."""
    t = torch.arange(s["T"], device="cuda")
    starts = s["q_start"].long()
    b = torch.searchsorted(starts[1:], t, right=True)
    real = b < s["case"]["B"]
    b = b.clamp(max=s["case"]["B"] - 1)
    i = t - starts[b]
    return b, i, s["ctx"].long()[b] - (starts[b + 1] - starts[b]) + i, real


def _rows(s, b, pos):
    """Index of cache rows: tensors that select [..., Hkv, D] at sequence b, position pos."""
    if s["case"]["layout"] == "paged":
        page = s["table"].long()[b, (pos // PAGE).clamp(0, s["table"].shape[1] - 1)]
        return page, pos % PAGE
    return b, pos


def _gather(s, cache, b, pos):
    x, y = _rows(s, b, pos)
    if s["case"]["layout"] == "nhd":
        return cache[x, y]
    return cache[x, :, y]


def _frequencies(case):
    """Radians per position of every pair, float64."""
    R = case["rotary"]
    i = torch.arange(R // 2, dtype=torch.float64, device="cuda")
    theta = THETA * FACTOR ** (R / (R - 2)) if case["scaling"] == "base" else THETA
    f = theta ** (-2 * i / R)
    if case["scaling"] == "linear":
        f = f / FACTOR
    elif case["scaling"] == "bands":   # by the wavelength's share of the original context
        turns = ORIGINAL * f / (2 * math.pi)
        mix = ((turns - BAND_LOW) / (BAND_HIGH - BAND_LOW)).clamp(0, 1)
        f = f / FACTOR * (1 - mix) + f * mix
    elif case["scaling"] == "ramp":    # a linear ramp between the pairs of two numbers of turns
        at = [R * math.log(ORIGINAL / (2 * math.pi * t)) / (2 * math.log(THETA)) for t in (TURNS_FAST, TURNS_SLOW)]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), R - 1)
        mix = ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        f = f / FACTOR * mix + f * (1 - mix)
    return f


def _gain(case):
    return 0.1 * math.log(FACTOR) + 1 if case["scaling"] == "ramp" else 1.0


def _turn(x, cos, sin, case):
    """x [T, H, D] float32 with its first `rotary` features rotated by pairs."""
    R = case["rotary"]
    if case["interleaved"]:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
    else:
        a, b = x[..., :R // 2], x[..., R // 2:R]
    ya, yb = a * cos - b * sin, b * cos + a * sin
    y = torch.stack([ya, yb], -1).flatten(-2) if case["interleaved"] else torch.cat([ya, yb], -1)
    return torch.cat([y, x[..., R:]], -1)


def _plain_rope(s):
    case = s["case"]
    b, i, pos, real = _tokens(s)
    angle = pos.double()[:, None] * _frequencies(case)
    cos = (angle.cos() * _gain(case)).float()[:, None]
    sin = (angle.sin() * _gain(case)).float()[:, None]
    q = _turn(s["q"].float(), cos, sin, case)
    s["out"].copy_(torch.where(real[:, None, None], q.to(s["out"].dtype), s["out"]))
    # rows behind the last sequence are dropped: their number is the caller's own
    T = s["T"] - case["pad"]
    x, y = _rows(s, b[:T], pos[:T])
    for cache, new, scale in ((s["k"], _turn(s["k_new"].float(), cos, sin, case)[:T], "k_scale"),
                              (s["v"], s["v_new"].float()[:T], "v_scale")):
        if case["kv"] == "fp8":
            new = (new / s[scale][b[:T]][..., None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        else:
            new = new.to(cache.dtype)
        if case["layout"] == "nhd":
            cache[x, y] = new
        else:
            cache[x, :, y] = new


def _plain_attend(s):
    case = s["case"]
    B, Hq, Hkv, n, c = case["B"], case["Hq"], case["Hkv"], case["n"], case["c"]
    G = Hq // Hkv
    ctx, starts = s["ctx"].long(), s["q_start"].long()
    count = starts[1:] - starts[:-1]
    # the keys that any token of the sequence sees: the sinks, then the union of the windows
    if case["window"] and case["window"] + case["sinks"] + c - 1 < n:
        first = (ctx - count - case["window"] + 1).clamp(min=case["sinks"])
        v = torch.arange(case["sinks"] + case["window"] + c - 1, device="cuda")
        j = torch.where(v < case["sinks"], v, first[:, None] + v - case["sinks"])
    else:
        j = torch.arange(n, device="cuda").expand(B, n)
    held = j < ctx[:, None]
    at = torch.where(held, j, 0)
    seq = torch.arange(B, device="cuda")[:, None].expand_as(at)
    k, v = _gather(s, s["k"], seq, at), _gather(s, s["v"], seq, at)       # [B, keys, Hkv, D]
    if case["kv"] == "fp8":
        k, v = k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn)
    k, v = k.float(), v.float()
    if case["kv"] == "fp8":
        k = k * s["k_scale"][:, None, :, None]
        v = v * s["v_scale"][:, None, :, None]
    v = v * held[..., None, None]
    i = torch.arange(c, device="cuda")
    tok = (starts[:-1, None] + i).clamp(max=s["T"] - 1)
    q = s["q"].float()[tok].view(B, c, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * c, D)
    p = ctx[:, None] - count[:, None] + i                                   # [B, c]
    seen = (j[:, None] <= p[..., None]) & held[:, None]
    if case["window"]:
        seen &= (j[:, None] > p[..., None] - case["window"]) | (j[:, None] < case["sinks"])
    x = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()) * SCALE          # [B, Hkv, G*c, keys]
    x = x.view(B, Hkv, G, c, -1).masked_fill_(~seen[:, None, None], -math.inf)
    x = torch.exp(x - x.amax(-1, keepdim=True).clamp(min=-1e30))
    y = torch.matmul(x.view(B, Hkv, G * c, -1), v.permute(0, 2, 1, 3).contiguous()).view(B, Hkv, G, c, D)
    y = y / x.sum(-1, keepdim=True).clamp(min=1e-30)
    b, i, _, real = _tokens(s)
    y = y.permute(0, 3, 1, 2, 4).reshape(B, c, Hq, D)[b, i.clamp(max=c - 1)]
    s["out"].copy_(torch.where(real[:, None, None], y.to(s["out"].dtype), s["out"]))


# ---------------------------------------------------------------------------
# what a call cannot do without, and its answer in 64 bits
# ---------------------------------------------------------------------------

def work(case):
    lens = _lengths(case)
    esz = 2 if case["dtype"] == "bf16" else 4
    ksz = 1 if case["kv"] == "fp8" else esz
    tokens = sum(c for c, _ in lens)
    if case["op"] == "rope":
        rows = 2 * case["Hq"] + 2 * case["Hkv"]
        return {"bytes": tokens * D * (rows * esz + 2 * case["Hkv"] * ksz),
                "flops": 3 * tokens * (case["Hq"] + case["Hkv"]) * case["rotary"]}
    keys = pairs = 0
    for c, L in lens:
        w, sk = case["window"] or L, case["sinks"]
        first = max(0, L - c - w + 1)                 # the first key of the union of the windows
        keys += L - first + min(sk, first)
        for p in range(L - c, L):
            lo = max(0, p - w + 1)
            pairs += p + 1 - lo + min(sk, lo)
    return {"bytes": 2 * keys * case["Hkv"] * D * ksz + 2 * tokens * case["Hq"] * D * esz,
            "flops": 4 * D * case["Hq"] * pairs}


def exact(case, seed):
    """The definitions, sequence by sequence, in float64."""
    s = prepare(case, seed)
    return _exact_rope(s) if case["op"] == "rope" else _exact_attend(s)


def _sequence_rows(s, b, L):
    """Index of the sequence's L cache rows, for either pool or contiguous caches."""
    p = torch.arange(L, device="cuda")
    if s["case"]["layout"] == "paged":
        return s["table"][b].long()[p // PAGE], p % PAGE
    return torch.full_like(p, b), p


def _exact_rope(s):
    case = s["case"]
    R, nhd = case["rotary"], case["layout"] == "nhd"
    fp8 = case["kv"] == "fp8"
    out = s["out"].double()
    K, V = ((x.view(torch.float8_e4m3fn) if fp8 else x).double() for x in (s["k"], s["v"]))
    freq = []
    for i in range(R // 2):
        theta = THETA * math.pow(FACTOR, R / (R - 2)) if case["scaling"] == "base" else THETA
        f = 1.0 / math.pow(theta, 2 * i / R)
        if case["scaling"] == "linear":
            f /= FACTOR
        if case["scaling"] == "bands":
            wave = 2 * math.pi / f
            if wave > ORIGINAL / BAND_LOW:
                f /= FACTOR
            elif wave > ORIGINAL / BAND_HIGH:
                mix = (ORIGINAL / wave - BAND_LOW) / (BAND_HIGH - BAND_LOW)
                f = (1 - mix) * f / FACTOR + mix * f
        if case["scaling"] == "ramp":
            pair = lambda turns: R / 2 * math.log(ORIGINAL / (turns * 2 * math.pi)) / math.log(THETA)  # noqa: E731
            lo, hi = max(0, math.floor(pair(TURNS_FAST))), min(R - 1, math.ceil(pair(TURNS_SLOW)))
            mix = min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001)))
            f = mix * f / FACTOR + (1 - mix) * f
        freq.append(f)
    freq = torch.tensor(freq, dtype=torch.float64, device="cuda")
    first = torch.arange(R // 2, device="cuda") * (2 if case["interleaved"] else 1)
    second = first + (1 if case["interleaved"] else R // 2)
    gain = 1 + 0.1 * math.log(FACTOR) if case["scaling"] == "ramp" else 1.0

    def rotated(x, pos):
        z = torch.polar(torch.full((), gain, dtype=torch.float64, device="cuda"), pos[:, None] * freq)[:, None]
        w = torch.complex(x[..., first], x[..., second]) * z
        y = x.clone()
        y[..., first], y[..., second] = w.real, w.imag
        return y

    at = 0
    for b, (c, L) in enumerate(_lengths(case)):
        pos = torch.arange(L - c, L, device="cuda", dtype=torch.float64)
        out[at:at + c] = rotated(s["q"][at:at + c].double(), pos)
        x, y = (r[L - c:] for r in _sequence_rows(s, b, L))
        for cache, new, scale in ((K, rotated(s["k_new"][at:at + c].double(), pos), "k_scale"),
                                  (V, s["v_new"][at:at + c].double(), "v_scale")):
            if fp8:
                new = (new / s[scale][b].double()[:, None]).clamp(-448, 448)
            if nhd:
                cache[x, y] = new
            else:
                cache[x, :, y] = new
        at += c
    return out, K, V


def _exact_attend(s):
    case = s["case"]
    G = case["Hq"] // case["Hkv"]
    fp8 = case["kv"] == "fp8"
    out = s["out"].double()
    at = 0
    for b, (c, L) in enumerate(_lengths(case)):
        x, y = _sequence_rows(s, b, L)
        p = torch.arange(L - c, L, device="cuda")[:, None]
        j = torch.arange(L, device="cuda")[None]
        hidden = j > p
        if case["window"]:
            hidden |= (j <= p - case["window"]) & (j >= case["sinks"])
        for h in range(case["Hkv"]):
            kv = []
            for cache, scale in ((s["k"], "k_scale"), (s["v"], "v_scale")):
                rows = cache[x, y, h] if case["layout"] == "nhd" else cache[x, h, y]
                kv.append(rows.view(torch.float8_e4m3fn).double() * s[scale][b, h].double() if fp8
                          else rows.double())
            q = s["q"][at:at + c, h * G:(h + 1) * G].double()
            for g in range(G):
                w = (q[:, g] @ kv[0].T * SCALE).masked_fill(hidden, -math.inf).softmax(-1)
                out[at:at + c, h * G + g] = w @ kv[1]
        at += c
    return out
