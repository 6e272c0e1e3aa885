"""Inputs and float64 answers for the tests of santa_rope_append, santa_attend_chunk and
santa_decode_window: a batch of new tokens over a cache of any layout, its attention from the
definition, and error bounds derived from the roundings that the kernels make."""

from __future__ import annotations

import math

import torch

from paper_2605_01910_amd import santa as S

D = 128
SCALE = 1.0 / math.sqrt(D)
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}  # half a step, relative to the value


class Batch:
    """lens: (new tokens, context length) per sequence.  The cache's rows at or past a sequence's
    context, unused pages and rows between padded strides hold `filler`."""

    def __init__(self, lens, Hq=8, Hkv=2, dtype=torch.bfloat16, fp8=False, layout="nhd", page=16, pad=0, n=None,
                 seed=0, gap=0, filler=float("nan"), pages=None, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.lens, self.Hq, self.Hkv, self.G, self.dtype, self.fp8 = lens, Hq, Hkv, Hq // Hkv, dtype, fp8
        self.B, self.layout, self.page = len(lens), layout, page
        self.T = sum(c for c, _ in lens) + pad
        self.n = n or max(1, max(L for _, L in lens))
        starts = [0]
        for c, _ in lens:
            starts.append(starts[-1] + c)
        self.starts = starts
        self.q_start = torch.tensor(starts, dtype=torch.int32, device=device)
        self.ctx = torch.tensor([L for _, L in lens], dtype=torch.int32, device=device)
        el = torch.uint8 if fp8 else dtype
        W = D + gap  # row pitch
        fill = 0x7f if fp8 else filler
        if layout == "paged":
            need = [-(-L // page) for _, L in lens]
            N = pages or sum(need) + 4
            perm = torch.randperm(min(N, 4096), generator=g, device=device) + max(0, N - 4096)
            shape = (N, Hkv, page, W)
            self.table = torch.zeros(self.B, max(1, -(-self.n // page)), dtype=torch.int32, device=device)
            self.table[:] = perm[sum(need)]  # a page of fillers
            at = 0
            for b, m in enumerate(need):
                self.table[b, :m] = perm[at:at + m].int()
                at += m
        else:
            shape = (self.B, self.n, Hkv, W) if layout == "nhd" else (self.B, Hkv, self.n, W)
        if pages:  # too large to fill: only the pages in use
            self.k, self.v = (torch.empty(shape, dtype=el, device=device) for _ in range(2))
            self.k[perm], self.v[perm] = fill, fill
        else:
            self.k, self.v = (torch.full(shape, fill, dtype=el, device=device) for _ in range(2))
        self.k, self.v = self.k[..., :D], self.v[..., :D]
        self.k_scale = (0.01 + 0.02 * torch.rand(self.B, Hkv, device=device, generator=g)) if fp8 else None
        self.v_scale = (0.01 + 0.02 * torch.rand(self.B, Hkv, device=device, generator=g)) if fp8 else None
        for b, (_, L) in enumerate(lens):
            for cache in (self.k, self.v):
                x = torch.randn(L, Hkv, D, device=device, generator=g)
                if cache is self.k and L:
                    x[torch.rand(L, generator=g, device=device) < 0.05] *= 3
                x = (x * 60).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) if fp8 else x.to(dtype)
                self.put(cache, b, torch.arange(L, device=device), x)
        self.q = torch.randn(self.T, Hq, D, device=device, generator=g).to(dtype)

    def index(self, b, pos):
        if self.layout == "paged":
            return self.table[b].long()[pos // self.page], pos % self.page
        return torch.full_like(pos, b), pos

    def put(self, cache, b, pos, rows):
        x, y = self.index(b, pos)
        if self.layout == "nhd":
            cache[x, y] = rows
        else:
            cache[x, :, y] = rows

    def rows(self, cache, b, pos):
        """Stored rows [len(pos), Hkv, D] as they are (codes for FP8)."""
        x, y = self.index(b, pos)
        return cache[x, y] if self.layout == "nhd" else cache[x, :, y]

    def values(self, cache, b, L):
        """float64 [L, Hkv, D] of the sequence's first L rows."""
        r = self.rows(cache, b, torch.arange(L, device=cache.device))
        if not self.fp8:
            return r.double()
        scale = self.k_scale if cache is self.k else self.v_scale
        return r.view(torch.float8_e4m3fn).double() * scale[b].double()[:, None]

    def kv(self):
        if self.layout == "paged":
            kv = S.kv_paged(self.k, self.v, self.table, self.ctx, self.n)
        else:
            kv = S.kv_contiguous(self.k, self.v, self.ctx, self.layout)
        if self.fp8:
            S.set_fp8_cache(kv, self.k_scale, self.v_scale)
        return kv

    def shape(self):
        sh = S.shape_of(self.q, self.Hkv)
        sh.batch = self.B
        return sh

    def chunk(self, hint=0):
        return S.chunk_of(self.q_start, self.T, hint)


def attend(bt, window=None, scale=SCALE, hint=0, splits=0, out=None, ws=None, stream=None):
    """santa_attend_chunk on the batch; window: (window, sinks) or None."""
    kv, sh, ch = bt.kv(), bt.shape(), bt.chunk(hint)
    win = S.window_of(*window) if window else None
    if out is None:
        out = torch.full_like(bt.q, 7.0)
    with S.options("auto", splits):
        if ws is None:
            ws = S.alloc_attend_workspace(sh, kv, ch, win)
        S.santa_attend_chunk(bt.q, kv, sh, ch, win, scale, out, ws, stream)
    torch.cuda.synchronize()
    S.check_workspace(ws)
    return out


def answer(bt, window=None, scale=SCALE):
    """(out, bound) in float64: the definition, and how far each element may be off.

    With weights p_j and A = sum p_j |v_j|, an output is off by at most
      2 d A          the weights: every score by d (below), numerator and denominator;
      h (A + |o|)    16-bit operands: a weight's rounding, and the output's (h: half a step);
      (n + 80) u A   n + 80 additions and products in 32 bits, u = 2^-24;
    and a score, in units of the exponent of e, by d = 140 u scale sum |q k| (a sum of 128
    products and the scales) + 2^-20 (the exponential and its argument's rounding)."""
    out = torch.full((bt.T, bt.Hq, D), float("nan"), dtype=torch.float64, device=bt.q.device)
    tol = torch.zeros_like(out)
    u, h = 2.0 ** -24, HALF[bt.dtype] if bt.dtype != torch.float32 else 2.0 ** -24
    for b, (c, L) in enumerate(bt.lens):
        if c == 0:
            continue
        k, v = bt.values(bt.k, b, L), bt.values(bt.v, b, L)
        p = torch.arange(L - c, L, device=k.device)[:, None]
        j = torch.arange(L, device=k.device)[None]
        seen = j <= p
        if window:
            seen = seen & ((j > p - window[0]) | (j < window[1]))
        at = bt.starts[b]
        for hq in range(bt.Hq):
            kv = hq // bt.G
            q = bt.q[at:at + c, hq].double()
            s = (q @ k[:, kv].T * scale).masked_fill(~seen, -math.inf)
            m = s.amax(-1, keepdim=True) if L else torch.full((c, 1), -math.inf, device=k.device).double()
            w = torch.where(seen, torch.exp(s - torch.where(m == -math.inf, 0.0, m)), 0.0)
            w = w / w.sum(-1, keepdim=True).clamp(min=1e-300)
            # by hand: 0 * inf is not part of the definition
            vv = torch.where(torch.isfinite(v[:, kv]), v[:, kv], 0.0)
            o, A = w @ vv, w @ vv.abs()
            for kind in (math.inf, -math.inf, math.nan):
                is_kind = (torch.isnan(v[:, kv]) if kind != kind else v[:, kv] == kind).double()
                hit = (seen.double() @ is_kind) > 0 if L else torch.zeros_like(o, dtype=torch.bool)
                o = torch.where(hit, o + kind, o)
            d = 140 * u * abs(scale) * (q.abs() @ torch.nan_to_num(k[:, kv], 0, 0, 0).abs().T).amax(-1, keepdim=True) \
                if L else torch.zeros(c, 1, device=k.device).double()
            out[at:at + c, hq] = o
            tol[at:at + c, hq] = A * (2 * (d + 2.0 ** -20) + h + (L + 80) * u) + h * torch.nan_to_num(o.abs(), 0, 0, 0)
    return out, tol


def check(bt, got, window=None, scale=SCALE, sentinel=7.0):
    want, tol = answer(bt, window, scale)
    used = bt.starts[-1]
    assert torch.all(got[used:] == sentinel), "rows behind the last sequence were written"
    got, want, tol = got[:used].double(), want[:used], tol[:used]
    odd = ~torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]) and torch.isfinite(got[~odd]).all()
    over = ((got - want).abs() - tol)[~odd]
    assert over.numel() == 0 or over.max() <= 0, f"off by {over.max().item():.3g} more than the bound"
