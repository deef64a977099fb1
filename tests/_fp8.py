"""What the tests of the cache in 8 bits hold the kernels to: e4m3 by its definition, in 64 bits, and a cache of random keys."""
from __future__ import annotations

import math

import numpy as np
import torch

# every e4m3 code's value: 4 bits of exponent (bias 7), 3 of mantissa, no infinities
_E, _M = np.arange(256) >> 3 & 15, np.arange(256) & 7
VALUES = np.where(_E == 0, _M * 2.0 ** -9, (8 + _M) * 2.0 ** (_E - 10.0)) * np.where(np.arange(256) > 127, -1.0, 1.0)
VALUES[[127, 255]] = np.nan
_POSITIVE = VALUES[:127]  # ascending, as the codes are


def values(codes: torch.Tensor) -> torch.Tensor:
    return torch.from_numpy(VALUES).to(codes.device)[codes.view(torch.uint8).long()]


def codes_of(x: np.ndarray) -> np.ndarray:
    """The code nearest to each x (64 bits, at most 448 or not finite), the even one of two; 0x7f for what is not finite."""
    a = np.abs(x)
    fine = np.isfinite(a)
    a = np.where(fine, a, 0.0)
    hi = np.searchsorted(_POSITIVE, a).clip(0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = _POSITIVE[hi] - a, a - _POSITIVE[lo]
    near = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    near = np.where(_POSITIVE[hi] == a, hi, near)
    return np.where(fine, near + 128 * np.signbit(x), 127).astype(np.uint8)


def least_exponent(top: float) -> int:
    """The least biased exponent with top within 448 of it, at least 1."""
    e = 1
    while top > 448 * 2.0 ** (e - 127):
        e += 1
    return e


class Append:
    """kv_append_fp8 for one of K and V, page by page in 64 bits."""

    def __init__(self, codes, scale, page):
        self.codes, self.scale, self.page = codes.copy(), scale.copy(), page

    def __call__(self, rows, held, table):
        """rows [new, heads, dim] behind `held` keys of a sequence with this row of the block table."""
        at = 0
        while at < len(rows):
            off = (held + at) % self.page
            n = min(self.page - off, len(rows) - at)
            p = table[(held + at) // self.page]
            part = rows[at:at + n]
            for h in range(part.shape[1]):
                x = part[:, h].astype(np.float64)
                b = least_exponent(np.abs(x[np.isfinite(x)]).max(initial=0.0))
                if off:
                    was = int(self.scale[p, h])
                    b = max(b, was)
                    if b > was:
                        old = self.codes[p * self.page:p * self.page + off, h]
                        self.codes[p * self.page:p * self.page + off, h] = codes_of(VALUES[old] * 2.0 ** (was - b))
                self.scale[p, h] = b
                self.codes[p * self.page + off:p * self.page + off + n, h] = codes_of(x * 2.0 ** (127 - b))
            at += n


def random_cache(g, ctxs, hkv, dim, page, spread=2, device="cuda", spare=2):
    """Codes and scales of shuffled pages that hold ctxs[s] keys each, the other rows not numbers; a scale of its own for every
    page and head, within 2^spread of the others'.  Returns a dict."""
    need = [-(-c // page) for c in ctxs]
    pages = sum(need) + spare
    order = torch.randperm(pages, generator=g)
    table = torch.zeros(len(ctxs), max(1, max(need)), dtype=torch.int32)
    there = torch.zeros(pages * page, dtype=torch.bool)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n].to(torch.int32)
        rows = (table[s, :n, None].long() * page + torch.arange(page)).reshape(-1)[:ctxs[s]]
        there[rows] = True
        at += n
    out = dict(table=table.to(device), page=page)
    for name in "kv":
        x = torch.randn(pages * page, hkv, dim, generator=g).clamp(-4, 4) * 100
        x[~there] = math.nan
        out[name] = x.to(torch.float8_e4m3fn).to(device)
        # (values around 1: codes around 100 times 2^-7)
        out[name + "_scale"] = (120 + torch.randint(-spread, spread + 1, (pages, hkv), generator=g)).to(torch.uint8).to(device)
    return out


def keys_of(c, name, s, n):
    """Keys (or values) 0 .. n - 1 of sequence s in 64 bits: [n, heads, dim]."""
    page = c["page"]
    j = torch.arange(n, device=c["k"].device)
    rows = c["table"][s].long()[j // page] * page + j % page
    return values(c[name][rows]) * torch.pow(2.0, c[name + "_scale"].double() - 127)[rows // page][..., None]


def attention(c, q, news, lens, causal, window, scale=0.0):
    """(o, lse, error bound of o, of lse) in 64 bits; news[s] queries of a sequence with lens[s] keys.

    The bounds: o is rounded to bf16 (2^-8 of it); every weight to fp16's 11 bits (2^-11, and 2^-13 for the fp32 numbers around
    it); a score is a sum of up to 256 products in fp32, off by 2^-16 of the sum of their sizes at most, and its weight by as
    much, relatively, in the numerator and in the sum."""
    hq, dim = q.shape[1], q.shape[2]
    hkv = c["k"].shape[1]
    scale = scale or dim ** -0.5
    o = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=q.device)
    bound, lse_bound = torch.zeros_like(o), torch.zeros_like(lse)
    first = 0
    for s, (b, n) in enumerate(zip(news, lens)):
        if b == 0:
            continue
        k, v = keys_of(c, "k", s, n), keys_of(c, "v", s, n)
        x = q[first:first + b].double()
        pos = torch.arange(n - b, n, device=q.device)[:, None]
        j = torch.arange(n, device=q.device)[None]
        seen = (j <= pos) if causal else torch.ones(b, n, dtype=torch.bool, device=q.device)
        if window:
            seen = seen & (j > pos - window)
        for h in range(hq):
            kv = h // (hq // hkv)
            sc = torch.where(seen, scale * x[:, h] @ k[:, kv].nan_to_num().T, -math.inf)
            size = scale * x[:, h].abs().nan_to_num() @ k[:, kv].abs().nan_to_num().T
            z = torch.logsumexp(sc, 1) if n else torch.full((b,), -math.inf, device=q.device, dtype=torch.float64)
            some = torch.isfinite(z)
            p = torch.where(some[:, None], torch.exp(sc - z.masked_fill(~some, 0.0)[:, None]), 0.0)
            o[first:first + b, h] = p @ v[:, kv].nan_to_num()
            lse[first:first + b, h] = z
            off = 2.0 ** -16 * (torch.where(seen, size, 0.0).amax(1) if n else torch.zeros(b, device=q.device, dtype=torch.float64))
            bound[first:first + b, h] = 2.0 ** -8 * o[first:first + b, h].abs() + \
                (2.0 ** -11 + 2.0 ** -13 + 2 * off)[:, None] * (p @ v[:, kv].abs().nan_to_num())
            lse_bound[first:first + b, h] = off + 2.0 ** -20 * (1 + z.masked_fill(~some, 0.0).abs()) + n * 2.0 ** -24
            # what is not a number makes the rows that see it none
            none = (torch.isnan(k[:, kv]).any(1) | torch.isnan(v[:, kv]).any(1))[None] & seen
            none = none.any(1) | (~torch.isfinite(x[:, h]).all(1) & seen.any(1))
            o[first:first + b, h][none] = math.nan
            lse[first:first + b, h][none] = math.nan
        first += b
    return o, lse, bound, lse_bound
