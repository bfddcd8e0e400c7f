"""Pages of 8 bits for the tests: e4m3 numbers from their definition, insertion slot by slot, packed data over such a cache."""
import math

import numpy as np
import torch

from paper_2406_10774_amd import binding as Q
from packed_util import D, Packed


def value_of(code):
    """1 sign, 4 exponent bits (bias 7), 3 mantissa bits; no infinities, all ones is NaN."""
    sign, exponent, mantissa = -1.0 if code & 128 else 1.0, (code >> 3) & 15, code & 7
    if exponent == 15 and mantissa == 7:
        return math.nan
    return sign * (math.ldexp(mantissa, -9) if exponent == 0 else math.ldexp(8 + mantissa, exponent - 10))


VALUES = np.array([value_of(c) for c in range(256)])
MAGNITUDES = VALUES[:127]                                       # ascending, codes 0 to 126


def nearest(x):
    """Codes of float64 numbers of magnitude up to 448: the nearest, ties to the even code; the sign of zero stays."""
    a = np.abs(x)
    hi = np.searchsorted(MAGNITUDES, a).clip(0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = MAGNITUDES[hi] - a, a - MAGNITUDES[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def exponent_for(most):
    e = -15
    while most > math.ldexp(448.0, e):
        e += 1
    return e


class Pages:
    """One pool (keys or values) as the header defines it: codes [N][Hkv][S][D], exponents [N][Hkv]."""

    def __init__(self, codes, scales):
        self.codes, self.e = codes.copy(), np.log2(scales).astype(int)

    def insert(self, page, head, first, x):
        """Tokens x [n][D] (float64 of fp16 numbers) from slot `first` on, in one call."""
        x = np.clip(x, -61440.0, 61440.0)
        e, old = exponent_for(np.abs(x).max()), int(self.e[page, head])
        if first > 0:
            e = max(e, old)
            if e != old:
                held = self.codes[page, head, :first]
                self.codes[page, head, :first] = nearest(VALUES[held] * 2.0 ** (old - e))
        self.codes[page, head, first:first + len(x)] = nearest(x * 2.0 ** -e)
        self.e[page, head] = e


def rounded(x):
    """Pages [N][Hkv][S][D] of fp16 numbers (NaN: no token) as codes and scales; slots without a token become NaN codes."""
    held = ~torch.isnan(x)
    most = torch.where(held, x, 0.0).abs().amax((2, 3)).double().clamp(max=61440.0)
    e = torch.ceil(torch.log2(most.clamp(min=2.0 ** -30) / 448.0)).clamp(min=-15)
    scale = torch.exp2(e)
    codes = (torch.where(held, x, 0.0).double().clamp(-61440.0, 61440.0) / scale[:, :, None, None]).float().to(torch.float8_e4m3fn)
    return torch.where(held, codes.view(torch.uint8), 0x7f).contiguous(), scale.float()


class Packed8(Packed):
    """Packed over a cache of 8 bits; the scales of pages without a token are NaN."""

    def __init__(self, *args, **kw):
        super().__init__(*args, **kw)
        nobody = torch.isnan(self.k_pool).all(3).all(2)
        k, ks = rounded(self.k_pool)
        v, vs = rounded(self.v_pool)
        self.scales = torch.stack([ks, vs], -1)
        self.scales[nobody] = math.nan
        self.k_pool, self.v_pool = k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn)
        self.describe()

    def describe(self, flags=0):
        self.cache = Q.Cache(self.k_pool, self.v_pool, self.meta, self.table, self.seq_lens, flags=flags, num_heads=self.H,
                             scales=self.scales)

    def cached(self, b, h):
        t = torch.arange(self.lens[b], device=self.dev)
        phys = self.table[b].long()[t // self.S]
        values = torch.from_numpy(VALUES).to(self.dev)
        return tuple(values[pool.view(torch.uint8)[phys, h, t % self.S].long()] * self.scales[phys, h, i].double()[:, None]
                     for i, pool in enumerate((self.k_pool, self.v_pool)))


def turned(x, table, position, interleaved):
    """The rotation as the header defines it, on the CPU: fp32 products and sums one by one, fp16 results."""
    x, table, position = x.cpu(), table.cpu(), position.cpu().long()
    rotary = table.shape[1]
    there = (position >= 0) & (position < table.shape[0])
    row = torch.where(there[:, None], table[position.clamp(0, table.shape[0] - 1)], math.nan)[:, None]
    c, s = row[..., :rotary // 2], row[..., rotary // 2:]
    r = x.float().clone()
    i = torch.arange(rotary // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rotary // 2)
    u, w = r[..., a].clone(), r[..., b].clone()
    uc, ws, us, wc = u * c, w * s, u * s, w * c
    r[..., a], r[..., b] = uc - ws, us + wc
    return torch.where(torch.arange(x.shape[-1]) < rotary, r.half(), x)


def table_of(positions, rotary, device="cuda:0", base=10000.0):
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * base ** (-torch.arange(0, rotary, 2, dtype=torch.float64) / rotary)
    return torch.cat([angle.cos(), angle.sin()], 1).float().to(device)
