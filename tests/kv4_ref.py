"""The 4-bit cache in 64 bits, from the formats' definitions: what its tests compare with.

Tolerances of attention, from the kernels' roundings (u = half a step, relative):
  - the output is rounded to bf16: 2^-8 |out|;
  - P is rounded to FP16: 2^-11 of each P, so at most 2^-11 sum p |v|.  P carries a factor
    2^15 and a row's largest is 1 before it, so a P below 2^-29 is an FP16 subnormal and off
    by up to half of their step, 2^-25 / 2^15 = 2^-40 of the largest (which is at most the
    whole sum of P): at most 2^-40 sum |v| more, over the keys that the row sees;
  - a score is a sum of 128 exact products in FP32 (each of the 128 additions off by
    2^-24 of the sum of magnitudes A = sum |q k| / sqrt(128)), then scaled, shifted and
    raised (4 more roundings of numbers no larger than 2 A log2(e), and 2^-22 of the
    exponential): p is off by a factor within e^(+-d), d = (128 + 8) 2^-24 * 2 A + 2^-21, in
    the sum of p v and in the sum of p alike: e^(2 d) - 1 together;
  - FP32 sums over n keys and merges: n / 64 chained additions of 64 lanes' parts and the
    merge, at most (n / 16 + 64) 2^-24 each for numerator and denominator.
"""
import math

import torch

D, PAGE = 128, 64


def pow2(e):
    """2^e exactly, from the format's fields (torch's power and ldexp are a rounding off on the GPU)."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def e2m1_value(c):
    c = c.double()
    sign, e, m = torch.floor(c / 8), torch.floor(c % 8 / 2), c % 2
    return torch.where(e > 0, (1 + m / 2) * pow2(e - 1), m / 2) * (1 - 2 * sign)


def e4m3_value(c):
    c = c.double()
    e, m = torch.floor(c % 128 / 8), c % 8
    x = torch.where(e > 0, (1 + m / 8) * pow2(e - 7), m / 512) * torch.where(c >= 128, -1.0, 1.0)
    return torch.where(c % 128 == 127, math.nan, x)


def _grid(a, bits, least, most):
    """a >= 0 to `bits` mantissa bits, ties to even, at most `most`; below 2^least on its binade's grid."""
    mant, exp = torch.frexp(a)
    step = pow2((exp - 1).clamp(min=least) - bits)
    return (torch.round(a / step) * step).clamp(max=most)


def quantize(x, t):
    """x [..., 128] in 64 bits under tensor scales t [...]: code values [..., 128], scale values [..., 8]."""
    g = x.reshape(*x.shape[:-1], 8, 16)
    scale = _grid(g.abs().amax(-1) / (6 * t[..., None]), 3, -6, 448.0)
    step = (scale * t[..., None])[..., None]
    y = torch.where(step > 0, g / torch.where(step > 0, step, 1.0), 0.0)
    return (_grid(y.abs(), 1, 0, 6.0) * torch.sign(y)).flatten(-2), scale


def tensor_scale(amax):
    k = -63
    t = torch.full_like(amax, 2.0 ** k)
    while k < 63:
        k += 1
        t = torch.where(2688 * t < amax, 2.0 ** k, t)
    return torch.where(amax > 0, t, 1.0)


class Tokens:
    """Codes (byte rows), scales and weights of tokens of a cache, in token order."""

    def __init__(self, cache, page_row, n):
        i = torch.arange(n, device=cache.k_codes.device)
        pg, o = page_row[i // PAGE].long(), i % PAGE
        self.k_codes = cache.k_codes[pg, :, o]                                     # [n][H][64]
        self.k_scales = cache.k_scales[pg, :, o]                                   # [n][H][8]
        vc = cache.v_codes.view(*cache.v_codes.shape[:2], 16, 16, 4, 4)
        self.v_codes = vc[pg, :, o // 4, :, o % 4].flatten(2)                      # [n][H][16 octets * 4]
        self.v_scales = cache.v_scales[pg, :, :, o]                                # [n][H][8]
        self.weights = None if cache.weights is None else cache.weights[pg, :, o]  # [n][H]

    @staticmethod
    def _values(codes, scales):
        c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
        return e2m1_value(c) * e4m3_value(scales).repeat_interleave(16, -1)

    def k(self):
        return self._values(self.k_codes, self.k_scales)

    def v(self):
        return self._values(self.v_codes, self.v_scales)


def attention(q, tokens, t_k, t_v, pos0, window, sinks):
    """q bf16 [R][Hq][128] at positions pos0 ..: out [R][Hq][128], the tolerance of every output,
    the share of every key [n][H] and its tolerance, all in 64 bits."""
    k, v = tokens.k() * t_k.double()[None, :, None], tokens.v() * t_v.double()[None, :, None]
    n, h = k.shape[:2]
    r, hq = q.shape[:2]
    g = hq // h
    pos = pos0 + torch.arange(r, device=q.device)
    j = torch.arange(n, device=q.device)
    seen = j <= pos[:, None]
    if window:
        seen &= (pos[:, None] - j < window) | (j < sinks)
    out, tol = torch.zeros(r, hq, D, dtype=torch.float64, device=q.device), torch.zeros(r, hq, D, dtype=torch.float64, device=q.device)
    share, share_tol = torch.zeros(n, h, dtype=torch.float64, device=q.device), torch.zeros(n, h, dtype=torch.float64, device=q.device)
    for hk in range(h):
        qq = q[:, hk * g:hk * g + g].double().reshape(r * g, D)
        mask = seen.repeat_interleave(g, 0)
        s = (qq @ k[:, hk].T) / math.sqrt(D)
        some = mask.any(1)
        p = torch.softmax(torch.where(mask, s, -math.inf)[some], -1)
        a = torch.where(mask, qq.abs() @ k[:, hk].abs().T, 0.0).amax(1)[some] / math.sqrt(D) if n else torch.zeros(0, device=q.device)
        d = (136 * 2.0 ** -24 * 2 * a + 2.0 ** -21)[:, None]
        o, mag = torch.zeros(r * g, D, dtype=torch.float64, device=q.device), torch.zeros(r * g, D, dtype=torch.float64, device=q.device)
        if some.any():
            o[some], spread = p @ v[:, hk], p @ v[:, hk].abs()
            mag[some] = (2.0 ** -11 + torch.expm1(2 * d) + 2 * (n / 16 + 64) * 2.0 ** -24) * spread
            mag[some] += 2.0 ** -40 * (mask[some].double() @ v[:, hk].abs())
            share[:, hk] = p.sum(0)
            share_tol[:, hk] = ((torch.expm1(2 * d) + (n / 16 + 64) * 2.0 ** -24) * p).sum(0) + r * g * 2.0 ** -24 * p.sum(0)
        out[:, hk * g:hk * g + g] = o.view(r, g, D)
        tol[:, hk * g:hk * g + g] = (2.0 ** -8 * (o.abs() + mag) + mag).view(r, g, D)
    return out, tol, share, share_tol


def keep(weights, budget, sinks, recent):
    """Indices kept of weights [n] (floats), ascending."""
    n = weights.numel()
    if n <= budget:
        return list(range(n))
    w = weights.tolist()
    mid = list(range(sinks, n - recent))
    rank = lambda i: (0 if math.isnan(w[i]) else 1, -w[i] if not math.isnan(w[i]) else 0.0, i)   # NaN first
    best = sorted(mid, key=rank)[:budget - sinks - recent]
    return sorted(list(range(sinks)) + best + list(range(n - recent, n)))


def random_cache(mp, pages, h_kv, seed, weights=False, device="cuda"):
    """A cache of random bytes: every code, scales with finite E4M3 values between 2^-3 and 2^5."""
    gen = torch.Generator(device=device).manual_seed(seed)
    c = mp.PagedCache4(pages, h_kv, device=device, weights=weights)
    for t in (c.k_codes, c.v_codes):
        t.copy_(torch.randint(0, 256, t.shape, generator=gen, device=device, dtype=torch.int32).to(torch.uint8))
    for t in (c.k_scales, c.v_scales):
        t.copy_(torch.randint(0x20, 0x60, t.shape, generator=gen, device=device, dtype=torch.int32).to(torch.uint8))
    if weights:
        c.weights.copy_(torch.rand(c.weights.shape, generator=gen, device=device))
    return c


def page_rows(lens, pages, seed, width=None):
    """A page table [B][width] of distinct random pages (-1 past a sequence's last)."""
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).int()
    need = [(n + PAGE - 1) // PAGE for n in lens]
    rows = torch.full((len(lens), width or max(1, *need) if len(need) > 1 else width or max(1, need[0])), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        rows[b, :n] = order[at:at + n]
        at += n
    return rows


def stale(cache, rows, lens):
    """Every byte that belongs to no token of the sequences becomes 0xFF (E4M3 NaN, weights NaN)."""
    used = torch.zeros(cache.num_pages, PAGE, dtype=torch.bool, device=cache.k_codes.device)
    for b, n in enumerate(lens):
        i = torch.arange(n, device=used.device)
        used[rows[b].to(used.device)[i // PAGE].long(), i % PAGE] = True
    pg, o = torch.nonzero(~used, as_tuple=True)
    cache.k_codes[pg, :, o] = 255
    cache.k_scales[pg, :, o] = 255
    cache.v_scales[pg, :, :, o] = 255
    cache.v_codes.view(*cache.v_codes.shape[:2], 16, 16, 4, 4)[pg, :, o // 4, :, o % 4] = 255
    if cache.weights is not None:
        cache.weights[pg, :, o] = math.nan
