"""Caches in 8 bits with junk wherever nothing may be read from, their rounding and their attention in 64 bits."""
import math

import torch

from _paged64 import Cache, DTYPES   # noqa: F401

E4M3 = torch.float8_e4m3fn
NAN = float("nan")


def scale_of(top):
    """The least power of two s, 2^-126 or more, with top <= 448 s; 1 for 0."""
    if top == 0:
        return 1.0
    m, e = math.frexp(top)
    return 2.0 ** max(-126, e - 9 if m <= 0.875 else e - 8)


def round_page(x):
    """x [B, D] of one head -> (bytes, scale)."""
    s = scale_of(float(x.abs().max()))
    return (x.double() / s).float().to(E4M3).view(torch.uint8), s


def page_score(k, v):
    nk, nv = k.double().square().sum(1).sqrt(), v.double().square().sum(1).sqrt()
    return float(torch.where(nv == 0, torch.zeros_like(nv), nv / nk).mean())


class QuantCache(Cache):
    """A Cache whose full pages are rounded.  k[s][h], v[s][h]: what a row's tokens stand for, in float64."""

    def __init__(self, seed, lens, Hk, D, B, dtype, shared, odd_scales=False, **kw):
        super().__init__(seed, lens, Hk, D, B, dtype, shared, **kw)
        g = torch.Generator().manual_seed(seed + 1000)
        self.k8, self.v8 = (torch.full(self.k_pool.shape, 0x7f, dtype=torch.uint8) for _ in range(2))
        self.scales = torch.full((self.pages,) + ((Hk,) if shared else ()) + (2,), NAN)
        self.k_tail, self.v_tail = (torch.full((len(lens), Hk, B, D), NAN, dtype=dtype) for _ in range(2))
        for s, n in enumerate(lens):
            for h in range(Hk):
                for i, (x, held, tail) in enumerate(((self.k, self.k8, self.k_tail), (self.v, self.v8, self.v_tail))):
                    for j in range(n // B):
                        rows = slice(j * B, (j + 1) * B)
                        page = int(self.table[s, j] if shared else self.table[s, h, j])
                        b, scale = round_page(x[s][h][rows])
                        if odd_scales:
                            scale *= float(1.0 + torch.rand(1, generator=g))
                        scale = float(torch.tensor(scale, dtype=torch.float32))
                        at = (page, slice(None), h) if shared else (page,)
                        held[at] = b
                        self.scales[(page, h, i) if shared else (page, i)] = scale
                        x[s][h][rows] = b.view(E4M3).float().double() * scale
                    tail[s, h, :n % B] = x[s][h][n - n % B:].to(dtype)

    def quant(self, pe, desc, dev):
        return pe.make_quant_cache(desc, *(x.to(dev) for x in (self.k8, self.v8, self.scales, self.k_tail, self.v_tail)))


def attend(q, k, v, dtype, scale=None):
    """q [n, D], k, v [t, D] in float64 -> (out, bound).  Half steps of 2^-24:
      - a logit's D products, of eight term products each at most (fp32 queries and keys), summed in any order, with the scales of the
        page and of the softmax: 8 D + 4 relative to sum |q_d k_d| scale, and what is left out of fp32 terms 2^-29; a weight twice that
        relative to itself, and exp2 and the scaling by V's scale 2^-22; bfloat16: what the weight's second term of 8 bits leaves of it, 2^-17;
      - a sum over t tokens of up to nine term products: 9 t + 4, above and below the division."""
    scale = q.shape[1] ** -0.5 if scale is None else scale
    if k.shape[0] == 0:
        z = torch.zeros((q.shape[0], v.shape[1]), dtype=torch.float64)
        return z, z
    terms = 8 if dtype == torch.float32 else 1
    x = q @ k.T * scale
    mag = q.abs() @ k.abs().T * abs(scale)
    w = torch.softmax(x, 1)
    off = 2 * ((terms * q.shape[1] + 4) * 2.0 ** -24 + 2.0 ** -29) * mag.amax(1, keepdim=True) + 2.0 ** -21 + (2.0 ** -17 if terms == 1 else 0) + 2 * (3 * terms * k.shape[0] + 4) * 2.0 ** -24
    return w @ v, off * (w @ v.abs())
