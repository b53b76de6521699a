"""Paged caches with junk wherever nothing may be read from, and plain attention over them in 64 bits."""
import math

import torch

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
NAN = float("nan")


class Cache:
    """Random pools of either layout.  Slots behind a row's end, and pages that no row has, hold NaN; unused table entries are -1.
    k[s][h], v[s][h]: a row's tokens in float64, in their order."""

    def __init__(self, seed, lens, Hk, D, B, dtype, shared, extra_blocks=1, extra_pages=3, scale=1.0):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.Hk, self.D, self.B, self.dtype, self.shared = list(lens), Hk, D, B, dtype, shared
        S, rows = len(lens), 1 if shared else Hk
        need = [-(-n // B) for n in lens]
        self.max_blocks = max(1, max(need) + extra_blocks)
        self.pages = sum(need) * rows + extra_pages
        ids = torch.randperm(self.pages, generator=g).int()
        table = torch.full((S, rows, self.max_blocks), -1, dtype=torch.int32)
        shape = (self.pages, B, Hk, D) if shared else (self.pages, B, D)
        pools = [torch.full(shape, NAN, dtype=dtype) for _ in range(2)]
        self.k, self.v = [], []
        at = 0
        for s, n in enumerate(lens):
            dense = [(torch.randn((n, Hk, D), generator=g) * torch.exp(0.5 * torch.randn((n, Hk, 1), generator=g)) * scale).to(dtype)
                     for _ in range(2)]
            for r in range(rows):
                table[s, r, :need[s]] = ids[at:at + need[s]]
                at += need[s]
                for j in range(need[s]):
                    part = slice(j * B, min(n, (j + 1) * B))
                    for pool, x in zip(pools, dense):
                        pool[table[s, r, j], :part.stop - part.start] = x[part] if shared else x[part, r]
            for store, x in zip((self.k, self.v), dense):
                store.append([x[:, h].double() for h in range(Hk)])
        self.k_pool, self.v_pool = pools
        self.table = table[:, 0].contiguous() if shared else table
        self.seq_lens = torch.tensor(lens, dtype=torch.int32)

    def desc(self, pe, Hq, **kw):
        return pe.make_desc(self.dtype, len(self.lens), self.Hk, Hq, self.D, self.B, self.max_blocks, self.pages,
                            pe.PE_LAYOUT_SHARED if self.shared else pe.PE_LAYOUT_PER_HEAD, **kw)

    def to(self, dev):
        return [x.to(dev) for x in (self.k_pool, self.v_pool, self.table, self.seq_lens)]


def attend(q, k, v, sees=None, scale=None):
    """q [n, D], k and v [t, D], sees [n, t] or None: (out, weights, bound), all float64.  bound[i][d] is how far an element may be
    off where the products are summed in 32 bits, in any order, and the weights carry their error:
      - a logit of D products is off by (D + 3) 2^-24 sum |q_d k_d| scale at most (D - 1 additions, the scale, the reference taken
        off it, each half a step), a weight by twice that relative to itself (its own and the sum's);
      - exp2 by 2^-23, and the weight's two bfloat16 terms by 2^-16 (nothing in fp32, which the bound does not tell apart);
      - a sum over t tokens by (t + 4) 2^-24 relative to the sum of the magnitudes, above and below the division.
    Relative to A = sum w |v|."""
    n, t = q.shape[0], k.shape[0]
    scale = q.shape[1] ** -0.5 if scale is None else scale
    if t == 0:
        z = torch.zeros((n, v.shape[1]), dtype=torch.float64)
        return z, torch.zeros((n, 0), dtype=torch.float64), z
    x = q @ k.T * scale
    mag = q.abs() @ k.abs().T * abs(scale)
    if sees is not None:
        x = x.masked_fill(~sees, -math.inf)
        mag = mag.masked_fill(~sees, 0.0)
    top = x.amax(1, keepdim=True)
    w = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = w.sum(1, keepdim=True)
    w = w / torch.where(total == 0, torch.ones_like(total), total)
    off = 2 * (q.shape[1] + 3) * 2.0 ** -24 * mag.amax(1, keepdim=True) + 2.0 ** -22 + 2.0 ** -16 + 2 * (t + 4) * 2.0 ** -24
    return w @ v, w, off * (w @ v.abs())


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def assert_close(got, want, bound, dtype):
    """Within `bound`, and the output's own rounding."""
    got = got.double().cpu()
    assert bool(torch.isfinite(got).all()), "not finite"
    far = (got - want).abs() - (bound + half_step(dtype) * (want.abs() + bound))
    assert bool((far <= 0).all()), "off by %g more than allowed, value %g" % (float(far.max()), float(want.flatten()[far.argmax()]))
