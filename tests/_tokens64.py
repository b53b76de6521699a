"""Plain forms of a plan of tokens (whole numbers, one sequence after the other) and of rotary positions (64 bits)."""
import math

import torch


def plan(lens, new, first, total, budget, free, used, table, spare, n_spare, B):
    """table, spare: lists of rows a sequence, changed in place.  Returns lens_out, used_out, cu, positions, slots."""
    left_from = max(0, min(used, len(free)))
    at, short, lens_out, cu = left_from, False, [], [0]
    pos, slots = [0] * total, [[-1] * (len(table[0]) if table else 1) for _ in range(total)]
    for s, (n, m) in enumerate(zip(lens, new)):
        m = max(m, 0)
        after = n + m
        kept = max(n, min(after, budget)) if budget else after
        have, need = -(-n // B), -(-kept // B) - -(-n // B)
        extra = n_spare if n == 0 and m > 0 else 0
        rows = table[s]
        serves = -(-kept // B) <= len(rows[0])
        if serves and need + extra:
            if short or at + len(rows) * (need + extra) > len(free):
                serves, short = False, True
            else:
                for h, row in enumerate(rows):
                    row[have:have + need] = free[at:at + need]
                    if extra:
                        spare[s][h][:] = free[at + need:at + need + extra]
                    at += need + extra
        for i in range(m):
            t = cu[-1] + i
            if t < total:
                pos[t] = (n if first is None else first[s]) + i
                for h, row in enumerate(rows):
                    if serves and kept == after:
                        page = row[(n + i) // B]
                        slots[t][h] = -1 if page < 0 else page * B + (n + i) % B
        lens_out.append(kept if serves else n)
        cu.append(cu[-1] + m)
    return lens_out, at, cu, pos, slots


def frequencies(R, base, scaling="none", factor=1.0, low=1.0, high=4.0, original=8192.0):
    f = [base ** (-2.0 * i / R) for i in range(R // 2)]
    if scaling == "linear":
        f = [x / factor for x in f]
    if scaling == "parts":
        keep = [min(1.0, max(0.0, (original * x / (2 * math.pi) - low) / (high - low))) for x in f]
        f = [x * (g + (1 - g) / factor) for x, g in zip(f, keep)]
    return f


def rotate(x, positions, f, interleaved, magnitude=1.0, transpose=False):
    """x [T, heads, D] -> (y, bound), float64.  bound: how far 32 bits may be off.  With half steps of 2^-24: an angle within an eighth of a
    turn is off by three in itself (its conversion, the constant and the product, times pi/4, and 2^-32 turns), its sine and cosine by two
    more, the magnitude by one, the two products and their sum by two: eight, relative to m (|x_a| + |x_b|).  The reference's own
    angle: position * f in 64 bits, 2^-52 of it."""
    n = 2 * len(f)
    p = positions.double()[:, None]
    angle = p * torch.tensor(f, dtype=torch.float64) * (-1.0 if transpose else 1.0)
    c, s = torch.cos(angle)[:, None] * magnitude, torch.sin(angle)[:, None] * magnitude
    y, bound = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64)
    a, b = (slice(0, n, 2), slice(1, n, 2)) if interleaved else (slice(0, n // 2), slice(n // 2, n))
    xa, xb = x.double()[..., a], x.double()[..., b]
    y[..., a], y[..., b] = xa * c - xb * s, xb * c + xa * s
    off = (8 * 2.0 ** -24 + angle.abs()[:, None] * 2.0 ** -52) * magnitude * (xa.abs() + xb.abs())
    bound[..., a], bound[..., b] = off, off
    return y, bound
