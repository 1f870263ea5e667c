"""Plain 64-bit forms of the rotary embedding, the paged append and the chunk attention, for the tests (CPU)."""
import math

import torch


def rotate(x, pos, axis_pairs, theta, interleaved, restart, inverse=False):
    """x [T, H, d] (any float type), pos [axes, T] -> fp64."""
    T, H, d = x.shape
    half = d // 2
    out = x.double().clone()
    first = 0
    for a, n in enumerate(axis_pairs):
        for i in range(n):
            p = first + i
            ang = pos[a].double() * theta ** -(i / n if restart else p / half)
            c, s = torch.cos(ang)[:, None], torch.sin(ang)[:, None] * (-1 if inverse else 1)
            ia, ib = (2 * p, 2 * p + 1) if interleaved else (p, p + half)
            u, v = x[:, :, ia].double(), x[:, :, ib].double()
            out[:, :, ia] = u * c - v * s
            out[:, :, ib] = v * c + u * s
        first += n
    assert first == half
    return out


def partner_sum(x, interleaved):
    """|x| + |y| of each element's pair (what the rounding of a rotation scales with)."""
    d = x.shape[-1]
    a = x.double().abs()
    if interleaved:
        s = a[..., 0::2] + a[..., 1::2]
        return torch.stack([s, s], -1).flatten(-2)
    s = a[..., :d // 2] + a[..., d // 2:]
    return torch.cat([s, s], -1)


def attention(q, rows_k, rows_v, n, lens, start, causal, group, scale):
    """q [T, Hq, d]; rows_k(s, h, j0, j1) -> the cached rows; returns out, sum p|V|, largest sum|q k| scale per row (fp64)."""
    T, Hq, d = q.shape
    out = torch.zeros(T, Hq, d, dtype=torch.float64)
    mag = torch.zeros(T, Hq, d, dtype=torch.float64)
    big = torch.zeros(T, Hq, dtype=torch.float64)
    t = 0
    for s, (a, b) in enumerate(zip(n, lens)):
        lo = max(start[s], 0) if start is not None else 0
        for h in range(Hq):
            if a == 0 or b <= lo:
                continue
            K, V = rows_k(s, h // group, lo, b).double(), rows_v(s, h // group, lo, b).double()
            for i in range(a):
                hi = (b - a + i + 1 if causal else b) - lo
                if hi <= 0:
                    continue
                qi = q[t + i, h].double()
                x = K[:hi] @ qi * scale
                p = torch.softmax(x, 0)
                out[t + i, h] = p @ V[:hi]
                mag[t + i, h] = p @ V[:hi].abs()
                big[t + i, h] = (K[:hi].abs() @ qi.abs()).max() * scale
        t += a
    return out, mag, big


def attention_tolerance(dtype, out, mag, big, d, longest):
    """Bound of |kernel - out|.  A logit is a dot product of d terms in fp32: off by at most d 2^-24 sum|q k| scale, plus its
    scaling and the exponential's argument (2^-22 of a logit's size, that size bounded by the same sum); that relative error enters numerator
    and denominator.  Sums over the slots in fp32: longest 2^-24 each.  exp2: 2^-21.  bf16 adds P rounded once (2^-8 of each
    term) and the result rounded once (2^-8 of it)."""
    rel = 2 * (big * (d * 2.0 ** -24 + 2.0 ** -22) + longest * 2.0 ** -24 + 2.0 ** -21)[..., None]
    tol = mag * rel + 1e-30
    if dtype == torch.bfloat16:
        tol = tol + mag * 2.0 ** -8 + (out.abs() + mag * (rel + 2.0 ** -8)) * 2.0 ** -8
    else:
        tol = tol + out.abs() * 2.0 ** -24
    return tol


def rotation_tolerance(dtype, ref, x, interleaved):
    """sincospif is good to 2 units in the last place (2^-23 absolute), its argument is rounded to fp32 in half turns (2 pi 2^-26),
    products and sum are rounded once each (2^-24 of |x| + |y| each, twice for the sum of two rounded products)."""
    tol = partner_sum(x, interleaved) * (2.0 ** -23 + 2 * math.pi * 2.0 ** -26 + 3 * 2.0 ** -24)
    return tol + (ref.abs() + tol) * (2.0 ** -8 if dtype == torch.bfloat16 else 0.0)
