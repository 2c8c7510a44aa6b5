"""The 4-bit cache in 64 bits on the CPU from its definition, and attention over what it holds (test infrastructure)."""
import math

import torch

LEVELS = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)


def held(x):
    """The values the cache holds for x [..., d]."""
    y = x.double().reshape(-1, 32)
    out = torch.empty_like(y)
    a = y.abs().amax(-1)
    bad = ~torch.isfinite(y).all(-1)
    m, e = torch.frexp(torch.where(bad, 0.0, a) / 6)
    s = torch.ldexp(torch.round(m * 64) / 64, e).clamp(max=1.3125 * 2.0 ** 125)
    s = torch.where(a < 2.0 ** -100, 0.0, s)
    q = torch.where(s[:, None] > 0, y.abs() / torch.where(s > 0, s, 1.0)[:, None], 0.0).nan_to_num(0, posinf=6)
    d = (q[..., None] - LEVELS).abs()                      # exact: few bits
    best = d.amin(-1, keepdim=True)
    tied = d == best
    even = torch.tensor([1.0 if i % 2 == 0 else 0.5 for i in range(8)])
    code = (tied * even).argmax(-1)                        # of two at the same distance the even one
    out = s[:, None] * torch.sign(y) * LEVELS[code]
    out[bad] = float("nan")
    return out.reshape(x.shape)


def attend(q, k, v, group, scale, first):
    """q [n, Hq, d], k, v [L, Hkv, d] in any type; row i sees keys 0 .. first + i.  (o [n, Hq, d], lse [Hq, n], and the sum of p |v|)."""
    n, hq, d = q.shape
    o, lse, size = torch.zeros(n, hq, d, dtype=torch.float64), torch.full((hq, n), -math.inf, dtype=torch.float64), torch.zeros(n, hq, d, dtype=torch.float64)
    for i in range(n):
        m = min(first + i + 1, k.shape[0])
        if m <= 0:
            continue
        for h in range(hq):
            s = scale * (k[:m, h // group].double() @ q[i, h].double())
            lse[h, i] = torch.logsumexp(s, 0)
            p = torch.exp(s - lse[h, i])
            o[i, h] = p @ v[:m, h // group].double()
            size[i, h] = p @ v[:m, h // group].double().abs()
    return o, lse, size
