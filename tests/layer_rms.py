"""Root-mean-square errors of attention and its gradient that rounding alone
explains, for one sequence and fp16 operands: a sharper limit than the worst
cases of ``layer_ref``.

Roundings of the addends of a sum are independent, so their squares add up.  A
rounding to nearest is off by at most half a step of the value, ``u`` relative
(2^-11) or 2^-25 below the normal numbers, and by a root mean square of that
over sqrt(3).  The sums here take the full half step for every rounding; the
factor sqrt(3) that this gives away is what the fp32 parts (scores, statistics,
sums: up to 4e-5 relative, a tenth of u) and the rounding of O inside delta in
the same direction for a whole row may use."""

import numpy as np

U16, TINY16 = 2.0 ** -11, 2.0 ** -25


def plane(x, causal):
    """P, dX and the exact results of one head's attention in float64 (no cap, no bias)."""
    q, k, v, do = (x[n][0, 0] for n in ("Q", "K", "V", "dO"))
    n, m, d = q.shape[0], k.shape[0], q.shape[1]
    scale = 1 / np.sqrt(d)
    s = q @ k.T * scale
    if causal:
        s = np.where(np.arange(m)[None] <= np.arange(n)[:, None] + (m - n), s, -np.inf)
    mx = s.max(1, keepdims=True)
    p = np.exp(s - mx)
    l = p.sum(1, keepdims=True)
    p /= l
    o = p @ v
    dx = p * (do @ v.T - (do * o).sum(1, keepdims=True))
    return p, dx, dict(O=o, L=mx + np.log(l), dQ=dx @ k * scale, dK=dx.T @ q * scale, dV=p.T @ do)


def limits(x, p, dx, out):
    """Root-mean-square error of every result that its roundings explain."""
    q, k, v, do = (x[n][0, 0] for n in ("Q", "K", "V", "dO"))
    scale = 1 / np.sqrt(q.shape[1])
    u2 = U16 ** 2
    final = {n: (U16 * np.abs(y) + TINY16) ** 2 for n, y in out.items()}
    o2 = u2 * ((p * p) @ (v * v)) + final["O"]                       # the weights' rounding, O's own
    row = p @ k * scale                                             # an error of delta moves a row's dX by -P
    delta2 = ((do * do) * (o2 + final["O"])).sum(1, keepdims=True)  # and O is rounded again as it is stored
    dx2 = u2 * dx * dx
    e = dict(O=o2, dQ=dx2 @ (k * k) * scale ** 2 + delta2 * row ** 2 + final["dQ"],
             dK=dx2.T @ (q * q) * scale ** 2 + (p * p * delta2).T @ (q * q) * scale ** 2 + final["dK"],
             dV=u2 * (p * p).T @ (do * do) + final["dV"])
    return {n: float(np.sqrt(y.mean())) for n, y in e.items()}


def rms(got, want):
    return float(np.sqrt(np.mean((np.asarray(got, dtype=np.float64).reshape(want.shape) - want) ** 2)))
