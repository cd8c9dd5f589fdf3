"""Plain float64 forms of group norm, rotary positions and gradient clipping with
their gradients, and bounds on what rounding may change.

The bounds are worst cases counted from the definitions, element by element,
with the constants of ``layer_ref``: ``u`` half a step of the stored type, ``E``
half a step of fp32, ``F`` = 8 E for an elementary function.  A sum of n terms
passes a term through ``depth(n)`` fp32 additions at most: a thread adds at most
one in 256 of them one after another (64 when they are few), then the threads of a
workgroup, its slices and the workgroups add up to 450 partial sums in turn."""

import numpy as np

from .layer_ref import E, F, U, outside, rounded  # noqa: F401


def depth(n):
    return min(n, 512 + n // 256)


def groupnorm(X, gamma, beta, groups, eps, act, dtype, dY=None):
    """X [batch, hh, ww, c]: {name: (value, bound)} of the results, and of the gradient's with dY."""
    u = U[dtype]
    B, H, W, C = X.shape
    K = C // groups
    x = X.reshape(B, H * W, groups, K)
    ga, be = gamma.reshape(groups, K), beta.reshape(groups, K)
    n = H * W * K
    d = depth(n)

    def mean(a):
        return a.mean((1, 3), keepdims=True)

    mu = mean(x)
    D = x - mu
    var = mean(D * D)
    r = 1 / np.sqrt(var + eps)
    xh = D * r
    e_mu = (d + 2) * E * mean(np.abs(x))
    e_D = e_mu + E * np.abs(D)
    # (squares about means of parts merge into squares about the whole's: twice the error of one pass)
    e_var = mean(4 * np.abs(D) * e_D + e_D * e_D) + (d + 8) * E * var
    e_r = r * (0.5 * e_var / (var + eps) + F)
    e_xh = e_D * r + np.abs(D) * e_r + E * np.abs(xh)
    z = xh * ga + be
    e_z = e_xh * np.abs(ga) + 2 * E * (np.abs(xh * ga) + np.abs(z))
    if act == "silu":
        s = 1 / (1 + np.exp(-z))
        rel = F + 4 * E * np.abs(z)  # of 1 / (1 + exp(-z)): the exponent's argument is rounded in base 2
        y, e_y = z * s, 1.1 * e_z + rel * np.abs(z * s)
        slope = s * (1 + z * (1 - s))
        e_slope = 0.5 * e_z + 3 * rel * s * (1 + np.abs(z) * (1 - s)) + 4 * E * s * np.abs(z) * (1 + rel)
    elif act == "relu":
        y, e_y = np.maximum(z, 0), e_z
        slope = (z > 0).astype(float)
        e_slope = (np.abs(z) <= e_z).astype(float)
    else:
        y, e_y, slope, e_slope = z, e_z, np.ones_like(z), np.zeros_like(z)
    out = {"Y": (y.reshape(X.shape), (e_y + (u + E) * np.abs(y)).reshape(X.shape)), "mu": (mu.reshape(B, groups), (e_mu + E * np.abs(mu)).reshape(B, groups)),
           "r": (r.reshape(B, groups), e_r.reshape(B, groups))}
    if dY is None:
        return out
    dy = dY.reshape(x.shape)
    dz = dy * slope
    e_dz = np.abs(dy) * e_slope + 2 * E * np.abs(dz)
    dzx = dz * xh
    e_dzx = e_dz * np.abs(xh) + np.abs(dz) * e_xh + E * np.abs(dzx)
    k = depth(B * H * W)
    db, dg = dz.sum((0, 1)), dzx.sum((0, 1))
    e_db = e_dz.sum((0, 1)) + (k + 2) * E * np.abs(dz).sum((0, 1)) + u * np.abs(db)
    e_dg = e_dzx.sum((0, 1)) + (k + 2) * E * np.abs(dzx).sum((0, 1)) + u * np.abs(dg)
    g, gx = dz * ga, dzx * ga
    c1, c2 = mean(g), mean(gx)
    e_c1 = mean(e_dz * np.abs(ga)) + (d + 4) * E * mean(np.abs(g))
    e_c2 = mean(e_dzx * np.abs(ga)) + (d + 4) * E * mean(np.abs(gx))
    inner = g - c1 - xh * c2
    e_in = e_dz * np.abs(ga) + e_c1 + e_xh * np.abs(c2) + np.abs(xh) * e_c2 + 4 * E * (np.abs(g) + np.abs(c1) + np.abs(xh * c2))
    dX = r * inner
    out["dX"] = (dX.reshape(X.shape), (e_r * np.abs(inner) + r * e_in + (2 * E + u) * np.abs(dX)).reshape(X.shape))
    out["dgamma"] = (dg.reshape(C), e_dg.reshape(C))
    out["dbeta"] = (db.reshape(C), e_db.reshape(C))
    return out


def turn(X, positions, axis, freq, interleaved, back, dtype):
    """X [batch, heads, n, d] turned by the angles (value, bound): the angle is exact, its
    cosine and sine are off by at most 3 E (the angle's rounding to fp32 inside an eighth of a
    turn, the sums' and their last bits)."""
    u = U[dtype]
    P = len(freq)
    place = positions[..., axis.astype(int)] if axis is not None else positions
    a = (place * freq)[:, None]
    c, s = np.cos(a), np.sin(a) * (-1 if back else 1)
    one, two = (slice(0, 2 * P, 2), slice(1, 2 * P, 2)) if interleaved else (slice(0, P), slice(P, 2 * P))
    x1, x2 = X[..., one], X[..., two]
    y, e = X.copy(), np.zeros_like(X)
    y[..., one], y[..., two] = x1 * c - x2 * s, x2 * c + x1 * s
    size = np.abs(x1) + np.abs(x2)
    e[..., one] = e[..., two] = 5 * E * size
    return y, e + u * np.abs(y) * (e > 0)


def clipped(grads, dtypes, max_norm, eps):
    """norm and the clipped gradients (value, bound); the sum of squares in 64 bits."""
    norm = np.sqrt(sum((g * g).sum() for g in grads))
    f = min(1.0, max_norm / (norm + eps))
    out = {"norm": (np.array([norm]), np.array([2 * E * norm]))}
    for i, (g, t) in enumerate(zip(grads, dtypes)):
        out[f"C{i}"] = (g * f, (U[t] + 8 * E) * np.abs(g * f))
    return out
