"""Plain float64 forms of LayerNorm and attention with their gradients, and
bounds on what rounding may change.

The bounds are worst cases counted from the definitions, element by element:
``u`` is half a step of the operands' type (2^-8 bf16, 2^-11 fp16, 2^-24
fp32), ``E`` half a step of fp32.  Sums of n terms in fp32 are off by at most
n E times the sum of magnitudes; elementary functions in fp32 by 8 E (the
hardware's exp2, log2, reciprocal and the compositions here)."""

import numpy as np


U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
E = 2.0 ** -24
F = 8 * E


def rounded(x, dtype):
    """float64 values of x stored in dtype, and the storage array."""
    import torch
    t = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    y = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float64)).to(t)
    store = y.view(torch.int16).numpy().view(np.uint16) if dtype == "bf16" else y.numpy()
    return y.double().numpy(), store


def layernorm(X, gamma, beta, dY, eps, dtype):
    """Results and bounds: {name: (value, bound)}."""
    u, L = U[dtype], X.shape[1]
    mu = X.mean(1, keepdims=True)
    D = X - mu
    var = (D * D).mean(1, keepdims=True)
    r = 1 / np.sqrt(var + eps)
    xh = D * r
    e_mu = L * E * np.abs(X).mean(1, keepdims=True)
    e_D = e_mu + E * np.abs(D)
    e_var = (2 * np.abs(D) * e_D).mean(1, keepdims=True) + (L + 3) * E * var
    e_r = r * (0.5 * e_var / (var + eps) + F)
    e_xh = e_D * r + np.abs(D) * e_r + E * np.abs(xh)
    Y = xh * gamma + beta
    e_Y = e_xh * np.abs(gamma) + 2 * E * (np.abs(xh * gamma) + np.abs(Y)) + u * np.abs(Y)
    out = {"Y": (Y, e_Y), "mu": (mu, e_mu + E * np.abs(mu)), "r": (r, e_r)}
    g = dY * gamma
    gx = g * xh
    c1, c2 = g.mean(1, keepdims=True), gx.mean(1, keepdims=True)
    e_c1 = (L + 2) * E * np.abs(g).mean(1, keepdims=True)
    e_gx = np.abs(g) * e_xh + 3 * E * np.abs(gx)
    e_c2 = e_gx.mean(1, keepdims=True) + (L + 2) * E * np.abs(gx).mean(1, keepdims=True)
    inner = g - c1 - xh * c2
    e_in = 2 * E * np.abs(g) + e_c1 + e_xh * np.abs(c2) + np.abs(xh) * e_c2 + 4 * E * (np.abs(g) + np.abs(c1) + np.abs(xh * c2))
    dX = r * inner
    out["dX"] = (dX, e_r * np.abs(inner) + r * e_in + (2 * E + u) * np.abs(dX))
    R = X.shape[0]
    t = dY * xh
    dg = t.sum(0)
    out["dgamma"] = (dg, (np.abs(dY) * e_xh).sum(0) + (R + 2) * E * np.abs(t).sum(0) + u * np.abs(dg))
    db = dY.sum(0)
    out["dbeta"] = (db, R * E * np.abs(dY).sum(0) + u * np.abs(db))
    return out


def bucket_map(radius, buckets):
    """A bucket of every distance -radius .. radius, neither sorted nor all used."""
    t = np.arange(-radius, radius + 1)
    return (np.abs(t) * 3 + (t > 0) * 5) % buckets


def attention(x, dtype, heads, kv_heads, cap=0.0, causal=False, radius=0, grad=False):
    """x: float64 arrays by input name.  Results and bounds: {name: (value, bound)}.
    Every product's bound is the operands' errors times magnitudes."""
    u = U[dtype]
    Q, K, V = x["Q"], x["K"], x["V"]
    B, H, N, D = Q.shape
    M = K.shape[2]
    G = H // kv_heads
    scale = 1 / np.sqrt(D)
    j = np.arange(M)
    res = {k: [np.zeros_like(Q), np.zeros_like(Q)] for k in ("O", "dQ")}
    res["L"] = [np.zeros((B, H, N, 1)), np.zeros((B, H, N, 1))]
    for k in ("dK", "dV"):
        res[k] = [np.zeros_like(K), np.zeros_like(K)]
    if radius:
        res["dT"] = [np.zeros_like(x["table"]), np.zeros_like(x["table"])]
    for b in range(B):
        size = int(x["lengths"][b]) if "lengths" in x else M
        pos = size - N + np.arange(N)
        rel = j[None] - pos[:, None]
        mask = np.broadcast_to(j[None] < size, (N, M)).copy()
        if causal:
            seen = rel <= 0
            if "prefix" in x:
                seen = seen | (j[None] < x["prefix"][b])
            mask &= seen
        if "documents" in x:
            d = x["documents"][b]
            mask &= d[pos][:, None] == d[None]
        for h in range(H):
            q, k, v = Q[b, h], K[b, h // G].copy(), V[b, h // G].copy()
            k[size:], v[size:] = 0, 0
            s0 = q @ k.T * scale
            e_s = (D + 2) * E * (np.abs(q) @ np.abs(k).T) * scale + 4 * E * np.abs(s0)
            t = None
            if cap:
                t = np.tanh(s0 / cap)
                s0 = cap * t
                e_s = e_s + cap * F
            if "slopes" in x:
                bias = x["slopes"][h] * np.abs(rel)
                e_s = e_s + 2 * E * np.abs(bias)
                s0 = s0 - bias
                e_s = e_s + E * np.abs(s0)
            if radius:
                which = x["bucket"][np.clip(rel, -radius, radius) + radius].astype(int)
                s0 = s0 + x["table"][h][which]
                e_s = e_s + E * np.abs(s0)
            s = np.where(mask, s0, -np.inf)
            some = mask.any(1, keepdims=True)
            mx = np.where(some, np.max(s, 1, keepdims=True), 0)
            p = np.where(mask, np.exp(s - mx), 0)
            l = p.sum(1, keepdims=True)
            l1 = np.where(some, l, 1)
            L = np.where(some, mx + np.log(l1), 0)
            p = p / l1
            # relative error of an exponential: the score's, the rounding of its argument in base 2, the function's
            e_p = np.where(mask, e_s + 4 * E * (np.abs(np.where(mask, s, 0)) + np.abs(mx)) + F, 0)
            e_l = (p * e_p).sum(1, keepdims=True) + M * E
            o = p @ v
            a = p @ np.abs(v)
            res["O"][0][b, h] = o
            res["O"][1][b, h] = (p * (e_p + e_l + u)) @ np.abs(v) + (M * E + F) * a + (u + F) * np.abs(o)
            res["L"][0][b, h] = L
            e_L = np.where(some, e_l + e_p.max(1, keepdims=True) + F * (1 + np.abs(np.log(l1))) + 4 * E * (np.abs(L) + np.abs(mx)), 0)
            res["L"][1][b, h] = e_L
            if not grad:
                continue
            do = x["dO"][b, h]
            dp = do @ v.T
            e_dp = (D + 2) * E * (np.abs(do) @ np.abs(v).T)
            delta = (do * o).sum(1, keepdims=True)
            e_delta = (np.abs(do) * (res["O"][1][b, h])).sum(1, keepdims=True) + (D + 2) * E * (np.abs(do) * np.abs(o)).sum(1, keepdims=True)
            e_pg = np.where(mask, e_s + e_L + 4 * E * (np.abs(np.where(mask, s, 0)) + np.abs(L)) + F, 0)
            dd = dp - delta
            ds = p * dd
            e_ds = p * (e_dp + e_delta + 2 * E * np.abs(dd)) + np.abs(ds) * (e_pg + 2 * E)
            if radius:
                for w in range(x["table"].shape[1]):
                    at = (which == w) & mask
                    res["dT"][0][h, w] += ds[at].sum()
                    res["dT"][1][h, w] += e_ds[at].sum() + (B * N + M) * E * np.abs(ds[at]).sum()
            if cap:
                f = 1 - t * t
                e_ds = e_ds * f + np.abs(ds) * 4 * F
                ds = ds * f
            e_dx = e_ds + (u + 2 * E) * np.abs(ds)
            res["dQ"][0][b, h] = ds @ k * scale
            res["dQ"][1][b, h] = (e_dx @ np.abs(k) + M * E * (np.abs(ds) @ np.abs(k))) * scale + (u + 2 * E) * np.abs(ds @ k * scale)
            res["dK"][0][b, h // G] += ds.T @ q * scale
            res["dK"][1][b, h // G] += (e_dx.T @ np.abs(q) + G * N * E * (np.abs(ds).T @ np.abs(q))) * scale
            res["dV"][0][b, h // G] += p.T @ do
            res["dV"][1][b, h // G] += (p * (e_pg + u)).T @ np.abs(do) + G * N * E * (p.T @ np.abs(do))
    for k in ("dK", "dV", "dT"):
        if k in res:
            res[k][1] += (u + 2 * E) * np.abs(res[k][0])
    return {k: tuple(v) for k, v in res.items() if grad or k in ("O", "L")}


# Smallest half step of fp16 (its subnormals), as an absolute floor of a rounding.
FLOOR = {"f32": 1e-37, "f16": 2.0 ** -25, "bf16": 1e-37}


def outside(got, value, bound, dtype):
    """Largest error over its bound (a result is right when it is at most 1)."""
    got = np.asarray(got, dtype=np.float64).reshape(value.shape)
    if not np.all(np.isfinite(got)):
        return np.inf
    return float(np.max(np.abs(got - value) / (bound + FLOOR[dtype])))
