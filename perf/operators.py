"""Performance cases of the operators of a transformer layer's training and serving.

* ``layernorm``: LayerNorm that keeps its row statistics, and its gradient with
  the column sums of the weight's and the bias's gradients;
* ``attention``: attention of any length whose scores may be capped by a tanh,
  biased by distance and masked (causal, prefix, documents, lengths), with
  shared key / value heads, and its form for single tokens over a long cache;
* ``attention_train``: that attention's forward pass and its gradient;
* ``bucket_train``: attention with a learned relative position bias by buckets,
  forward and gradient (the bias table's gradient among the results).

With ``own`` false the operators run in their plain form (elementary torch
operations in 32 bits); with ``own`` true as the framework's plans, through the
calls a training or serving loop makes (``graphs.build``, ``PlanRunner``,
``bind``, ``launch_bound``).
"""

import math

import torch

own = False

TORCH_DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-5
LOW = -1e30   # the score of a masked pair
TINY = 1e-30  # divisor of a row whose mask leaves nothing


def _attn(name, op, dtype, batch, heads, kv_heads, n, m, d, cap=0.0, slopes=False, causal=False, prefix=False, documents=0,
          lengths=False, radius=0, buckets=0):
    """cap: 0 is none; documents: how many are packed into a row (0: no document mask);
    radius, buckets: distances -radius .. radius (those beyond are the ends') map to that many buckets."""
    c = dict(op=op, dtype=dtype, batch=batch, heads=heads, kv_heads=kv_heads, n=n, m=m, d=d, cap=cap, slopes=slopes, causal=causal,
             prefix=prefix, documents=documents, lengths=lengths, radius=radius, buckets=buckets)
    return dict(c, name=name) if name else c


def listed():
    return [
        # LayerNorm of a short prompt's rows at the width of the MLP block of
        # this repository's benchmark: launches and latency count
        dict(name="layernorm_32x768_f16", op="layernorm", dtype="f16", m=32, d=768),
        # that MLP block's own LayerNorm, trained
        dict(name="layernorm_4096x768_f16", op="layernorm", dtype="f16", m=4096, d=768),
        # eight sequences of 197 tokens in fp32, at a width that no vector divides
        dict(name="layernorm_1576x1001_f32", op="layernorm", dtype="f32", m=1576, d=1001),
        # a long batch of a wide model
        dict(name="layernorm_16384x4096_bf16", op="layernorm", dtype="bf16", m=16384, d=4096),
        # one sequence's next token over a short cache, capped scores
        _attn("decode_512_f16", "attention", "f16", 1, 8, 8, 1, 512, 64, cap=20.0, lengths=True),
        # sixteen sequences' next tokens over caches of many lengths, four query heads to a key head
        _attn("decode_16x8192_bf16", "attention", "bf16", 16, 32, 8, 1, 8192, 128, lengths=True),
        # a prefix and its continuation, odd sizes, in fp32, biased by distance
        _attn("prefix_197x333_f32", "attention", "f32", 2, 3, 3, 197, 333, 40, slopes=True, causal=True, prefix=True),
        # a prompt of 4096 tokens, causal, capped scores, shared key heads
        _attn("prompt_4096_bf16", "attention", "bf16", 1, 16, 4, 4096, 4096, 128, cap=20.0, causal=True),
        # a row packed with eleven documents, causal inside each, trained
        _attn("documents_4000_f16", "attention_train", "f16", 1, 12, 12, 4000, 4000, 64, causal=True, documents=11),
        # a training step's attention at ordinary size, capped, shared key heads
        _attn("train_2048_bf16", "attention_train", "bf16", 2, 16, 4, 2048, 2048, 128, cap=20.0, causal=True),
        # an encoder with learned bucket bias, eight sequences of 512
        _attn("buckets_512_f16", "bucket_train", "f16", 8, 12, 12, 512, 512, 64, radius=128, buckets=32),
        # the same in fp32 on few odd rows, causal, with lengths
        _attn("buckets_77_f32", "bucket_train", "f32", 3, 4, 4, 77, 77, 32, causal=True, lengths=True, radius=64, buckets=16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("layernorm", "attention", "attention", "attention_train", "bucket_train"))
    dtype = rng.choice(("f32", "f16", "bf16", "f16", "bf16"))
    if op == "layernorm":
        d = _log(rng, 48, 8192)
        if rng.random() < 0.7:
            d = max(8, d // 8 * 8)
        m = _log(rng, 1, max(2, min(16384, 33554432 // d)))
        return dict(op=op, dtype=dtype, m=m, d=d)
    d = rng.choice((32, 40, 64, 64, 80, 96, 128, 128))
    kv = rng.choice((1, 2, 3, 4, 8))
    if op == "bucket_train":
        n = _log(rng, 20, 1024)
        batch = max(1, min(8, 2048 // n))
        r = rng.choice((16, 64, 128))
        return _attn(None, op, dtype, batch, kv, kv, n, n, d, causal=rng.random() < 0.4, lengths=rng.random() < 0.3, radius=r,
                     buckets=rng.choice((8, 16, 32)))
    group = rng.choice((1, 1, 2, 4))
    cap, slopes = rng.choice((0.0, 0.0, 20.0, 50.0)), rng.random() < 0.3
    if op == "attention" and rng.random() < 0.4:
        m = _log(rng, 64, 16384)
        return _attn(None, op, dtype, rng.choice((1, 2, 5, 16)), kv * group, kv, 1, m, d, cap=cap, slopes=slopes, lengths=True)
    m = _log(rng, 33, 1024 if dtype == "f32" else 3000)
    n = m if op == "attention_train" or rng.random() < 0.6 else _log(rng, 2, m)
    mask = rng.choice(("none", "causal", "causal", "prefix", "documents"))
    return _attn(None, op, dtype, rng.choice((1, 2)), kv * group, kv, n, m, d, cap=cap, slopes=slopes, causal=mask != "none",
                 prefix=mask == "prefix", documents=rng.choice((2, 5)) if mask == "documents" else 0)


# ---- what the inputs hold --------------------------------------------------


def _lengths(c):
    """Keys in use by each sequence: from few to all of the cache."""
    return [max(c["n"], c["m"] * (b + 1) // c["batch"]) for b in range(c["batch"])]


def _prefixes(c):
    return [c["m"] * (b + 1) // (2 * c["batch"] + 1) for b in range(c["batch"])]


def _documents(c):
    """Document of every key position: pieces of uneven lengths."""
    k = c["documents"]
    ends = [round(c["m"] * (i / k) ** 1.4) for i in range(1, k + 1)]
    return [sum(j >= e for e in ends) for j in range(c["m"])]


def _bucket_map(c):
    """Bucket of every distance -radius .. radius: one each near zero, then by the
    logarithm, keys before and after the query apart."""
    r, half = c["radius"], c["buckets"] // 2
    out = []
    for t in range(-r, r + 1):
        a, near = abs(t), max(1, half // 2)
        b = a if a < near else min(half - 1, near + int(math.log(a / near) / math.log(r / near) * (half - near)))
        out.append(b + (half if t > 0 else 0))
    return out


def _pairs(c):
    """Unmasked (query, key) pairs of one head, over the batch."""
    n, m = c["n"], c["m"]
    total = 0
    docs = _documents(c) if c["documents"] else None
    first = {}
    for j, x in enumerate(docs or ()):
        first.setdefault(x, j)
    for b in range(c["batch"]):
        size = _lengths(c)[b] if c["lengths"] else m
        off = size - n
        if not c["causal"]:
            total += n * size if docs is None else sum(docs[: size].count(docs[i + off]) for i in range(n))
            continue
        p = _prefixes(c)[b] if c["prefix"] else 0
        for i in range(n):
            end = min(size, max(i + off + 1, p))
            total += end - (first[docs[i + off]] if docs else 0)
    return total


def work(case):
    """Bytes: every input read once, every output written once.  Flops: the
    products over unmasked pairs (two forward, five backward); for LayerNorm
    what its sums and its normalization take."""
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "layernorm":
        m, d = case["m"], case["d"]
        return dict(bytes=e * (4 * m * d + 4 * d) + 8 * m, flops=20 * m * d)
    n, m, d, h = case["n"], case["m"], case["d"], case["heads"]
    q, kv = case["batch"] * h * n * d, case["batch"] * case["kv_heads"] * m * d
    if case["lengths"]:
        kv = sum(_lengths(case)) * case["kv_heads"] * d
    pairs = _pairs(case) * h
    if case["op"] == "attention":
        return dict(bytes=e * (2 * q + 2 * kv) + 4 * case["batch"] * h * n, flops=4 * pairs * d)
    return dict(bytes=e * (4 * q + 4 * kv) + 4 * case["batch"] * h * n, flops=14 * pairs * d)


def _tensors(case, seed):
    """The inputs by name, on the GPU, drawn from the seed alone."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = TORCH_DTYPE[case["dtype"]]

    def normal(*shape, mean=0.0, std=1.0):
        return (torch.randn(shape, generator=gen, device="cuda") * std + mean).to(t)

    def whole(values):
        return torch.tensor(values, dtype=torch.float32, device="cuda")

    if case["op"] == "layernorm":
        m, d = case["m"], case["d"]
        return dict(X=normal(m, d, mean=0.2, std=1.5), gamma=normal(d, mean=1.0, std=0.1), beta=normal(d, std=0.1), dY=normal(m, d))
    b, h, hk, n, m, d = (case[k] for k in ("batch", "heads", "kv_heads", "n", "m", "d"))
    x = dict(Q=normal(b, h, n, d, std=1.5), K=normal(b, hk, m, d, std=1.5), V=normal(b, hk, m, d))
    if case["op"] != "attention":
        x["dO"] = normal(b, h, n, d)
    if case["slopes"]:
        x["slopes"] = whole([2.0 ** (-8.0 * (i + 1) / h) for i in range(h)])
    if case["lengths"]:
        size = _lengths(case)
        order = torch.randperm(b, generator=gen, device="cuda").tolist()
        x["lengths"] = whole([size[i] for i in order])
    if case["prefix"]:
        x["prefix"] = whole(_prefixes(case))
    if case["documents"]:
        x["documents"] = whole(_documents(case)).expand(b, m).contiguous()
    if case["buckets"]:
        x["bucket"] = whole(_bucket_map(case))
        x["table"] = normal(h, case["buckets"])
    return x


_SIZES = ("batch", "heads", "kv_heads", "n", "m", "d", "cap", "slopes", "causal", "prefix", "documents", "lengths", "radius", "buckets")


def _bound(workload, x, sizes, dtype):
    from paper_2406_09465_amd import graphs
    from paper_2406_09465_amd.runner import PlanRunner
    w = graphs.build(workload, dtype=dtype, **sizes)
    r = PlanRunner(w, "fused")
    r.ins = [x[k] for k in w.input_names]
    return r.bind()


def prepare(case, seed):
    x = _tensors(case, seed)
    state = dict(case=case, x=x)
    if own:
        if case["op"] == "layernorm":
            sizes = dict(m=case["m"], d=case["d"], eps=EPS)
            pair = ("layernorm", "layernorm_grad")
        else:
            sizes = {k: case[k] for k in _SIZES}
            sizes["documents"] = bool(case["documents"])
            pair = ("mha", "mha_grad")
        fwd = _bound(pair[0], x, sizes, case["dtype"])
        state["plans"] = [fwd]
        if case["op"] != "attention":
            saved = dict(zip(fwd.w.output_names, fwd.outs))
            state["plans"].append(_bound(pair[1], {**x, **saved}, sizes, case["dtype"]))
    return state


def run(state):
    if own:
        out = []
        for r in state["plans"]:
            r.launch_bound()
            out += r.outs
        return out
    t = TORCH_DTYPE[state["case"]["dtype"]]
    if state["case"]["op"] == "layernorm":
        y, mu, r, dx, dg, db = _layernorm({k: v.float() for k, v in state["x"].items()})
        return [y.to(t), mu, r, dx.to(t), dg.to(t), db.to(t)]
    o, lse, *grads = _attention(state["case"], {k: v.float() for k, v in state["x"].items()})
    return [o.to(t), lse] + [g.to(t) for g in grads]


# ---- the plain form: elementary operations in 32 bits ----------------------


def _layernorm(x):
    X, gamma, dY = x["X"], x["gamma"], x["dY"]
    mu = X.mean(-1, keepdim=True)
    D = X - mu
    r = 1.0 / torch.sqrt((D * D).mean(-1, keepdim=True) + EPS)
    xh = D * r
    g = dY * gamma
    dX = r * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))
    return xh * gamma + x["beta"], mu, r, dX, (dY * xh).sum(0), dY.sum(0)


def _attention(c, x):
    b, h, hk, n, m, d = (c[k] for k in ("batch", "heads", "kv_heads", "n", "m", "d"))
    Q = x["Q"].reshape(b, hk, h // hk * n, d)
    K, V = x["K"], x["V"]
    dev = Q.device
    s0 = (Q @ K.transpose(2, 3).contiguous()).reshape(b, h, n, m) * (1.0 / math.sqrt(d))
    th = None
    if c["cap"]:
        th = torch.tanh(s0 * (1.0 / c["cap"]))
        s0 = th * c["cap"]
    key = torch.arange(m, device=dev, dtype=torch.float32)
    end = x["lengths"] if c["lengths"] else torch.full((b,), float(m), device=dev)
    pos = end[:, None] - n + torch.arange(n, device=dev, dtype=torch.float32)  # the queries are the last n positions
    rel = key - pos[:, :, None]
    if c["slopes"]:
        s0 = s0 - x["slopes"][:, None, None] * rel.abs()[:, None]
    which = None
    if c["buckets"]:
        which = x["bucket"][(rel + c["radius"]).clamp(0, 2 * c["radius"]).long()].long()
        s0 = s0 + x["table"][:, which].transpose(0, 1)
    mask = torch.ones(b, n, m, dtype=torch.bool, device=dev)
    if c["causal"]:
        mask = rel <= 0
        if c["prefix"]:
            mask = mask | (key < x["prefix"][:, None])[:, None]
    if c["documents"]:
        doc = x["documents"]
        mask = mask & (doc[:, None] == doc.gather(1, pos.long())[:, :, None])
    if c["lengths"]:
        mask = mask & (key < end[:, None])[:, None]
        V = V * (key < end[:, None])[:, None, :, None]
    mask = mask[:, None]
    top = torch.where(mask, s0, LOW).amax(-1, keepdim=True)
    e = torch.where(mask, torch.exp(s0 - top), 0.0)
    l = e.sum(-1, keepdim=True)
    p = e / l.clamp(min=TINY)
    del e
    group = (b, hk, h // hk * n, -1)
    o = (p.reshape(group) @ V).reshape(b, h, n, d)
    lse = torch.where(l > 0, top + torch.log(l.clamp(min=TINY)), 0.0)
    if c["op"] == "attention":
        return o, lse
    dO = x["dO"]
    dp = (dO.reshape(group) @ V.transpose(2, 3).contiguous()).reshape(b, h, n, m)
    ds = p * (dp - (dO * o).sum(-1, keepdim=True))
    del dp
    out = []
    if c["buckets"]:
        ids = which[:, None].expand(b, h, n, m).transpose(0, 1).reshape(h, -1)
        out = [torch.zeros(h, c["buckets"], device=dev).scatter_add(1, ids, ds.transpose(0, 1).reshape(h, -1))]
    if c["cap"]:
        ds = ds * (1.0 - th * th)
    ds = ds * (1.0 / math.sqrt(d))
    dq = (ds.reshape(group) @ K).reshape(b, h, n, d)
    dk = ds.reshape(group).transpose(2, 3).contiguous() @ Q
    dv = p.reshape(group).transpose(2, 3).contiguous() @ dO.reshape(group)
    if c["lengths"]:
        dv = dv * (key < end[:, None])[:, None, :, None]
    return [o, lse, dq, dk, dv] + out


# ---- the definitions in 64 bits, head by head -------------------------------


def exact(case, seed):
    x = {k: v.double() for k, v in _tensors(case, seed).items()}
    if case["op"] == "layernorm":
        X = x["X"]
        var, mu = torch.var_mean(X, -1, unbiased=False, keepdim=True)
        r = (var + EPS) ** -0.5
        n = (X - mu) * r
        g = x["dY"] * x["gamma"]
        w = X.shape[1]
        dx = (g - (g.sum(1, True) + n * (g * n).sum(1, True)) / w) * r
        return [torch.addcmul(x["beta"], n, x["gamma"]), mu, r, dx, (x["dY"] * n).sum(0), x["dY"].sum(0)]
    B, H, N, M, D = (case[k] for k in ("batch", "heads", "n", "m", "d"))
    rep = H // case["kv_heads"]
    q, k, v = x["Q"], x["K"], x["V"]
    o, lse = torch.zeros_like(q), torch.zeros(B, H, N, 1, dtype=torch.float64, device=q.device)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    dt = torch.zeros_like(x["table"]) if case["buckets"] else None
    j = torch.arange(M, device=q.device)
    for b in range(B):
        size = int(x["lengths"][b]) if case["lengths"] else M
        i = torch.arange(size - N, size, device=q.device)
        dist = j[None, :] - i[:, None]
        allowed = j[None, :].expand(N, M) < size
        if case["causal"]:
            ok = dist <= 0
            if case["prefix"]:
                ok = ok | (j[None, :] < int(x["prefix"][b]))
            allowed = allowed & ok
        if case["documents"]:
            doc = x["documents"][b].long()
            allowed = allowed & (doc[i][:, None] == doc[None, :])
        if case["buckets"]:
            r = case["radius"]
            ids = x["bucket"].long()[dist.clamp(-r, r) + r]
        for h in range(H):
            kh, vh = k[b, h // rep], v[b, h // rep]
            z = torch.mm(q[b, h], kh.t().contiguous()) / math.sqrt(D)
            slope = 1.0 / math.sqrt(D)
            if case["cap"]:
                th = torch.tanh(z / case["cap"])
                z, slope = case["cap"] * th, slope * (1 - th ** 2)
            if case["slopes"]:
                z = z - x["slopes"][h] * dist.abs()
            if case["buckets"]:
                z = z + x["table"][h][ids]
            z = z.masked_fill(~allowed, -math.inf)
            ls = torch.logsumexp(z, 1, keepdim=True)
            some = torch.isfinite(ls)
            p = torch.exp(z - torch.where(some, ls, torch.zeros_like(ls)))
            o[b, h] = p @ vh
            lse[b, h] = torch.where(some, ls, torch.zeros_like(ls))
            if case["op"] == "attention":
                continue
            g = x["dO"][b, h]
            dp = torch.mm(g, vh.t().contiguous())
            dz = p * (dp - (p * dp).sum(1, keepdim=True))
            if case["buckets"]:
                dt[h] += torch.bincount(ids.reshape(-1), dz.reshape(-1), minlength=case["buckets"])
            dz = dz * slope
            dq[b, h] = dz @ kh
            dk[b, h // rep] += dz.t().contiguous() @ q[b, h]
            dv[b, h // rep] += p.t().contiguous() @ g
    if case["op"] == "attention":
        return [o, lse]
    return [o, lse, dq, dk, dv] + ([dt] if case["buckets"] else [])
