"""Performance cases of the operators around an image or video transformer's
training step.

* ``groupnorm``: group norm with an activation, channels last, that keeps its
  statistics; ``groupnorm_train``: with its gradient;
* ``rotary``: rotary positions with several axes (time, height, width) of
  queries and keys, as they lie or out of the packed product of a projection;
  ``rotary_train``: with its gradient;
* ``clip``: the global norm of many gradients, and the gradients clipped by it.

With ``own`` false the operators run in their plain form (elementary torch
operations in 32 bits; angles and the global norm in 64); with ``own`` true as
the framework's plans, through the calls a training or serving loop makes
(``graphs.build``, ``PlanRunner``, ``bind``, ``launch_bound``).
"""

import math

import torch

own = False

TORCH_DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-5        # of a variance
CLIP_EPS = 1e-6   # beside the global norm


def _norm(name, op, dtype, batch, hh, ww, c, groups, act):
    x = dict(op=op, dtype=dtype, batch=batch, hh=hh, ww=ww, c=c, groups=groups, act=act)
    return dict(x, name=name) if name else x


def _rot(name, op, dtype, batch, heads, kv_heads, n, d, rot, axes, interleaved=False, packed=False, first=0, step=1.0):
    """rot: dims of a head that turn; first: position of the first token; step: from one position to the next."""
    x = dict(op=op, dtype=dtype, batch=batch, heads=heads, kv_heads=kv_heads, n=n, d=d, rot=rot, axes=axes, interleaved=interleaved,
             packed=packed, first=first, step=step)
    return dict(x, name=name) if name else x


def _clip(name, dtype, layers, width, hidden, odd=False, limit=1.0):
    """Gradients of ``layers`` layers (``odd``: and of tensors of odd sizes, one element among them)."""
    x = dict(op="clip", dtype=dtype, layers=layers, width=width, hidden=hidden, odd=odd, limit=limit)
    return dict(x, name=name) if name else x


def listed():
    return [
        # the smallest map of a denoising network at one image: launches and latency count
        _norm("groupnorm_16x16x320_f16", "groupnorm", "f16", 1, 16, 16, 320, 32, "silu"),
        # the widest map of such a network, eight images, trained; ten channels to a group
        _norm("groupnorm_8x64x64x320_bf16", "groupnorm_train", "bf16", 8, 64, 64, 320, 32, "silu"),
        # maps of odd sizes in fp32, six channels to a group
        _norm("groupnorm_2x131x77x30_f32", "groupnorm_train", "f32", 2, 131, 77, 30, 5, "relu"),
        # what the convolution of this repository's benchmark leaves, four images, trained
        _norm("groupnorm_4x416x416x64_f16", "groupnorm_train", "f16", 4, 416, 416, 64, 16, "silu"),
        # sixteen sequences' next tokens, out of the projection's packed product
        _rot("rotary_16x1_bf16", "rotary", "bf16", 16, 32, 8, 1, 128, 128, 3, packed=True, first=5000),
        # two images of 64 x 64 patches, two axes, trained
        _rot("rotary_2x4096_f16", "rotary_train", "f16", 2, 12, 12, 4096, 64, 64, 2),
        # odd sizes in fp32, neighbouring pairs, part of a head, far positions between whole numbers
        _rot("rotary_3x1001_f32", "rotary_train", "f32", 3, 5, 5, 1001, 80, 48, 1, interleaved=True, first=900000, step=0.25),
        # two videos of 16 x 24 x 24 patches, four query heads to a key head, packed, trained
        _rot("rotary_2x9216_bf16", "rotary_train", "bf16", 2, 32, 8, 9216, 128, 128, 3, packed=True),
        # the gradients of one small layer: launches and latency count
        _clip("clip_1x128_f32", "f32", 1, 128, 320),
        # six layers of the width of this repository's MLP block
        _clip("clip_6x768_bf16", "bf16", 6, 768, 2048),
        # tensors of odd sizes, few of them a whole vector
        _clip("clip_odd_f32", "f32", 2, 333, 1001, odd=True),
        # layers of a wide model: two hundred million gradients
        _clip("clip_7x1920_bf16", "bf16", 7, 1920, 5184),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("norm", "norm", "rotary", "rotary", "clip"))
    dtype = rng.choice(("f32", "f16", "bf16", "f16", "bf16"))
    if kind == "norm":
        groups = rng.choice((1, 2, 5, 8, 16, 32, 32))
        per = _log(rng, 1, min(64, 2048 // groups))
        c = groups * per
        side = _log(rng, 4, 416)
        while side * side * c > 11000000:
            side = max(4, side * 2 // 3)
        other = max(1, round(side * rng.uniform(0.5, 1.0)))
        batch = max(1, min(_log(rng, 1, 16), 40000000 // (side * other * c)))
        return _norm(None, rng.choice(("groupnorm", "groupnorm_train")), dtype, batch, side, other, c, groups, rng.choice(("none", "relu", "silu", "silu")))
    if kind == "rotary":
        d = rng.choice((32, 48, 64, 64, 80, 96, 128, 128))
        axes = rng.choice((1, 2, 2, 3, 3))
        rot = rng.choice((d, d, d // 2))
        kv = rng.choice((1, 2, 3, 5, 8))
        heads = kv * rng.choice((1, 1, 2, 4))
        op = rng.choice(("rotary", "rotary_train"))
        batch = rng.choice((1, 2, 5, 16))
        n = 1 if op == "rotary" and rng.random() < 0.4 else _log(rng, 2, max(3, min(9216, 90000000 // (batch * (heads + 2 * kv) * d))))
        return _rot(None, op, dtype, batch, heads, kv, n, d, rot, axes, interleaved=rng.random() < 0.3, packed=rng.random() < 0.5,
                    first=rng.choice((0, 0, _log(rng, 10, 1000000))), step=rng.choice((1.0, 1.0, 0.5)))
    width = _log(rng, 16, 1920)
    if rng.random() < 0.6:
        width = max(16, width // 16 * 16)
    hidden = max(8, round(width * rng.uniform(1.0, 2.7)))
    return _clip(None, dtype, rng.randint(1, 7), width, hidden, odd=rng.random() < 0.3, limit=rng.choice((0.5, 1.0, 1.0, 1e5)))


# ---- what the inputs hold --------------------------------------------------


def _pieces(c):
    """(shape, whether a norm's weight or a bias, whose gradients are fp32) of every gradient."""
    w, h = c["width"], c["hidden"]
    out = []
    for _ in range(c["layers"]):
        out += [((w,), True), ((w,), True), ((w, w + w // 2), False), ((w, w), False), ((w,), True), ((w,), True), ((w, h), False), ((h, w), False)]
    if c["odd"]:
        out += [((1,), True), ((77,), False), ((5, 7, 3), False), ((1,), False), ((333, 41), True)]
    return out


def _sections(c):
    """Which axis every pair of a head turns by: as even a share each as there is, in order."""
    pairs = c["rot"] // 2
    return [i * c["axes"] // pairs for i in range(pairs)]


def _frequencies(c):
    """Radians per position of every pair: 10000^(-place in its axis' share)."""
    at = _sections(c)
    out = []
    for i, a in enumerate(at):
        out.append(10000.0 ** (-(i - at.index(a)) / at.count(a)))
    return out


def _grid(c):
    """Position of every token along every axis: frames of rows of patches, row by row."""
    side = max(1, round(c["n"] ** (1 / c["axes"])))
    out = []
    for i in range(c["n"]):
        place = []
        for _ in range(c["axes"] - 1):
            place.append(i % side)
            i //= side
        place.append(i)
        out.append([c["first"] + c["step"] * p for p in reversed(place)])
    return out


def work(case):
    """Bytes: every input read once, every output written once.  Flops: what
    sums, normalization, activation and rotation take."""
    e = 4 if case["dtype"] == "f32" else 2
    op = case["op"]
    if op.startswith("groupnorm"):
        n = case["batch"] * case["hh"] * case["ww"] * case["c"]
        train = op == "groupnorm_train"
        return dict(bytes=(5 if train else 2) * n * e + (6 if train else 2) * case["c"] * e + 16 * case["batch"] * case["groups"], flops=(30 if train else 10) * n)
    if op.startswith("rotary"):
        heads = case["heads"] + (2 if case["packed"] else 1) * case["kv_heads"]
        n = case["batch"] * heads * case["n"] * case["d"]
        passes = 2 if op == "rotary_train" else 1
        return dict(bytes=passes * (2 * n * e + 4 * case["batch"] * case["n"] * case["axes"] + 4 * case["rot"]), flops=passes * 3 * n)
    sizes = [(math.prod(s), 4 if vector else e) for s, vector in _pieces(case)]
    return dict(bytes=sum(2 * n * b for n, b in sizes) + 4, flops=sum(3 * n for n, _ in sizes))


def _tensors(case, seed):
    """The inputs by name, on the GPU, drawn from the seed alone."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = TORCH_DTYPE[case["dtype"]]

    def normal(*shape, mean=0.0, std=1.0, dtype=t):
        return (torch.randn(shape, generator=gen, device="cuda") * std + mean).to(dtype)

    op = case["op"]
    if op.startswith("groupnorm"):
        b, hh, ww, c = (case[k] for k in ("batch", "hh", "ww", "c"))
        at = torch.randn(c, generator=gen, device="cuda") * 0.5  # channels differ in their means
        x = dict(X=(torch.randn((b, hh, ww, c), generator=gen, device="cuda") * 1.5 + at).to(t), gamma=normal(c, mean=1.0, std=0.2), beta=normal(c, std=0.2))
        if op == "groupnorm_train":
            x["dY"] = normal(b, hh, ww, c)
        return x
    if op.startswith("rotary"):
        b, h, hk, n, d = (case[k] for k in ("batch", "heads", "kv_heads", "n", "d"))
        x = {}
        if case["packed"]:
            x["QKV"] = normal(b, n, h + 2 * hk, d)
        else:
            x["Q"], x["K"] = normal(b, h, n, d), normal(b, hk, n, d)
        if op == "rotary_train":
            x["dQr"], x["dKr"] = normal(b, h, n, d), normal(b, hk, n, d)
            if case["packed"]:
                x["dV"] = normal(b, hk, n, d)
        place = torch.tensor(_grid(case), dtype=torch.float32, device="cuda")
        # sequences of a batch start at places of their own
        first = torch.randint(0, 64, (b, 1, 1), generator=gen, device="cuda").float()
        x["positions"] = (place[None] + first).contiguous()
        x["freq"] = torch.tensor(_frequencies(case), dtype=torch.float32, device="cuda")
        if case["axes"] > 1:
            x["axis"] = torch.tensor(_sections(case), dtype=torch.float32, device="cuda")
        return x
    out = {}
    for i, (shape, vector) in enumerate(_pieces(case)):
        out[f"G{i}"] = normal(*shape, std=10.0 ** (-3 + i % 3), dtype=torch.float32 if vector else t)
    return out


def _bound(workload, x, **sizes):
    from paper_2406_09465_amd import graphs
    from paper_2406_09465_amd.runner import PlanRunner
    w = graphs.build(workload, **sizes)
    r = PlanRunner(w, "fused")
    r.ins = [x[k] for k in w.input_names]
    return r.bind()


def prepare(case, seed):
    x = _tensors(case, seed)
    state = dict(case=case, x=x)
    if own:
        op = case["op"]
        if op == "clip":
            pieces = _pieces(case)
            state["plans"] = [_bound("grad_clip", x, shapes=[s for s, _ in pieces], dtypes=["f32" if v else case["dtype"] for _, v in pieces],
                                     max_norm=case["limit"], eps=CLIP_EPS)]
            return state
        if op.startswith("groupnorm"):
            name, sizes = "groupnorm", {k: case[k] for k in ("batch", "hh", "ww", "c", "groups", "act", "dtype")}
            sizes["eps"] = EPS
        else:
            name, sizes = "rotary", {k: case[k] for k in ("batch", "heads", "kv_heads", "n", "d", "rot", "axes", "interleaved", "packed", "dtype")}
        fwd = _bound(name, x, **sizes)
        state["plans"] = [fwd]
        if op.endswith("_train"):
            saved = dict(zip(fwd.w.output_names, fwd.outs))
            state["plans"].append(_bound(name + "_grad", {**x, **saved}, **sizes))
    return state


def run(state):
    if own:
        out = []
        for r in state["plans"]:
            r.launch_bound()
            out += r.outs
        return out
    c, x = state["case"], state["x"]
    t = TORCH_DTYPE[c["dtype"]]
    if c["op"].startswith("groupnorm"):
        return _groupnorm(c, {k: v.float() for k, v in x.items()}, t)
    if c["op"].startswith("rotary"):
        return _rotary(c, x, t)
    return _clipped(c, list(x.values()))


# ---- the plain form: elementary operations in 32 bits ----------------------


def _groupnorm(c, x, t):
    b, g = c["batch"], c["groups"]
    per = c["c"] // g
    X = x["X"].reshape(b, -1, g, per)
    gamma, beta = x["gamma"].reshape(g, per), x["beta"].reshape(g, per)
    mu = X.mean((1, 3), keepdim=True)
    D = X - mu
    r = 1.0 / torch.sqrt((D * D).mean((1, 3), keepdim=True) + EPS)
    xh = D * r
    z = xh * gamma + beta
    s = 1.0 / (1.0 + torch.exp(-z)) if c["act"] == "silu" else None
    y = z * s if c["act"] == "silu" else torch.where(z > 0, z, 0.0) if c["act"] == "relu" else z
    out = [y.reshape(x["X"].shape).to(t), mu.reshape(b, g), r.reshape(b, g)]
    if c["op"] == "groupnorm":
        return out
    dz = x["dY"].reshape(X.shape)
    if c["act"] == "silu":
        dz = dz * (s * (1.0 + z * (1.0 - s)))
    elif c["act"] == "relu":
        dz = torch.where(z > 0, dz, 0.0)
    gr = dz * gamma
    dX = r * (gr - gr.mean((1, 3), keepdim=True) - xh * (gr * xh).mean((1, 3), keepdim=True))
    return out + [dX.reshape(x["X"].shape).to(t), (dz * xh).sum((0, 1)).reshape(-1).to(t), dz.sum((0, 1)).reshape(-1).to(t)]


def _turn(c, X, co, si):
    """X [batch, heads, n, d] in 32 bits, turned."""
    p = c["rot"] // 2
    turned, rest = X[..., : 2 * p], X[..., 2 * p:]
    if c["interleaved"]:
        pair = turned.reshape(*turned.shape[:-1], p, 2)
        a, b = pair[..., 0], pair[..., 1]
        out = torch.stack((a * co - b * si, b * co + a * si), -1).reshape(turned.shape)
    else:
        a, b = turned[..., :p], turned[..., p:]
        out = torch.cat((a * co - b * si, b * co + a * si), -1)
    return torch.cat((out, rest), -1)


def _rotary(c, x, t):
    h, hk = c["heads"], c["kv_heads"]
    place = x["positions"].double()
    if c["axes"] > 1:
        place = place[..., x["axis"].long()]
    angle = place * x["freq"].double()  # 64 bits: 32 lose the angles of far positions
    co, si = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    if c["packed"]:
        q, k, v = x["QKV"].transpose(1, 2).split((h, hk, hk), 1)
        out = [_turn(c, q.float(), co, si).to(t), _turn(c, k.float(), co, si).to(t), v.contiguous()]
    else:
        out = [_turn(c, x["Q"].float(), co, si).to(t), _turn(c, x["K"].float(), co, si).to(t)]
    if c["op"] == "rotary":
        return out
    dq, dk = _turn(c, x["dQr"].float(), co, -si).to(t), _turn(c, x["dKr"].float(), co, -si).to(t)
    if c["packed"]:
        return out + [torch.cat((dq, dk, x["dV"]), 1).transpose(1, 2).contiguous()]
    return out + [dq, dk]


def _clipped(c, grads):
    norm = torch.sqrt(sum((g.double() * g.double()).sum() for g in grads)).float().reshape(1)  # 64 bits: a long sum
    scale = torch.clamp(c["limit"] / (norm + CLIP_EPS), max=1.0)
    return [norm] + [(g.float() * scale).to(g.dtype) for g in grads]


# ---- the definitions in 64 bits ---------------------------------------------


def exact(case, seed):
    x = {k: v.double() for k, v in _tensors(case, seed).items()}
    if case["op"].startswith("groupnorm"):
        return _exact_groupnorm(case, x)
    if case["op"].startswith("rotary"):
        return _exact_rotary(case, x)
    total = math.sqrt(sum(float(torch.dot(g.flatten(), g.flatten())) for g in x.values()))
    scale = min(1.0, case["limit"] / (total + CLIP_EPS))
    return [torch.tensor([total], dtype=torch.float64, device="cuda")] + [g * scale for g in x.values()]


def _exact_groupnorm(case, x):
    """Image by image and group by group."""
    B, G = case["batch"], case["groups"]
    per = case["c"] // G
    X = x["X"]
    Y, mu, r = torch.empty_like(X), torch.empty((B, G), dtype=torch.float64, device="cuda"), torch.empty((B, G), dtype=torch.float64, device="cuda")
    train = case["op"] == "groupnorm_train"
    dX, dgamma, dbeta = torch.empty_like(X), torch.zeros_like(x["gamma"]), torch.zeros_like(x["beta"])
    for b in range(B):
        for k in range(G):
            at = slice(k * per, (k + 1) * per)
            part = X[b, :, :, at]
            var, mean = torch.var_mean(part, unbiased=False)
            rs = (var + EPS) ** -0.5
            mu[b, k], r[b, k] = mean, rs
            n = (part - mean) * rs
            z = torch.addcmul(x["beta"][at], n, x["gamma"][at])
            if case["act"] == "silu":
                sg = torch.sigmoid(z)
                Y[b, :, :, at] = z * sg
                slope = sg + z * sg * (1 - sg)
            elif case["act"] == "relu":
                Y[b, :, :, at] = z.clamp(min=0)
                slope = (z > 0).double()
            else:
                Y[b, :, :, at] = z
                slope = None
            if not train:
                continue
            d = x["dY"][b, :, :, at] if slope is None else x["dY"][b, :, :, at] * slope
            dbeta[at] += d.sum((0, 1))
            dgamma[at] += (d * n).sum((0, 1))
            d = d * x["gamma"][at]
            count = d.numel()
            dX[b, :, :, at] = (d - (d.sum() + n * (d * n).sum()) / count) * rs
    return [Y, mu, r] + ([dX, dgamma, dbeta] if train else [])


def _exact_rotary(case, x):
    """Pairs as complex numbers times e^(i angle)."""
    h, hk, p = case["heads"], case["kv_heads"], case["rot"] // 2
    place = x["positions"]
    if case["axes"] > 1:
        place = place.index_select(2, x["axis"].long())
    e = torch.polar(torch.ones((), dtype=torch.float64, device="cuda").expand(place.shape).contiguous(), place * x["freq"]).unsqueeze(1)

    def times(X, factor):
        out = X.clone()
        first = slice(0, 2 * p, 2) if case["interleaved"] else slice(0, p)
        second = slice(1, 2 * p, 2) if case["interleaved"] else slice(p, 2 * p)
        w = torch.complex(X[..., first].contiguous(), X[..., second].contiguous()) * factor
        out[..., first], out[..., second] = w.real, w.imag
        return out

    if case["packed"]:
        heads = x["QKV"].permute(0, 2, 1, 3).contiguous()
        out = [times(heads[:, :h], e), times(heads[:, h:h + hk], e), heads[:, h + hk:]]
    else:
        out = [times(x["Q"], e), times(x["K"], e)]
    if case["op"] == "rotary":
        return out
    back = [times(x["dQr"], e.conj()), times(x["dKr"], e.conj())]
    if case["packed"]:
        return out + [torch.cat(back + [x["dV"]], 1).permute(0, 2, 1, 3)]
    return out + back
