"""LayerNorm's gradient and attention of any length with its gradient on the
GPU, against plain float64 forms with bounds counted from the definitions."""

import numpy as np
import pytest

from paper_2406_09465_amd import graphs

from . import layer_ref as ref

pytestmark = pytest.mark.gpu


def _run(w, x, plan="fused"):
    from paper_2406_09465_amd.runner import PlanRunner
    r = PlanRunner(w, plan)
    out = r.run(x)
    return out


def _check(out, want, dtype, f32=()):
    for k, (v, b) in want.items():
        if k in out:
            worst = ref.outside(out[k], v, b, "f32" if k in f32 else dtype)
            assert worst <= 1.0, (k, worst)


LN = [("f32", 5, 8), ("f32", 37, 77), ("f16", 1, 768), ("f16", 300, 768), ("bf16", 129, 1024), ("f16", 1000, 100), ("bf16", 41, 250),
      ("f16", 19, 333), ("f32", 70, 4096), ("bf16", 33, 8192), ("f32", 9, 2), ("f16", 12, 16384)]


@pytest.mark.parametrize("dtype,m,d", LN)
def test_layernorm_and_gradient(dtype, m, d):
    rng = np.random.default_rng(m * 1000 + d)
    x, s = {}, {}
    for n, sh, mean, std in (("X", (m, d), 0.4, 1.5), ("gamma", (d,), 1.0, 0.2), ("beta", (d,), 0.0, 0.2), ("dY", (m, d), 0.0, 1.0)):
        x[n], s[n] = ref.rounded(rng.normal(mean, std, sh), dtype)
    want = ref.layernorm(x["X"], x["gamma"], x["beta"], x["dY"], 1e-5, dtype)
    out = _run(graphs.build("layernorm", m=m, d=d, dtype=dtype), s)
    _check(out, want, dtype, ("mu", "r"))
    s["mu"], s["r"] = out["mu"].astype(np.float32), out["r"].astype(np.float32)
    for plan in ("fused", "layered"):
        _check(_run(graphs.build("layernorm_grad", m=m, d=d, dtype=dtype), s, plan), want, dtype)


def _inputs(dtype, batch, heads, kv_heads, n, m, d, slopes=False, prefix=(), documents=None, lengths=(), radius=0, buckets=0, grad=False, seed=0):
    rng = np.random.default_rng(seed)
    x, s = {}, {}
    for name, shape, std in (("Q", (batch, heads, n, d), 1.5), ("K", (batch, kv_heads, m, d), 1.0), ("V", (batch, kv_heads, m, d), 1.0),
                             ("dO", (batch, heads, n, d), 1.0)):
        x[name], s[name] = ref.rounded(rng.normal(0, std, shape), dtype)
    if slopes:
        x["slopes"], s["slopes"] = ref.rounded(2.0 ** -(1.0 + np.arange(heads)), "f32")
    if len(prefix):
        x["prefix"], s["prefix"] = ref.rounded(np.array(prefix), "f32")
    if documents is not None:
        x["documents"], s["documents"] = ref.rounded(np.array(documents), "f32")
    if len(lengths):
        x["lengths"], s["lengths"] = ref.rounded(np.array(lengths), "f32")
    if radius:
        x["bucket"], s["bucket"] = ref.rounded(ref.bucket_map(radius, buckets), "f32")
        x["table"], s["table"] = ref.rounded(rng.normal(0, 1, (heads, buckets)), dtype)
    return x, s


def _docs(batch, m, k, seed):
    """Documents in no order: a number comes again later."""
    rng = np.random.default_rng(seed)
    return np.repeat(rng.integers(0, k, (batch, (m + 6) // 7)), 7, axis=1)[:, :m]


FWD = [
    dict(dtype="f32", n=7, d=8),
    dict(dtype="f16", n=50, d=64),
    dict(dtype="bf16", n=130, d=40, heads=3),
    dict(dtype="f16", n=200, d=128, heads=4, kv_heads=2, causal=True),
    dict(dtype="bf16", n=257, d=80, causal=True, cap=5.0, batch=2),
    dict(dtype="f32", n=33, m=100, d=24, causal=True, slopes=True, heads=4, kv_heads=1),
    dict(dtype="f16", n=65, m=190, d=64, causal=True, prefix=(100, 3), batch=2, heads=4, kv_heads=4),
    dict(dtype="bf16", n=300, d=32, docs=3, batch=2),
    dict(dtype="f32", n=150, d=32, docs=40, causal=True, heads=2, kv_heads=1),
    dict(dtype="f16", n=1, m=1, d=64),
    dict(dtype="f16", n=1, m=3, d=64, heads=8, kv_heads=2),
    dict(dtype="bf16", n=1, m=1000, d=128, heads=8, kv_heads=2, lengths=(1000, 1, 313), batch=3),
    dict(dtype="f16", n=1, m=5000, d=64, heads=4, kv_heads=4, lengths=(64, 4097), batch=2, cap=10.0, slopes=True),
    dict(dtype="f32", n=1, m=700, d=48, heads=6, kv_heads=3, lengths=(512,)),
    dict(dtype="bf16", n=3, m=500, d=64, heads=4, kv_heads=1, lengths=(300, 40), batch=2, causal=True),
    dict(dtype="f16", n=90, d=256, heads=2, kv_heads=1, causal=True),
    dict(dtype="f16", n=100, d=32, radius=16, buckets=8, heads=3),
    dict(dtype="bf16", n=70, m=300, d=64, radius=5, buckets=32, heads=4, kv_heads=2, causal=True),
    dict(dtype="f32", n=40, d=16, radius=100, buckets=7, heads=2, lengths=(40, 33), batch=2, n_=33),
    dict(dtype="bf16", n=700, m=2100, d=128, heads=2, kv_heads=2),
]


def _unpack(c, grad=False):
    c = dict(c)
    n = c.pop("n_", c.pop("n"))
    c.pop("n", None)
    m = c.pop("m", max([n] + [int(v) for v in c.get("lengths", ())]))
    batch, heads = c.pop("batch", 1), c.pop("heads", 2)
    kv = c.pop("kv_heads", heads)
    d, dtype, docs = c.pop("d"), c.pop("dtype"), c.pop("docs", 0)
    cap, causal = c.pop("cap", 0.0), c.pop("causal", False)
    documents = _docs(batch, m, docs, n) if docs else None
    x, s = _inputs(dtype, batch, heads, kv, n, m, d, documents=documents, seed=n + d, **c)
    sizes = dict(batch=batch, heads=heads, kv_heads=kv, n=n, m=m, d=d, dtype=dtype, cap=cap, causal=causal, slopes=c.get("slopes", False),
                 prefix=bool(c.get("prefix")), documents=bool(docs), lengths=bool(c.get("lengths")), radius=c.get("radius", 0),
                 buckets=c.get("buckets", 0))
    want = ref.attention(x, dtype, heads, kv, cap=cap, causal=causal, radius=c.get("radius", 0), grad=grad)
    return sizes, x, s, want


@pytest.mark.parametrize("case", FWD, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items() if k != "lengths"))
def test_attention(case):
    sizes, x, s, want = _unpack(case)
    _check(_run(graphs.build("mha", **sizes), s), want, sizes["dtype"], ("L",))


GRAD = [
    dict(dtype="f32", n=7, d=8),
    dict(dtype="f16", n=50, d=64),
    dict(dtype="bf16", n=130, d=40, heads=3, cap=4.0),
    dict(dtype="f16", n=200, d=128, heads=4, kv_heads=2, causal=True),
    dict(dtype="f32", n=33, m=100, d=24, causal=True, slopes=True, heads=4, kv_heads=1),
    dict(dtype="f16", n=65, m=190, d=64, causal=True, prefix=(100, 3), batch=2, heads=4, kv_heads=4),
    dict(dtype="bf16", n=300, d=32, docs=3, batch=2),
    dict(dtype="f32", n=150, d=32, docs=40, causal=True, heads=2, kv_heads=1, cap=3.0),
    dict(dtype="bf16", n=3, m=500, d=64, heads=4, kv_heads=1, lengths=(300, 40), batch=2, causal=True),
    dict(dtype="f16", n=90, d=256, heads=2, kv_heads=1, causal=True),
    dict(dtype="f16", n=1, m=1, d=64),
    dict(dtype="f16", n=100, d=32, radius=16, buckets=8, heads=3, batch=2),
    dict(dtype="bf16", n=70, m=300, d=64, radius=5, buckets=32, heads=4, kv_heads=2, causal=True),
    dict(dtype="f32", n=33, m=40, d=16, radius=100, buckets=7, heads=2, lengths=(40, 33), batch=2),
    dict(dtype="bf16", n=260, m=1100, d=128, heads=2, kv_heads=2),
]


@pytest.mark.parametrize("case", GRAD, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items() if k != "lengths"))
def test_attention_gradient(case):
    sizes, x, s, want = _unpack(case, grad=True)
    out = _run(graphs.build("mha", **sizes), s)
    _check(out, want, sizes["dtype"], ("L",))
    _, s["O"] = ref.rounded(out["O"], sizes["dtype"])
    s["L"] = out["L"].astype(np.float32)
    _check(_run(graphs.build("mha_grad", **sizes), s), want, sizes["dtype"])


@pytest.mark.parametrize("case", [c for c in GRAD if c["n"] * c.get("m", c["n"]) <= 70 * 300 and c.get("m", c["n"]) > 1],
                         ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items() if k != "lengths"))
def test_one_kernel_per_primitive(case):
    """The unfused plans store every tensor: sixteen-bit products and fp32 planes
    as the graph says, so the same bounds hold."""
    sizes, x, s, want = _unpack(case, grad=True)
    out = _run(graphs.build("mha", **sizes), s, "unfused")
    _check(out, want, sizes["dtype"], ("L",))
    _, s["O"] = ref.rounded(out["O"], sizes["dtype"])
    s["L"] = out["L"].astype(np.float32)
    _check(_run(graphs.build("mha_grad", **sizes), s, "unfused"), want, sizes["dtype"])


PRIMITIVES = [
    ("lt", [(5, 1, 7), (6, 1)], {}), ("le", [(40, 3), (3,)], {}), ("gt", [(33,), (33,)], {}), ("ge", [(4, 9), (4, 1)], {}),
    ("eq", [(5, 8), (5, 8)], {}), ("lt", [(9, 5)], dict(scalar=1.0)), ("select", [(4, 1, 6), (5, 6), (1, 1, 6)], {}),
    ("select", [(3, 8), (3, 8)], dict(scalar=-2.5)), ("iota", [], dict(shape=(5, 7), axis=0)), ("iota", [], dict(shape=(3, 2, 9), axis=-1)),
    ("gather", [(4, 1, 1, 6), (5, 7)], {}), ("gather", [(9,), (2, 3, 8)], {}), ("gather", [(2, 3, 1, 5), (2, 1, 4)], {}),
    ("bin_sum", [(3, 4, 5, 7), (5, 7)], dict(shape=(4, 1, 1, 6))), ("bin_sum", [(6, 50), (6, 50)], dict(shape=(9,))),
    ("bin_sum", [(2, 300, 40), (300, 1)], dict(shape=(2, 1, 1, 33))),
]


@pytest.mark.parametrize("op,shapes,attrs", PRIMITIVES, ids=str)
def test_primitive_kernels(op, shapes, attrs):
    """Every new primitive's own kernel against the oracle (NaN and values outside
    a table among the indices)."""
    from oracle import primitives as prim
    rng = np.random.default_rng(5)
    x = [rng.integers(-2, 8, s).astype(np.float64) for s in shapes]
    for i in ([1] if op in ("gather", "bin_sum") else []):
        x[i].reshape(-1)[0], x[i].reshape(-1)[-1] = np.nan, 1e30
    if op in ("gather", "bin_sum"):
        x[0] = ref.rounded(rng.normal(size=shapes[0]), "f32")[0]
    w = graphs.layout_probe(op, "f32", shapes, **attrs)
    got = _run(w, {f"in{i}": v.astype(np.float32) for i, v in enumerate(x)}, "unfused")["out"]
    if op in ("lt", "le", "gt", "ge", "eq"):
        want = prim.elementwise(op, x, attrs.get("scalar"))
    elif op == "select":
        want = prim.select(*x, *([attrs["scalar"]] if "scalar" in attrs else []))
    elif op == "iota":
        want = prim.iota(**attrs)
    elif op == "gather":
        want = prim.gather(*x)
    else:
        want = prim.bin_sum(*x, attrs["shape"])
        # fp32 sums of at most x.size terms
        assert np.max(np.abs(got - want)) <= x[0].size * 2.0 ** -24 * np.abs(x[0]).sum()
        return
    assert np.array_equal(got, want)


def test_rows_that_the_mask_leaves_empty():
    """Lengths of 0 and of fewer positions than queries: rows without a key are
    zeros with zero gradients, the others are what they are alone."""
    case = dict(dtype="f16", n=40, m=64, d=64, heads=4, kv_heads=2, lengths=(0, 7, 64), batch=3, causal=True)
    sizes, x, s, want = _unpack(case, grad=True)
    out = _run(graphs.build("mha", **sizes), s)
    _check(out, want, "f16", ("L",))
    assert np.all(out["O"][0] == 0) and np.all(out["L"][0] == 0) and np.all(out["O"][1, :, :33] == 0)
    _, s["O"] = ref.rounded(out["O"], "f16")
    s["L"] = out["L"].astype(np.float32)
    out = _run(graphs.build("mha_grad", **sizes), s)
    _check(out, want, "f16")
    assert np.all(out["dQ"][0] == 0) and np.all(out["dK"][0] == 0) and np.all(out["dV"][1, :, 7:] == 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 5, 70])
def test_whatever_lies_behind_a_sequence(dtype, n):
    """K and V past a sequence's length hold NaN, infinities and the type's lowest
    values: the results are those of zeros there, and their gradients are zero."""
    case = dict(dtype=dtype, n=n, m=150, d=64, heads=4, kv_heads=2, lengths=(70, 133), batch=2, causal=True, cap=8.0)
    sizes, x, s, want = _unpack(case, grad=True)
    bad = {"f32": np.array([np.nan, np.inf, -np.inf, np.finfo(np.float32).min], np.float32),
           "bf16": np.array([0x7FC0, 0x7F80, 0xFF80, 0xFF7F], np.uint16)}[dtype]
    for k in ("K", "V"):
        for b, size in enumerate((70, 133)):
            rows = s[k][b, :, size:]
            rows[...] = np.resize(bad, rows.shape)
    out = _run(graphs.build("mha", **sizes), s)
    _check(out, want, dtype, ("L",))
    _, s["O"] = ref.rounded(out["O"], dtype)
    s["L"] = out["L"].astype(np.float32)
    out = _run(graphs.build("mha_grad", **sizes), s)
    _check(out, want, dtype)
    assert np.all(out["dK"][0, :, 70:] == 0) and np.all(out["dV"][1, :, 133:] == 0)


def test_large_scores():
    """Scores in the hundreds, either sign, growing along the keys: the running
    maximum moves in every tile."""
    for dtype in ("f32", "f16"):
        case = dict(dtype=dtype, n=64, m=400, d=64, heads=2)
        sizes, x, s, _ = _unpack(case)
        x["K"], s["K"] = ref.rounded(x["K"] * np.linspace(0.1, 40, 400)[None, None, :, None], dtype)
        want = ref.attention(x, dtype, 2, 2)
        _check(_run(graphs.build("mha", **sizes), s), want, dtype, ("L",))


def _bits(t):
    import torch
    return t.view(torch.int32 if t.element_size() == 4 else torch.int16).cpu().numpy().copy()


REPEAT = [
    ("layernorm_grad", dict(m=700, d=768, dtype="f16")),
    ("mha", dict(batch=2, heads=8, kv_heads=2, n=1, m=3000, d=64, dtype="bf16", lengths=True)),
    ("mha", dict(heads=2, n=300, m=1500, d=128, dtype="f16", causal=True)),
    ("mha_grad", dict(batch=2, heads=4, kv_heads=4, n=200, d=64, dtype="f16", radius=30, buckets=16)),
]


def _random_runner(name, sizes, seed=0, plan="fused"):
    import torch
    from paper_2406_09465_amd.runner import TORCH_DTYPE, PlanRunner
    w = graphs.build(name, **sizes)
    r = PlanRunner(w, plan)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    for k, i in zip(w.input_names, w.graph.inputs()):
        _, dt, shape = w.graph.node_info(i)
        if k == "lengths":
            t = torch.linspace(1, sizes["m"], sizes["batch"], device="cuda").round()
        elif k == "bucket":
            t = torch.from_numpy(ref.bucket_map(sizes["radius"], sizes["buckets"])).float().cuda()
        else:
            t = torch.randn(shape, generator=gen, device="cuda")
        r.ins.append(t.to(TORCH_DTYPE[dt]).contiguous())
    return r.bind()


@pytest.mark.parametrize("name,sizes", REPEAT, ids=str)
def test_same_bits_again_on_another_stream_and_replayed(name, sizes):
    """Hand-overs between workgroups are in a fixed order: every execution gives
    the same bits, on a stream of its own, allocation-free and as a replayed graph
    with eager work between the replays."""
    import torch
    from paper_2406_09465_amd._abi import pointer_array
    r = _random_runner(name, sizes)
    r.launch_bound()
    torch.cuda.synchronize()
    first = [_bits(t) for t in r.outs]

    def same(outs=None):
        torch.cuda.synchronize()
        for a, b in zip(first, outs or r.outs):
            assert np.array_equal(a, _bits(b))
        for t in outs or r.outs:
            t.fill_(7)

    same()
    for _ in range(3):
        r.launch_bound()
        same()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    r.launch(s)
    same()
    other = [torch.empty_like(t) for t in r.outs]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        r.launch(torch.cuda.current_stream())
    for _ in range(3):
        g.replay()
        same()
        r.bind().launch_bound()
        same()
    if r.plan.workspace_bytes() < 30e6:
        unsplit = r.plan
        unsplit.execute_noalloc(pointer_array([t.data_ptr() for t in r.ins]), pointer_array([t.data_ptr() for t in other]),
                                torch.cuda.current_stream().cuda_stream)
        same(other)


def test_a_cache_past_32_bits():
    """Keys and values of 5.4 GB each: the last sequence lies behind 2^32 bytes."""
    import torch
    from paper_2406_09465_amd.runner import PlanRunner
    batch, m, d = 5, 4194304 // 2, 256
    w = graphs.build("mha", batch=batch, heads=2, kv_heads=1, n=1, m=m, d=d, dtype="f16", lengths=True)
    r = PlanRunner(w, "fused")
    gen = torch.Generator(device="cuda").manual_seed(1)
    kv = [torch.zeros(batch, 1, m, d, dtype=torch.float16, device="cuda") for _ in range(2)]
    q = torch.randn(batch, 2, 1, d, generator=gen, device="cuda").half()
    size = 900
    for t in kv:
        t[-1, 0, :size] = torch.randn(size, d, generator=gen, device="cuda").half()
        t[-1, 0, size:] = float("nan")
    lengths = torch.tensor([1.0, 1.0, 1.0, 1.0, float(size)], device="cuda")
    r.ins = [q, kv[0], kv[1], lengths]
    r.launch()
    torch.cuda.synchronize()
    x = dict(Q=q[-1:].double().cpu().numpy(), K=kv[0][-1:, :, :size].double().cpu().numpy(), V=kv[1][-1:, :, :size].double().cpu().numpy())
    want = ref.attention(x, "f16", 2, 1)
    for out, k in zip(r.outs, ("O", "L")):
        assert ref.outside(out[-1:].double().cpu().numpy(), *want[k], "f32" if k == "L" else "f16") <= 1.0


def test_a_layer_in_training():
    """LayerNorm, attention over its result and both gradients, chained as a
    training step runs them, in fp32 against float64 (the plans' fp32 tolerance)."""
    from .helpers import TOL, close
    rng = np.random.default_rng(9)
    b, h, n, d = 2, 3, 90, 32
    rows, width = b * n, h * d
    X, sX = ref.rounded(rng.normal(0.2, 1.3, (rows, width)), "f32")
    gamma, sg = ref.rounded(rng.normal(1, 0.1, width), "f32")
    beta, sb = ref.rounded(rng.normal(0, 0.1, width), "f32")
    dO, sdO = ref.rounded(rng.normal(0, 1, (b, h, n, d)), "f32")
    heads = lambda y: np.ascontiguousarray(y.reshape(b, n, h, d).transpose(0, 2, 1, 3))  # noqa: E731
    flat = lambda y: np.ascontiguousarray(y.transpose(0, 2, 1, 3)).reshape(rows, width)  # noqa: E731
    f32 = lambda y: np.asarray(y, dtype=np.float32)  # noqa: E731
    ln = _run(graphs.build("layernorm", m=rows, d=width, dtype="f32"), dict(X=sX, gamma=sg, beta=sb))
    y = heads(f32(ln["Y"]))
    sizes = dict(batch=b, heads=h, n=n, d=d, dtype="f32", causal=True)
    at = _run(graphs.build("mha", **sizes), dict(Q=y, K=y, V=y))
    gr = _run(graphs.build("mha_grad", **sizes), dict(Q=y, K=y, V=y, dO=sdO, O=f32(at["O"]), L=f32(at["L"])))
    dY = f32(flat(gr["dQ"] + gr["dK"] + gr["dV"]))
    back = _run(graphs.build("layernorm_grad", m=rows, d=width, dtype="f32"),
                dict(X=sX, gamma=sg, mu=f32(ln["mu"]), r=f32(ln["r"]), dY=dY))
    w = ref.layernorm(X, gamma, beta, np.zeros_like(X), 1e-5, "f32")
    yw = heads(w["Y"][0])
    a = ref.attention(dict(Q=yw, K=yw, V=yw, dO=dO), "f32", h, h, causal=True, grad=True)
    w = ref.layernorm(X, gamma, beta, flat(a["dQ"][0] + a["dK"][0] + a["dV"][0]), 1e-5, "f32")
    for k in ("dX", "dgamma", "dbeta"):
        ok, mx, rel = close(back[k], w[k][0], TOL["f32"])
        assert ok, (k, mx, rel)


@pytest.mark.parametrize("workload,sizes", [
    ("attention", dict(n=1024, d=64, dtype="f16")), ("attention", dict(n=300, d=40, nk=700, dtype="bf16")),
    ("attention", dict(n=70, d=128, nk=256, dtype="f32")), ("attention", dict(n=1, d=64, nk=1000, dtype="f16")),
    ("sra", dict(hh=136, ww=136, c=64, r=8, dtype="f16")), ("sra", dict(hh=160, ww=128, c=32, r=4, dtype="bf16")),
], ids=str)
def test_workloads_past_the_keys_that_fit_lds(workload, sizes):
    """The workloads' fused plans with more keys than one workgroup's LDS holds."""
    from oracle import configs as OC
    from oracle.graph import run_unfused
    from synthetic import storage_to_f64
    from synthetic import workloads as W

    from .helpers import TOL, close
    w = graphs.build(workload, **sizes)
    assert w.graph.family(*w.kernels("fused")[-1]) == "plane"
    raw = W.inputs(workload, **sizes)
    want = run_unfused(OC.build(workload, **{k: v for k, v in sizes.items()}), {k: storage_to_f64(v, sizes["dtype"]) for k, v in raw.items()})
    got = _run(w, raw)
    ok, mx, rel = close(got["O"], want["O"], TOL[sizes["dtype"]])
    assert ok, (mx, rel)


WIDE = [
    dict(dtype="f32", n=50, m=70, d=256, heads=2, kv_heads=1, causal=True),
    dict(dtype="f32", n=40, d=192, heads=2, cap=4.0),
    dict(dtype="f16", n=60, d=64, radius=3000, buckets=9, heads=3, batch=2),
    dict(dtype="bf16", n=45, d=32, radius=30, buckets=300, heads=2, causal=True),
]


@pytest.mark.parametrize("case", WIDE, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()))
def test_gradient_at_the_ends_of_what_a_kernel_holds(case):
    """The widest heads in fp32, a bucket map too long for LDS, many buckets."""
    test_attention_gradient(case)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_a_cap_far_above_the_scores(dtype):
    """cap tanh(s / cap) is s to 1e-9 then.  The tanh (two steps of fp32) and the two
    products by constants add 6 half steps of |s| to the bound's 8, so its double holds."""
    case = dict(dtype=dtype, n=70, m=130, d=64, heads=2)
    sizes, x, s, want = _unpack(case, grad=True)
    sizes["cap"] = 1e5
    out = _run(graphs.build("mha", **sizes), s)
    _check(out, {k: (v, 2 * b) for k, (v, b) in want.items()}, dtype, ("L",))
    _, s["O"] = ref.rounded(out["O"], dtype)
    s["L"] = out["L"].astype(np.float32)
    _check(_run(graphs.build("mha_grad", **sizes), s), {k: (v, 2 * b) for k, (v, b) in want.items()}, dtype)


def _masked_rows(mask, n, m, vectors, low, scale=0.1):
    """Softmax attention with a mask made from two vectors u [n, 1] and v [1, m]: the
    product, the row maxima and the sums as results."""
    b = graphs._B("f32")
    for k, sh in (("Q", (n, 16)), ("K", (m, 16)), ("V", (m, 16)), ("u", (n, 1)), ("v", (1, m))):
        b.inp(k, sh)
    b.op("KT", "transpose", ["K"], perm=(1, 0))
    b.op("S0", "matmul", ["Q", "KT"])
    b.op("S", "mul", ["S0"], scalar=scale)
    prims = ["KT", "S0", "S"]
    for name, op, ins, attrs in mask:
        b.op(name, op, ins, **attrs)
        prims.append(name)
    c = mask[-1][0]
    b.op("Sm", "select", [c, "S"], scalar=low)
    b.op("m", "reduce_max", ["Sm"], axis=-1, keepdim=True)
    b.op("Z", "sub", ["S", "m"])
    b.op("Ex", "exp", ["Z"])
    b.op("E", "select", [c, "Ex"], scalar=0.0)
    b.op("l", "reduce_sum", ["E"], axis=-1, keepdim=True)
    b.op("O", "matmul", ["E", "V"])
    w = graphs._finish(b, "masked", ["O", "m", "l"], {})
    w.plans["fused"] = [(prims + ["Sm", "m", "Z", "Ex", "E", "l", "O"], ["O", "m", "l"])]
    return w


MASKS = {
    "abs": ([("a", "abs", ["v"], {}), ("c", "ge", ["a"], dict(scalar=0.0))], lambda u, v: np.broadcast_to(np.abs(v) >= 0, (u.size, v.size))),
    "difference": ([("d", "sub", ["u", "v"], {}), ("c", "le", ["d"], dict(scalar=1e30))], lambda u, v: u - v <= 1e30),
    "sum": ([("d", "add", ["v", "u"], {}), ("a", "abs", ["d"], {}), ("c", "ge", ["a"], dict(scalar=0.5))], lambda u, v: np.abs(u + v) >= 0.5),
    "product": ([("d", "mul", ["v", "u"], {}), ("c", "lt", ["d"], dict(scalar=1e30))], lambda u, v: u * v < 1e30),
    "equal": ([("c", "eq", ["u", "v"], {})], lambda u, v: u == v),
    "either": ([("g", "gt", ["v", "u"], {}), ("h", "lt", ["v"], dict(scalar=-3.0)), ("c", "max", ["g", "h"], {})], lambda u, v: (v > u) | (v < -3)),
}


@pytest.mark.parametrize("name", MASKS)
@pytest.mark.parametrize("low", [-1e30, -3.4e38, -np.inf])
def test_masks_from_vectors_that_hold_anything(name, low):
    """NaN and infinities among the values that a mask compares (a comparison with
    NaN is false), tiles that are clean, mixed and all of a kind; the maximum of a
    row that is left empty is the masked score itself."""
    n, m = 150, 420
    ops, truth = MASKS[name]
    rng = np.random.default_rng(11)
    x, s = {}, {}
    for k, sh in (("Q", (n, 16)), ("K", (m, 16)), ("V", (m, 16))):
        x[k], s[k] = ref.rounded(rng.normal(0, 1.5, sh), "f32")
    u, v = rng.integers(-2, 3, (n, 1)).astype(np.float32), rng.integers(-2, 3, (1, m)).astype(np.float32)
    v[0, 3], v[0, 40], v[0, 70] = np.nan, np.inf, -np.inf
    v[0, 128:192], v[0, 192:256], v[0, 256:320] = np.nan, np.inf, -np.inf
    u[5], u[40], u[77] = np.nan, np.inf, -np.inf
    s["u"], s["v"] = u, v
    with np.errstate(invalid="ignore"):
        mask = truth(u.astype(np.float64), v.astype(np.float64))
    sc = x["Q"] @ x["K"].T * 0.1
    some = mask.any(1, keepdims=True)
    mx = np.max(np.where(mask, sc, -np.inf), 1, keepdims=True)
    e = np.where(mask, np.exp(sc - np.where(some, mx, 0)), 0)
    w = _masked_rows(ops, n, m, (u, v), low)
    assert w.graph.family(*w.kernels("fused")[0]) == "plane"
    got = _run(w, s)
    # 18 roundings of the product and the scale; an exponential's error is its argument's
    e_s = 18 * ref.E * np.abs(x["Q"]) @ np.abs(x["K"]).T * 0.1
    assert np.array_equal(got["m"][~some[:, 0]], np.full((int((~some).sum()), 1), low, np.float32).astype(np.float64))
    assert np.all(np.abs(got["m"] - np.where(some, mx, 0))[some] <= e_s.max(1, keepdims=True)[some])
    rel = 2 * e_s.max(1, keepdims=True) + ref.F + 4 * ref.E * np.abs(sc).max() * 2
    assert np.all(np.abs(got["l"] - e.sum(1, keepdims=True)) <= (rel + m * ref.E) * e.sum(1, keepdims=True))
    assert np.all(np.abs(got["O"] - e @ x["V"]) <= (rel + m * ref.E) * (e @ np.abs(x["V"])))


def test_allocation_free_sums_of_long_rows():
    """The column sums' hand-over of rows of 16384 exceeds the library's static
    memory: without an allocation fewer workgroups hand over."""
    import torch
    from paper_2406_09465_amd._abi import pointer_array
    m, d = 600, 16384
    rng = np.random.default_rng(4)
    x, s = {}, {}
    for k, sh in (("X", (m, d)), ("gamma", (d,)), ("beta", (d,)), ("dY", (m, d))):
        x[k], s[k] = ref.rounded(rng.normal(0.1, 1, sh), "f16")
    want = ref.layernorm(x["X"], x["gamma"], x["beta"], x["dY"], 1e-5, "f16")
    s["mu"], s["r"] = want["mu"][0].astype(np.float32), want["r"][0].astype(np.float32)
    from paper_2406_09465_amd.runner import PlanRunner
    r = PlanRunner(graphs.build("layernorm_grad", m=m, d=d, dtype="f16"), "fused")
    r.set_inputs(s)
    r.plan.execute_noalloc(pointer_array([t.data_ptr() for t in r.ins]), pointer_array([t.data_ptr() for t in r.outs]),
                           torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    for k, t in zip(r.w.output_names, r.outs):
        assert ref.outside(t.double().cpu().numpy(), *want[k], "f16") <= 1.0, k


BLOCKS = [
    dict(dtype="f16", n=150, d=64, heads=6, kv_heads=2, docs=3, causal=True, batch=2),
    dict(dtype="f32", n=61, m=90, d=32, heads=4, kv_heads=1, causal=True, cap=4.0, slopes=True),
    dict(dtype="bf16", n=250, m=260, d=128, heads=8, kv_heads=2, lengths=(251, 260), batch=2, causal=True),
    dict(dtype="f16", n=120, d=64, heads=96, kv_heads=48, docs=2, batch=8),
]


@pytest.mark.parametrize("case", BLOCKS, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items() if k != "lengths"))
def test_heads_of_a_group_that_end_inside_a_tile(case):
    """Query heads that share a key head are rows of one axis: each starts a tile."""
    test_attention_gradient(case)


PAIRS = [
    dict(dtype="f16", n=120, d=64, heads=32, docs=3, batch=8, causal=True),
    dict(dtype="bf16", n=70, m=200, d=40, heads=64, kv_heads=32, docs=5, batch=6, causal=True, cap=6.0),
]


@pytest.mark.parametrize("case", PAIRS, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()))
def test_gradients_of_many_packed_heads(case):
    """So many tiles of 32 that two waves, not four, share one."""
    test_attention_gradient(case)


@pytest.mark.parametrize("kind", ["runs", "apart", "past the last bucket", "one"])
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_bucket_maps(kind, dtype):
    """Equal buckets that are neighbours, or apart by one or two distances, or equal
    only once they are clamped to the table."""
    case = dict(dtype=dtype, n=150, d=32, radius=40, buckets=6, heads=3, batch=2)
    sizes, x, s, _ = _unpack(case)
    t = np.arange(-40, 41)
    maps = {"runs": np.minimum(np.abs(t) // 3, 5), "apart": (t * t) % 6, "past the last bucket": 4 + np.abs(t) % 3 * 2, "one": 0 * t + 3}
    x["bucket"], s["bucket"] = ref.rounded(maps[kind], "f32")
    x["bucket"] = np.clip(x["bucket"], 0, 5)
    want = ref.attention(x, dtype, 3, 3, radius=40, grad=True)
    out = _run(graphs.build("mha", **sizes), s)
    _check(out, want, dtype, ("L",))
    _, s["O"] = ref.rounded(out["O"], dtype)
    s["L"] = out["L"].astype(np.float32)
    _check(_run(graphs.build("mha_grad", **sizes), s), want, dtype)
