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
