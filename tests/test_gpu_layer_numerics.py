"""fp16 attention and its gradient where values below fp16's normal numbers meet
others: small and large gradients, long rows, a key that takes nearly all of a
row's weight.  Limits are counted from the roundings (layer_rms, layer_ref)."""

import numpy as np
import pytest

from paper_2406_09465_amd import graphs

from . import layer_ref as ref
from . import layer_rms as rms
from .test_gpu_layer_ops import _check, _run, _unpack

pytestmark = pytest.mark.gpu


def _stored(x):
    pairs = {k: ref.rounded(v, "f16") for k, v in x.items()}
    return {k: v[0] for k, v in pairs.items()}, {k: v[1] for k, v in pairs.items()}


def _train(sizes, s):
    """Forward and gradient of one case: all results by name."""
    out = _run(graphs.build("mha", **sizes), s)
    s = dict(s, O=ref.rounded(out["O"], "f16")[1], L=out["L"].astype(np.float32))
    return {**out, **_run(graphs.build("mha_grad", **sizes), s)}


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("std", [1e-4, 1e-3, 1.0, 300.0])
def test_gradients_of_every_size(std, d, causal):
    """dO from the smallest that a training step meets to loss-scaled ones."""
    n = 1500
    rng = np.random.default_rng(3)
    x, s = _stored({k: rng.normal(0, f, (1, 1, n, d)) for k, f in (("Q", 1.5), ("K", 1.0), ("V", 1.0), ("dO", std))})
    p, dx, want = rms.plane(x, causal)
    lim = rms.limits(x, p, dx, want)
    out = _train(dict(heads=1, n=n, d=d, dtype="f16", causal=causal), s)
    off = {k: rms.rms(out[k], want[k]) / lim[k] for k in lim}
    assert all(v <= 1.0 for v in off.values()), off


@pytest.mark.parametrize("n,m", [(40, 50000), (7, 100000)])
def test_gradients_of_long_rows(n, m):
    """Weights of 2e-5 and 1e-5 each: below the normal numbers of fp16, all of them."""
    d = 32
    rng = np.random.default_rng(4)
    x, s = _stored({k: rng.normal(0, f, (1, 1, r, d)) for k, f, r in (("Q", 0.5, n), ("K", 0.5, m), ("V", 1.0, m), ("dO", 100.0, n))})
    p, dx, want = rms.plane(x, False)
    lim = rms.limits(x, p, dx, want)
    out = _train(dict(heads=1, n=n, m=m, d=d, dtype="f16"), s)
    off = {k: rms.rms(out[k], want[k]) / lim[k] for k in lim}
    assert all(v <= 1.0 for v in off.values()), off


@pytest.mark.parametrize("at", [0, 1700])
@pytest.mark.parametrize("n,m", [(1, 2000), (8, 4096), (200, 2000)])
def test_a_key_that_takes_nearly_all_weight(n, m, at):
    """One key scores 14 above the others, with zeros as its value: the result is
    what the others' weights, 8e-7 each, leave, and so are their gradients."""
    d, heads = 64, 2
    rng = np.random.default_rng(5)
    x = {"Q": rng.normal(0, 0.05, (1, heads, n, d)), "K": rng.normal(0, 0.05, (1, heads, m, d)), "V": 1 + rng.normal(0, 0.2, (1, heads, m, d)),
         "dO": rng.normal(0, 100.0, (1, heads, n, d))}
    x["Q"][..., 0], x["K"][..., 0] = 8.0, 0.0
    x["K"][:, :, at, :], x["V"][:, :, at, :] = 0.0, 0.0
    x["K"][:, :, at, 0] = 14.03125
    x, s = _stored(x)
    want = ref.attention(x, "f16", heads, heads, grad=True)
    _check(_train(dict(heads=heads, n=n, m=m, d=d, dtype="f16"), s), want, "f16", ("L",))


def test_gradients_past_the_range_of_fp16():
    """P (dP - delta) up to 4e5, past what fp16 holds, where the results do not pass it."""
    n, d = 200, 64
    rng = np.random.default_rng(6)
    x, s = _stored({k: rng.normal(0, f, (1, 1, n, d)) for k, f in (("Q", 0.002), ("K", 0.002), ("V", 1500.0), ("dO", 1500.0))})
    p, dx, want = rms.plane(x, False)
    assert np.abs(dx).max() > 65504 and all(np.abs(want[k]).max() < 65504 for k in want)
    lim = rms.limits(x, p, dx, want)
    out = _train(dict(heads=1, n=n, d=d, dtype="f16"), s)
    off = {k: rms.rms(out[k], want[k]) / lim[k] for k in lim}
    assert all(v <= 1.0 for v in off.values()), off


@pytest.mark.parametrize("n", [1, 70])
def test_whatever_lies_behind_a_sequence_in_fp16(n):
    """NaN, infinities and fp16's lowest number past a sequence's length move no scale:
    results with dO of deviation 1e-3 are those of zeros there."""
    case = dict(dtype="f16", n=n, m=150, d=64, heads=4, kv_heads=2, lengths=(70, 133), batch=2, causal=True)
    sizes, x, s, _ = _unpack(case)
    x["dO"], s["dO"] = ref.rounded(x["dO"] * 1e-3, "f16")
    want = ref.attention(x, "f16", 4, 2, causal=True, grad=True)
    for k in ("K", "V"):
        for b, size in enumerate((70, 133)):
            rows = s[k][b, :, size:]
            rows[...] = np.resize(np.array([np.nan, np.inf, -np.inf, -65504], np.float16), rows.shape)
    out = _train(sizes, s)
    _check(out, want, "f16", ("L",))
    assert np.all(out["dK"][0, :, 70:] == 0) and np.all(out["dV"][1, :, 133:] == 0)
