"""Masks of plane kernels as `select` takes them: every value that is not 0 is
true (negative ones and NaN too), a mask that is read as a number keeps its
value, and its roundings are those of the graph."""

import numpy as np
import pytest

from paper_2406_09465_amd import graphs

from . import layer_ref as ref
from .test_gpu_layer_ops import _masked_rows, _run

pytestmark = pytest.mark.gpu

# primitives of the mask from u [n, 1] and v [1, m], and its value
VALUES = {
    "negated": ([("a", "le", ["v", "u"], {}), ("c", "neg", ["a"], {})], lambda u, v: -(v <= u).astype(float)),
    "distance back": ([("a", "sub", ["v", "u"], {}), ("c", "min", ["a"], dict(scalar=0.0))], lambda u, v: np.fmin(v - u, 0)),  # (min drops a NaN)
    "less one": ([("a", "lt", ["v", "u"], {}), ("c", "sub", ["a"], dict(scalar=1.0))], lambda u, v: (v < u) - 1.0),
    "distance": ([("c", "sub", ["u", "v"], {})], lambda u, v: u - v),
    "twice": ([("a", "le", ["v", "u"], {}), ("c", "mul", ["a"], dict(scalar=2.0))], lambda u, v: 2.0 * (v <= u)),
    "plain": ([("c", "ge", ["u", "v"], {})], lambda u, v: 1.0 * (u >= v)),
}


def _inputs(n, m, u, v, dtype="f32"):
    rng = np.random.default_rng(21)
    x, s = {}, {}
    for k, sh in (("Q", (n, 16)), ("K", (m, 16)), ("V", (m, 16))):
        x[k], s[k] = ref.rounded(rng.normal(0, 1.5, sh), dtype)
    s["u"], s["v"] = u.astype(np.float32), v.astype(np.float32)
    return x, s


def _softmax_check(got, x, mask, bias=0.0, e_bias=0.0):
    sc = x["Q"] @ x["K"].T * 0.1 + bias
    some = mask.any(1, keepdims=True)
    mx = np.max(np.where(mask, sc, -np.inf), 1, keepdims=True)
    e = np.where(mask, np.exp(sc - np.where(some, mx, 0)), 0)
    m = mask.shape[1]
    # 18 roundings of the product and the scale; an exponential's error is its argument's
    e_s = 18 * ref.E * np.abs(x["Q"]) @ np.abs(x["K"]).T * 0.1 + e_bias
    assert np.all(np.abs(got["m"] - np.where(some, mx, 0))[some] <= e_s.max(1, keepdims=True)[some])
    rel = 2 * e_s.max(1, keepdims=True) + ref.F + 8 * ref.E * np.abs(sc).max()
    assert np.all(np.abs(got["l"] - e.sum(1, keepdims=True)) <= (rel + m * ref.E) * e.sum(1, keepdims=True))
    assert np.all(np.abs(got["O"] - e @ x["V"]) <= (rel + m * ref.E) * (e @ np.abs(x["V"])))


@pytest.mark.parametrize("n,m", [(150, 420), (1, 300), (400, 150)])
@pytest.mark.parametrize("name", VALUES)
def test_masks_whose_truth_is_not_one(name, n, m):
    """Positions (queries at the end), tiles without a pair, mixed and full, and
    vectors that are NaN for some."""
    ops, value = VALUES[name]
    u, v = np.arange(n, dtype=np.float64)[:, None] + max(0, m - n), np.arange(m, dtype=np.float64)[None]
    if n > 100:
        u[70], u[3] = np.nan, np.inf
    x, s = _inputs(n, m, u, v)
    with np.errstate(invalid="ignore"):
        mask = value(u, v) != 0
    w = _masked_rows(ops, n, m, None, -1e30)
    assert w.graph.family(*w.kernels("fused")[0]) == "plane"
    _softmax_check(_run(w, s), x, mask)


@pytest.mark.parametrize("name", VALUES)
def test_a_mask_that_is_also_a_bias(name):
    """S - mask under that mask: the mask counts as the number it is."""
    ops, value = VALUES[name]
    n, m = 150, 420
    u, v = np.arange(n, dtype=np.float64)[:, None] + m - n, np.arange(m, dtype=np.float64)[None]
    x, s = _inputs(n, m, u, v)
    b = graphs._B("f32")
    for k, sh in (("Q", (n, 16)), ("K", (m, 16)), ("V", (m, 16)), ("u", (n, 1)), ("v", (1, m))):
        b.inp(k, sh)
    b.op("KT", "transpose", ["K"], perm=(1, 0))
    b.op("S0", "matmul", ["Q", "KT"])
    b.op("S1", "mul", ["S0"], scalar=0.1)
    for k, op, ins, attrs in ops:
        b.op(k, op, ins, **attrs)
    b.op("cs", "mul", ["c"], scalar=0.125)
    b.op("S", "sub", ["S1", "cs"])
    b.op("Sm", "select", ["c", "S"], scalar=-1e30)
    b.op("m", "reduce_max", ["Sm"], axis=-1, keepdim=True)
    b.op("Z", "sub", ["S", "m"])
    b.op("Ex", "exp", ["Z"])
    b.op("E", "select", ["c", "Ex"], scalar=0.0)
    b.op("l", "reduce_sum", ["E"], axis=-1, keepdim=True)
    b.op("O", "matmul", ["E", "V"])
    w = graphs._finish(b, "masked", ["O", "m", "l"], {})
    prims = ["KT", "S0", "S1"] + [o[0] for o in ops] + ["cs", "S", "Sm", "m", "Z", "Ex", "E", "l", "O"]
    w.plans["fused"] = [(prims, ["O", "m", "l"])]
    assert w.graph.family(*w.kernels("fused")[0]) == "plane"
    val = value(u, v)
    _softmax_check(_run(w, s), x, val != 0, bias=-0.125 * val, e_bias=4 * ref.E * np.abs(0.125 * val).max())


@pytest.mark.parametrize("rows", [True, False])
@pytest.mark.parametrize("name", VALUES)
def test_a_mask_that_is_also_a_factor(name, rows):
    """select(mask, S mask, 0) times a stored tensor, rows or columns owned, with its
    sums by bins where rows are."""
    ops, value = VALUES[name]
    n, m = 190, 330
    u, v = np.arange(n, dtype=np.float64)[:, None] + m - n, np.arange(m, dtype=np.float64)[None]
    x, s = _inputs(n, m, u, v)
    b = graphs._B("f32")
    for k, sh in (("Q", (n, 16)), ("K", (m, 16)), ("V", (m, 16)), ("u", (n, 1)), ("v", (1, m))):
        b.inp(k, sh)
    b.op("KT", "transpose", ["K"], perm=(1, 0))
    b.op("S", "matmul", ["Q", "KT"])
    for k, op, ins, attrs in ops:
        b.op(k, op, ins, **attrs)
    b.op("Sc", "mul", ["S", "c"])
    b.op("X", "select", ["c", "Sc"], scalar=0.0)
    prims = ["KT", "S"] + [o[0] for o in ops] + ["Sc", "X"]
    outs = ["O"]
    if rows:
        b.op("O", "matmul", ["X", "V"])
        b.op("which", "sub", ["v", "u"])
        b.op("at", "add", ["which"], scalar=8.0)
        b.op("T", "bin_sum", ["X", "at"], shape=(1, 1, 17))
        prims, outs = prims + ["O", "which", "at", "T"], ["O", "T"]
    else:
        b.op("XT", "transpose", ["X"], perm=(1, 0))
        b.op("O", "matmul", ["XT", "Q"])
        prims += ["XT", "O"]
    w = graphs._finish(b, "factor", outs, {})
    w.plans["fused"] = [(prims, outs)]
    assert w.graph.family(*w.kernels("fused")[0]) == "plane"
    got = _run(w, s)
    val = value(u, v)
    X = x["Q"] @ x["K"].T * val
    A = np.abs(x["Q"]) @ np.abs(x["K"]).T * np.abs(val)  # 17 roundings of the product, one of the factor
    W = x["V"] if rows else x["Q"]
    X, A = (X, A) if rows else (X.T, A.T)
    assert np.all(np.abs(got["O"] - X @ W) <= (20 + X.shape[1]) * ref.E * (A @ np.abs(W)) + 1e-30)
    if rows:
        k = np.clip(v - u + 8, 0, 16).astype(int) + 0 * X.astype(int)
        for i in range(17):
            assert abs(got["T"][0, 0, i] - X[k == i].sum()) <= (20 + n + m) * ref.E * A[k == i].sum() + 1e-30, i


def test_a_mask_rounds_as_its_primitives_do():
    """u v - 1 <= 0 with u v = 1 + 2^-36: the product rounds to 1, so every pair holds,
    in full tiles, whose mask is known from ranges, and in the last one alike."""
    n, m = 150, 420
    u, v = np.full((n, 1), 1 + 2.0 ** -12), np.full((1, m), 1 - 2.0 ** -12 + 2.0 ** -24)
    x, s = _inputs(n, m, u, v)
    assert s["u"][0, 0] * s["v"][0, 0] == np.float32(1) and float(s["u"][0, 0]) * float(s["v"][0, 0]) > 1
    ops = [("a", "mul", ["u", "v"], {}), ("b", "add", ["a"], dict(scalar=-1.0)), ("c", "le", ["b"], dict(scalar=0.0))]
    w = _masked_rows(ops, n, m, None, -1e30)
    assert w.graph.family(*w.kernels("fused")[0]) == "plane"
    _softmax_check(_run(w, s), x, np.ones((n, m), bool))
