"""A sum by bins of a plane that no product reads (a bias table's gradient on its
own): the streamed axis is split over workgroups, whose sums are joined."""

import numpy as np
import pytest

from paper_2406_09465_amd import graphs

from . import layer_ref as ref
from .test_gpu_layer_ops import _run

SIZES = [(2048, 2048, False), (33, 1500, True), (700, 300, True), (1, 4000, False)]


def bins_only(dtype, n, m, causal, bins=8, d=64):
    """T[k] = sum of exp(scale Q K^T) over the pairs whose distance j - i + 3, clamped, is k."""
    b = graphs._B(dtype)
    b.inp("Q", (n, d))
    b.inp("K", (m, d))
    prims = ["KT", "S", "Sc", "E", "key", "pos", "rel", "at"]
    b.op("KT", "transpose", ["K"], perm=(1, 0))
    b.op("S", "matmul", ["Q", "KT"], "f32")
    b.op("Sc", "mul", ["S"], "f32", scalar=0.05)
    b.op("E", "exp", ["Sc"], "f32")
    b.op("key", "iota", [], "f32", shape=(1, m), axis=1)
    b.op("pos", "iota", [], "f32", shape=(n, 1), axis=0)
    b.op("rel", "sub", ["key", "pos"], "f32")
    b.op("at", "add", ["rel"], "f32", scalar=3.0)
    x = "E"
    if causal:
        b.op("seen", "le", ["key", "pos"], "f32")
        b.op("X", "select", ["seen", "E"], "f32", scalar=0.0)
        prims, x = prims + ["seen", "X"], "X"
    b.op("T", "bin_sum", [x, "at"], "f32", shape=(1, 1, bins))
    w = graphs._finish(b, "bins", ["T"], {})
    w.plans["fused"] = [(prims + ["T"], ["T"])]
    return w


@pytest.mark.gpu
@pytest.mark.parametrize("n,m,causal", SIZES)
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_sums_by_bins_alone(dtype, n, m, causal):
    rng = np.random.default_rng(8)
    x, s = {}, {}
    for k, r in (("Q", n), ("K", m)):
        x[k], s[k] = ref.rounded(rng.normal(0, 1, (r, 64)), dtype)
    got = _run(bins_only(dtype, n, m, causal), s)["T"].reshape(-1)
    sc = x["Q"] @ x["K"].T * 0.05
    rel = np.arange(m)[None] - np.arange(n)[:, None]
    e = np.exp(sc) * ((rel <= 0) if causal else 1.0)
    at = np.clip(rel + 3, 0, 7)
    # an exponential's error is its argument's (66 roundings of the product) and the function's; a sum's one per addend
    e_s = 66 * ref.E * (np.abs(x["Q"]) @ np.abs(x["K"]).T) * 0.05 + ref.F
    for k in range(8):
        want, bound = e[at == k].sum(), (e * e_s)[at == k].sum() + (n + m) * ref.E * e[at == k].sum()
        assert abs(got[k] - want) <= bound, (k, got[k], want, bound)
