"""Arguments of the layer operators that no kernel can take."""

import types

import pytest

from paper_2406_09465_amd import graphs


@pytest.mark.parametrize("eps", [float("nan"), float("inf"), -1e-5])
def test_eps_that_is_no_variance(eps):
    with pytest.raises(ValueError, match="eps"):
        graphs.build("layernorm", m=5, d=8, eps=eps)
    graphs.build("layernorm", m=5, d=8, eps=0.0).plan("fused").compile()


@pytest.mark.parametrize("cap", [1e-38, 1e-45, -0.5])
def test_caps_whose_reciprocal_is_no_fp32_number(cap):
    for name in ("mha", "mha_grad"):
        with pytest.raises(ValueError, match="cap"):
            graphs.build(name, n=8, heads=2, d=16, cap=cap)
        graphs.build(name, n=8, heads=2, d=16, cap=1e-30).plan("fused").compile()


def test_more_threads_than_a_launch_holds():
    """A launch takes fewer than 2^32 threads: one workgroup for each of 2^24 heads is too many."""
    for batch, family in ((1 << 17, "plane"), (1 << 18, "none")):
        w = graphs.build("mha", batch=batch, heads=64, n=1, m=1, d=8)
        assert w.graph.family(*w.kernels("fused")[0]) == family
    for rows, family in ((4095, "binsum"), (4096, "none")):
        w = graphs.layout_probe("bin_sum", "f32", [(rows, 8), (8,)], shape=(rows, 1, 4096))
        assert w.graph.family([w.ids["out"]], [w.ids["out"]]) == family


def test_inputs_that_are_not_what_the_graph_says():
    import torch

    from paper_2406_09465_amd.runner import check_inputs
    w = graphs.build("mha", batch=2, heads=4, kv_heads=2, n=3, m=8, d=16, dtype="f16")
    make = lambda *s, dtype=torch.float16: torch.zeros(s, dtype=dtype)  # noqa: E731
    q, kv = make(2, 4, 3, 16), make(2, 2, 8, 16)
    ok = lambda *t: check_inputs(w.graph, w.input_names, t, "cpu")  # noqa: E731
    ok(q, kv, kv)
    for bad, what in (((q, kv), "3 inputs"), ((q, kv, make(2, 2, 7, 16)), "input V is f16"), ((q, make(2, 4, 8, 16), kv), "input K"),
                      ((make(2, 4, 3, 16, dtype=torch.float32), kv, kv), "input Q"), ((q, make(2, 8, 2, 16).transpose(1, 2), kv), "contiguous")):
        with pytest.raises(ValueError, match=what):
            ok(*bad)
    with pytest.raises(ValueError, match="on cpu"):
        check_inputs(w.graph, w.input_names, (q, kv, kv), "cuda")
    other = types.SimpleNamespace(dtype=q.dtype, shape=q.shape, is_contiguous=lambda: True, device=torch.device("cuda", 1))
    with pytest.raises(ValueError, match="on cuda:1"):
        check_inputs(w.graph, w.input_names, (other, kv, kv), "cuda:0")
