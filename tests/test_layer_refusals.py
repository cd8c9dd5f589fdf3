"""Arguments of the layer operators that no kernel can take."""

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
