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
