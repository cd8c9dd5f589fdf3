"""Generated code of plane kernels past the sizes of the other tests."""

import pytest

from paper_2406_09465_amd import codeobj, graphs
from tests import test_gpu_layer_ops as cases
from tests import test_gpu_plane_joins as joins
from tests.test_gpu_plane_bins import SIZES, bins_only


@pytest.mark.parametrize("n,m,causal", SIZES)
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_sums_by_bins_alone_compile(dtype, n, m, causal):
    w = bins_only(dtype, n, m, causal)
    assert w.graph.family(*w.kernels("fused")[0]) == "plane"
    p = w.plan("fused")
    p.compile()
    for kernel, r in codeobj.kernel_resources(p.kernel_code(0)).items():
        assert r["scratch"] == 0 and r["lds"] <= 160 * 1024, (kernel, r)


@pytest.mark.parametrize("name,case", [("mha", c) for c in joins.FWD] + [("mha_grad", c) for c in joins.GRAD], ids=str)
def test_joins_of_many_splits_keep_to_their_registers(name, case):
    p = graphs.build(name, **cases._unpack(case)[0]).plan("fused")
    p.compile()
    for k in range(p.num_kernels()):
        for kernel, r in codeobj.kernel_resources(p.kernel_code(k)).items():
            assert r["scratch"] == 0 and r["vgpr_spill"] == 0 and r["lds"] <= 160 * 1024, (kernel, r)
