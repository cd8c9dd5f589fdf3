"""Group norm, rotary positions and gradient clipping without a GPU: definitions,
gradients by differences, refusals, kernel families and compiled code."""

import math

import numpy as np
import pytest

from oracle import primitives as prim
from oracle.graph import run_unfused
from paper_2406_09465_amd import codeobj, graphs
from paper_2406_09465_amd._abi import Graph, KorchError
from tests import test_gpu_vision_ops as cases
from tests import vision_ref as ref
from tests.helpers import disassemble
from tests.test_layer_ops import _differences, _oracle_copy


def _oracle(name, x, **sizes):
    w = graphs.build(name, **sizes)
    return run_unfused(_oracle_copy(w), {k: x[k] for k in w.input_names})


# ---- the graphs compute the plain forms ------------------------------------------


def test_angle_primitives_by_definition():
    x, y = np.array([[0.5], [-3.0]]), np.array([2.0, 0.0, 7.0])
    assert np.array_equal(prim.elementwise("cos_mul", [x, y]), np.cos(x * y)) and np.array_equal(prim.elementwise("sin_mul", [x, y]), np.sin(x * y))
    g = Graph()
    a, b = g.input("f32", (3, 1)), g.input("f32", (4,))
    o = g.op("cos_mul", [a, b], "f32")
    assert g.node_info(o)[2] == (3, 4)
    with pytest.raises(KorchError, match="two tensors"):
        g.op("sin_mul", [a], "f32", scalar=2.0)
    with pytest.raises(KorchError, match="broadcast"):
        g.op("sin_mul", [a, g.input("f32", (2, 4))], "f32")


@pytest.mark.parametrize("case", [c for c in cases.GN if math.prod(c[1:5]) < 2e5], ids=str)
def test_groupnorm_graphs_compute_the_plain_form(case):
    z = cases._gn_sizes(case)
    x, _ = cases._gn_inputs(*case[:5])
    want = ref.groupnorm(x["X"], x["gamma"], x["beta"], z["groups"], 1e-5, z["act"], z["dtype"], x["dY"])
    x.update(_oracle("groupnorm", x, **z))
    x.update(_oracle("groupnorm_grad", x, **z))
    for k, (v, _) in want.items():
        assert np.allclose(x[k], v, rtol=1e-9, atol=1e-10), k


@pytest.mark.parametrize("case", [c for c in cases.ROT if c["n"] < 200], ids=str)
def test_rotary_graphs_compute_the_plain_form(case):
    c, x, _ = cases._rot_case(case)
    for name, want in zip(("rotary", "rotary_grad"), cases._rot_want(c, x)):
        out = _oracle(name, x, **c)
        assert set(out) == set(want)
        for k, (v, _) in want.items():
            assert np.allclose(out[k], v, rtol=1e-12, atol=1e-12), k


@pytest.mark.parametrize("max_norm", [0.5, 1e6])
@pytest.mark.parametrize("case", cases.CLIP, ids=lambda c: f"{len(c['shapes'])}x{c['shapes'][0]}")
def test_clip_graphs_compute_the_plain_form(case, max_norm):
    dt, x, _ = cases._clip_case(case)
    out = _oracle("grad_clip", x, **case, max_norm=max_norm)
    for k, (v, _) in ref.clipped(list(x.values()), dt, max_norm, 1e-6).items():
        assert np.allclose(out[k], v, rtol=1e-10), k


@pytest.mark.parametrize("act", graphs.ACTIVATIONS)
def test_groupnorm_gradient_by_differences(act):
    x, _ = cases._gn_inputs("f32", 2, 3, 3, 8)
    f = lambda y: ref.groupnorm(y["X"], y["gamma"], y["beta"], 2, 1e-5, act, "f32")["Y"][0]  # noqa: E731
    want = ref.groupnorm(x["X"], x["gamma"], x["beta"], 2, 1e-5, act, "f32", x["dY"])
    rng = np.random.default_rng(1)
    for name in ("X", "gamma", "beta"):
        for at, d in _differences(f, x, name, x["dY"], rng):
            # central differences of step 1e-5: off by about step^2 and 1e-16 / step (no Z of these inputs is within a step of 0)
            assert abs(d - want["d" + name][0][at]) < 1e-8 + 1e-7 * abs(d), (name, at)


def test_rotary_gradient_by_differences():
    c, x, _ = cases._rot_case(dict(dtype="f32", batch=1, heads=2, kv_heads=1, n=3, d=8, rot=6, axes=2, packed=True))
    grad = _oracle("rotary_grad", x, **c)["dQKV"]
    rng = np.random.default_rng(2)

    def f(y):
        out = _oracle("rotary", y, **c)
        return np.concatenate([out["Qr"], out["Kr"], out["V"]], 1)

    weight = np.concatenate([x["dQr"], x["dKr"], x["dV"]], 1)
    for at, d in _differences(f, x, "QKV", weight, rng, 10):
        assert abs(d - grad[at]) < 1e-8 + 1e-7 * abs(d), at


# ---- refusals -----------------------------------------------------------------------


@pytest.mark.parametrize("name,sizes,what", [
    ("groupnorm", dict(c=30, groups=4), "multiple of groups"),
    ("groupnorm", dict(c=0, groups=4), "positive"),
    ("groupnorm", dict(batch=0), "positive"),
    ("groupnorm", dict(hh=1, ww=1, c=8, groups=8), "two elements"),
    ("groupnorm", dict(eps=float("nan")), "eps"),
    ("groupnorm", dict(eps=-1e-5), "eps"),
    ("groupnorm_grad", dict(act="gelu"), "act"),
    ("groupnorm_grad", dict(c=30, groups=4), "multiple of groups"),
    ("rotary", dict(rot=7), "rot"),
    ("rotary", dict(rot=0), "rot"),
    ("rotary", dict(d=32, rot=64), "rot"),
    ("rotary", dict(d=33), "rot"),
    ("rotary", dict(heads=6, kv_heads=4), "multiple of kv_heads"),
    ("rotary_grad", dict(axes=0), "positive"),
    ("rotary_grad", dict(n=0), "positive"),
    ("grad_clip", dict(shapes=[]), "one shape"),
    ("grad_clip", dict(shapes=[(3,), (4,)], dtypes=["f32"]), "a type for each"),
    ("grad_clip", dict(shapes=[(3, 0)]), "positive sizes"),
    ("grad_clip", dict(shapes=[()]), "positive sizes"),
    ("grad_clip", dict(max_norm=0.0), "max_norm"),
    ("grad_clip", dict(max_norm=float("inf")), "max_norm"),
    ("grad_clip", dict(eps=-1.0), "eps"),
], ids=str)
def test_arguments_refused(name, sizes, what):
    with pytest.raises(ValueError, match=what):
        graphs.build(name, **sizes)


@pytest.mark.parametrize("name,sizes,what", [
    ("groupnorm", dict(eps=1e39), "eps"),
    ("groupnorm_grad", dict(eps=float("inf")), "eps"),
    ("grad_clip", dict(max_norm=1e39), "max_norm"),
    ("grad_clip", dict(max_norm=1e-50), "max_norm"),
    ("grad_clip", dict(max_norm=float("nan")), "max_norm"),
    ("grad_clip", dict(eps=1e39), "eps"),
], ids=str)
def test_numbers_that_fp32_does_not_hold_refused(name, sizes, what):
    with pytest.raises(ValueError, match=what):
        graphs.build(name, **sizes)


def test_inputs_refused():
    import torch

    from paper_2406_09465_amd.runner import check_inputs
    w = graphs.build("rotary", batch=2, heads=2, n=3, d=8, axes=2, dtype="f16")
    ok = [torch.zeros(2, 2, 3, 8).half(), torch.zeros(2, 2, 3, 8).half(), torch.zeros(2, 3, 2), torch.zeros(4), torch.zeros(4)]
    check_inputs(w.graph, w.input_names, ok, "cpu")
    for i, bad in ((0, ok[0].float()), (2, torch.zeros(3, 2)), (2, torch.zeros(2, 3, 2).double()), (4, torch.zeros(8)[::2]), (1, torch.zeros(2, 3, 2, 8).half().transpose(1, 2))):
        with pytest.raises(ValueError, match="input"):
            check_inputs(w.graph, w.input_names, ok[:i] + [bad] + ok[i + 1:], "cpu")


def test_more_than_the_fused_kernels_take():
    """Past the limits a kernel has no family, and the plan of one kernel per primitive remains."""
    w = graphs.build("groupnorm", hh=4, ww=4, c=8194, groups=2)
    assert w.graph.family(*w.kernels("layered")[0]) == "group" or w.plan("unfused").num_kernels() > 5
    w = graphs.build("groupnorm", hh=200, ww=200, c=8194, groups=2)
    assert "none" in [w.graph.family(*k) for k in w.kernels("fused")]
    with pytest.raises(KorchError) as e:
        w.plan("fused").compile()
    assert e.value.code == -20
    w = graphs.build("rotary", batch=1 << 16, heads=1, n=1 << 15, d=2)  # 2^31 tokens
    assert w.graph.family(*w.kernels("fused")[0]) != "rotary"


def test_look_alikes_are_not_taken():
    """Graphs that differ from a turn of pairs in one place are no rotary kernel's."""
    def build(change):
        b = graphs._B("f32")
        a = graphs._Rotary(b, 1, 2, 2, 3, 8, 8, 1, False, False)
        b.inp("Q", (1, 2, 3, 8))
        a.angles()
        if change == "a factor per head":
            b.inp("co2", (1, 2, 3, 4))
            b.ids["co"] = b.ids["co2"]
            b.inputs.remove("co2"), b.inputs.append("co")
            a.prims.remove("co")
        a.turn("Qr", "Q", 2, False)
        out = "Qr"
        if change == "halves swapped":
            b.op("sw", "concat", ["Qr_b", "Qr_a"], axis=-1)
            a.prims[-1] = out = "sw"
        w = graphs._finish(b, "r", [out], {})
        return w.graph.family([w.ids[p] for p in a.prims], [w.ids[out]])

    assert build(None) == "rotary" and build("halves swapped") != "rotary" and build("a factor per head") != "rotary"
    # a scaled sum of squares is no norm's
    w = graphs.build("grad_clip", shapes=[(5,), (6,)], dtype="f32")
    prims, outs = w.kernels("fused")[0]
    assert w.graph.family(prims, outs) == "multi"
    first = w.ids["G0_s"]
    assert w.graph.family([w.ids["G0_q"], first], [first]) in ("colreduce", "row", "rowcol")


@pytest.mark.parametrize("name,sizes", [
    ("groupnorm", dict(batch=2, hh=3, ww=5, c=12, groups=4, act="silu")),
    ("groupnorm", dict(batch=2, hh=1, ww=1, c=12, groups=4, act="none")),
    ("groupnorm", dict(batch=2, hh=300, ww=5, c=6, groups=6, act="relu")),
    ("groupnorm_grad", dict(batch=3, hh=3, ww=5, c=12, groups=4, act="none")),
    ("groupnorm_grad", dict(batch=3, hh=700, ww=9, c=12, groups=4, act="none")),
    ("grad_clip", dict(shapes=[(5,), (3, 4)])),
], ids=str)
def test_every_kernel_that_a_family_takes_is_generated(name, sizes):
    """What the matchers accept, the generators write, for all convex parts of the graphs."""
    w = graphs.build(name, dtype="f32", **sizes)
    taken = 0
    for prims, outs in w.graph.candidates(max_prims=7, max_outs=2, only_supported=True):
        if w.graph.family(prims, outs) in ("group", "multi"):
            assert len(w.graph.kernel_source(prims, outs)) > 1000
            taken += 1
    assert taken > 20
    # a sum over a group's channels of stored sums belongs to no kernel of other sums
    if name == "groupnorm_grad":
        ids = [w.ids[k] for k in ("dZx", "sg", "c1_g", "c1_s", "c1")]
        assert w.graph.family(ids, [w.ids["sg"], w.ids["c1"]]) == "none"


# ---- kernels --------------------------------------------------------------------------


def _plans():
    for c in cases.GN:
        for name in ("groupnorm", "groupnorm_grad"):
            for plan in ("fused", "layered"):
                yield name, cases._gn_sizes(c), plan
    for c in cases.ROT:
        for name in ("rotary", "rotary_grad"):
            yield name, {k: v for k, v in c.items() if k not in ("first", "step")}, "fused"
    for c in cases.CLIP:
        yield "grad_clip", c, "fused"
    for name, sizes in cases.REPEAT:
        yield name, sizes, "fused"


@pytest.mark.parametrize("name,sizes,plan", list(_plans()), ids=lambda v: str(v)[:120])
def test_fused_plans_compile_without_spills(name, sizes, plan):
    p = graphs.build(name, **sizes).plan(plan)
    p.compile()
    fams = {p.kernel_info(k)[0] for k in range(p.num_kernels())}
    # neighbours in heads of odd widths, and one tensor's product, are the pointwise family's
    alone = sizes.get("d") == 9 or len(sizes.get("shapes", "..")) == 1
    assert fams - {"pointwise"} <= {"group", "rotary", "multi"} and ("pointwise" in fams) == alone
    for k in range(p.num_kernels()):
        code = p.kernel_code(k)
        for kernel, r in codeobj.kernel_resources(code).items():
            assert r["scratch"] == 0 and r["vgpr_spill"] == 0 and r["lds"] <= 160 * 1024, (kernel, r)
        assert not any(op.startswith("v_pk_") and op.endswith("_f32") for op, _ in disassemble(code))


def test_launches():
    """Small maps and their gradients are one kernel, large ones two; rotary is one; the norm and the clipping two."""
    assert graphs.build("groupnorm", hh=16, ww=16).plan("fused").num_kernels() == 1
    assert graphs.build("groupnorm_grad", hh=16, ww=16).plan("fused").num_kernels() == 1
    assert graphs.build("groupnorm", batch=4, hh=416, ww=416, c=64).plan("fused").num_kernels() == 2
    assert graphs.build("groupnorm_grad", batch=4, hh=416, ww=416, c=64).plan("fused").num_kernels() == 2
    assert graphs.build("rotary", axes=3, packed=True).plan("fused").num_kernels() == 1
    assert graphs.build("grad_clip").plan("fused").num_kernels() == 2
