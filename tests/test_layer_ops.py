"""Attention of any length, LayerNorm's gradient and their primitives without a
GPU: definitions, refusals, kernel families and compiled code."""

import numpy as np
import pytest

from oracle import primitives as prim
from oracle.graph import Graph as OracleGraph
from oracle.graph import run_unfused
from paper_2406_09465_amd import codeobj, graphs
from paper_2406_09465_amd._abi import Graph, KorchError
from tests import layer_ref as ref
from tests import test_gpu_layer_ops as cases
from tests.helpers import disassemble, lds_load_faults


def _oracle_copy(w):
    """The workload's graph as the oracle's."""
    g = OracleGraph()
    names = {v: k for k, v in w.ids.items()}
    for v in range(w.graph.num_nodes()):
        op, dtype, shape = w.graph.node_info(v)
        if op == "input":
            g.input(names[v], shape, dtype)
            continue
        a = w.graph.node_attrs(v)
        attrs = dict(axis=a["axis"], keepdim=a["keepdim"], perm=a["perm"], shape=a["shape"], dtype=dtype, value=a["value"], begin=a["begin"], end=a["end"], lo=a["begin"],
                     hi=a["end"])
        if a["scalar"] is not None:
            attrs["scalar"] = a["scalar"]
        if op in ("reduce_sum", "reduce_mean", "reduce_max"):
            attrs.pop("shape")
        g.op(op, w.graph.node_inputs(v), name=names[v], **attrs)
        assert g.nodes[-1].shape == shape, (names[v], op, g.nodes[-1].shape, shape)
    for o in w.graph.outputs():
        g.output(o)
    return g


# ---- the plain forms, the primitives, the graphs -------------------------------


def test_new_primitives_by_definition():
    rng = np.random.default_rng(0)
    x, y = rng.integers(0, 4, (3, 1, 5)), rng.integers(0, 4, (2, 1))
    for op, f in (("lt", np.less), ("le", np.less_equal), ("gt", np.greater), ("ge", np.greater_equal), ("eq", np.equal)):
        assert np.array_equal(prim.elementwise(op, [x, y]), f(x, y).astype(float))
    assert np.array_equal(prim.select([1, 0, -1], [1.0, np.nan, 3.0], 7.0), [1, 7, 3])
    assert np.array_equal(prim.iota((2, 3), 1), [[0, 1, 2], [0, 1, 2]]) and np.array_equal(prim.iota((2, 3), 0), [[0, 0, 0], [1, 1, 1]])
    table = rng.normal(size=(4, 1, 1, 6))
    idx = np.array([[-3, 0, 2], [5, 9, np.nan]])
    got = prim.gather(table, idx)
    at = np.array([[0, 0, 2], [5, 5, 0]])
    assert got.shape == (4, 2, 3) and all(got[h, i, j] == table[h, 0, 0, at[i, j]] for h in range(4) for i in range(2) for j in range(3))
    # adjoint: <gather(t), y> = <t, bin_sum(y)>
    v = rng.normal(size=(3, 4, 2, 3))
    sums = prim.bin_sum(v, idx, (4, 1, 1, 6))
    assert sums.shape == table.shape
    assert np.isclose((np.broadcast_to(got, v.shape) * v).sum(), (table * sums).sum())


@pytest.mark.parametrize("case", [c for c in cases.GRAD if c["n"] * c.get("m", c["n"]) * c["d"] < 2e5], ids=str)
def test_graphs_compute_the_plain_form(case):
    """The primitives of the builders' graphs, one at a time in float64, give the plain float64 forms."""
    sizes, x, _, want = cases._unpack(case, grad=True)
    w = graphs.build("mha", **sizes)
    out = run_unfused(_oracle_copy(w), {k: x[k] for k in w.input_names})
    for k in ("O", "L"):
        assert np.allclose(out[k], want[k][0], rtol=1e-9, atol=1e-11), k
    x = {**x, "O": want["O"][0], "L": want["L"][0]}
    w = graphs.build("mha_grad", **sizes)
    out = run_unfused(_oracle_copy(w), {k: x[k] for k in w.input_names})
    for k in w.output_names:
        assert np.allclose(out[k], want[k][0], rtol=1e-8, atol=1e-10), k


def test_layernorm_graphs_compute_the_plain_form():
    rng = np.random.default_rng(1)
    x = dict(X=rng.normal(0.3, 2, (7, 12)), gamma=rng.normal(1, 0.2, 12), beta=rng.normal(0, 0.2, 12), dY=rng.normal(size=(7, 12)))
    want = ref.layernorm(x["X"], x["gamma"], x["beta"], x["dY"], 1e-5, "f32")
    for name in ("layernorm", "layernorm_grad"):
        w = graphs.build(name, m=7, d=12, dtype="f32")
        out = run_unfused(_oracle_copy(w), {k: x[k] for k in w.input_names})
        for k in w.output_names:
            assert np.allclose(out[k], want[k][0], rtol=1e-10, atol=1e-12), k
        x.update(out)


def _differences(f, x, name, weight, rng, count=6):
    """Central differences of sum(weight * f(x)) by a few elements of x[name], and their places."""
    out = []
    for _ in range(count):
        at = tuple(int(rng.integers(0, s)) for s in x[name].shape)
        d = []
        for sign in (1, -1):
            y = dict(x)
            y[name] = x[name].copy()
            y[name][at] += sign * 1e-5
            d.append(float((weight * f(y)).sum()))
        out.append((at, (d[0] - d[1]) / 2e-5))
    return out


@pytest.mark.parametrize("case", [
    dict(dtype="f32", n=5, m=9, d=8, heads=4, kv_heads=2, causal=True, cap=2.0, slopes=True),
    dict(dtype="f32", n=6, d=8, heads=2, radius=3, buckets=5, batch=2),
    dict(dtype="f32", n=8, d=8, docs=2, causal=True, heads=2),
], ids=str)
def test_attention_gradient_by_differences(case):
    sizes, x, _, want = cases._unpack(case, grad=True)
    rng = np.random.default_rng(2)
    kw = dict(heads=sizes["heads"], kv_heads=sizes["kv_heads"], cap=sizes["cap"], causal=sizes["causal"], radius=sizes["radius"])
    f = lambda y: ref.attention(y, "f32", **kw)["O"][0]  # noqa: E731
    for name, grad in (("Q", "dQ"), ("K", "dK"), ("V", "dV"), ("table", "dT")):
        if name in x:
            for at, d in _differences(f, x, name, x["dO"], rng):
                # central differences of step 1e-5: off by about step^2 and 1e-16 / step
                assert abs(d - want[grad][0][at]) < 1e-8 + 1e-7 * abs(d), (name, at)


def test_layernorm_gradient_by_differences():
    rng = np.random.default_rng(3)
    x = dict(X=rng.normal(0.3, 2, (5, 9)), gamma=rng.normal(1, 0.2, 9), beta=rng.normal(0, 0.2, 9))
    dY = rng.normal(size=(5, 9))
    f = lambda y: ref.layernorm(y["X"], y["gamma"], y["beta"], dY, 1e-5, "f32")["Y"][0]  # noqa: E731
    want = ref.layernorm(x["X"], x["gamma"], x["beta"], dY, 1e-5, "f32")
    for name, grad in (("X", "dX"), ("gamma", "dgamma"), ("beta", "dbeta")):
        for at, d in _differences(f, x, name, dY, rng):
            assert abs(d - want[grad][0][at]) < 1e-8 + 1e-7 * abs(d), (name, at)


# ---- refusals -------------------------------------------------------------------


@pytest.mark.parametrize("bad", [
    dict(heads=6, kv_heads=4), dict(n=9, m=8), dict(n=0), dict(prefix=True), dict(buckets=8), dict(radius=8), dict(cap=-1.0), dict(d=0),
], ids=str)
def test_builder_refuses(bad):
    for name in ("mha", "mha_grad"):
        with pytest.raises(ValueError):
            graphs.build(name, **{**dict(n=8, heads=2, d=16), **bad})


@pytest.mark.parametrize("dtype,d", [("f16", 20), ("bf16", 4), ("f32", 10), ("f16", 264)])
def test_head_widths_that_no_family_takes(dtype, d):
    """Rows that are not runs of 16 bytes, and heads wider than 256: infinite cost."""
    w = graphs.build("mha", n=40, heads=2, d=d, dtype=dtype)
    assert w.graph.family(*w.kernels("fused")[0]) == "none"
    with pytest.raises(KorchError, match="KORCH_E_UNSUPPORTED"):
        w.plan("fused").compile()


def test_a_mask_computed_from_scores_is_not_a_plane_kernel():
    """A tile's mask must be known before its scores."""
    b = graphs._B("f32")
    for n in "QKV":
        b.inp(n, (64, 16))
    b.op("KT", "transpose", ["K"], perm=(1, 0))
    b.op("S", "matmul", ["Q", "KT"])
    b.op("c", "gt", ["S"], scalar=0.0)
    b.op("Sm", "select", ["c", "S"], scalar=-1e30)
    b.op("m", "reduce_max", ["Sm"], axis=-1)
    b.op("Z", "sub", ["S", "m"])
    b.op("Ex", "exp", ["Z"])
    b.op("E", "select", ["c", "Ex"], scalar=0.0)
    b.op("l", "reduce_sum", ["E"], axis=-1)
    b.op("U", "matmul", ["E", "V"])
    b.op("O", "div", ["U", "l"])
    w = graphs._finish(b, "t", ["O"], {})
    assert w.graph.family([b.ids[k] for k in ("KT", "S", "c", "Sm", "m", "Z", "Ex", "E", "l", "U", "O")], [b.ids["O"]]) == "none"


@pytest.mark.parametrize("op,shapes,attrs,what", [
    ("select", [(2, 3), (4, 3)], dict(scalar=0.0), "broadcast"),
    ("select", [(2, 3)], dict(scalar=0.0), "takes 2 inputs"),
    ("lt", [(2, 3), (4,)], {}, "broadcast"),
    ("gather", [(3, 5)], {}, "takes 2 inputs"),
    ("gather", [(3, 5), (4,)], {}, "broadcast"),
    ("gather", [((1 << 24) + 1,), (4,)], {}, "2\\^24"),
    ("bin_sum", [(3, 5), (3, 5)], {}, "bad rank"),
    ("bin_sum", [(3, 5), (3, 5)], dict(shape=(2, 1, 4)), "neither 1 nor"),
    ("bin_sum", [(3, 5), (3, 6)], dict(shape=(4,)), "broadcast"),
    ("bin_sum", [(3, 5), (3, 5)], dict(shape=(5000,)), "4096"),
    ("iota", [], dict(shape=(3, 4), axis=2), "axis"),
    ("iota", [], dict(shape=((1 << 24) + 1,), axis=0), "2\\^24"),
], ids=str)
def test_primitive_shapes_refused(op, shapes, attrs, what):
    g = Graph()
    ins = [g.input("f32", s) for s in shapes]
    with pytest.raises(KorchError, match=what):
        g.op(op, ins, "f32", **attrs)


# ---- kernels ---------------------------------------------------------------------


def _plans():
    for dtype, m, d in cases.LN:
        for name in ("layernorm", "layernorm_grad"):
            yield name, dict(m=m, d=d, dtype=dtype)
    for c in cases.FWD:
        yield "mha", cases._unpack(c)[0]
    for c in cases.GRAD:
        yield "mha_grad", cases._unpack(c)[0]


@pytest.mark.parametrize("name,sizes", list(_plans()), ids=str)
def test_fused_plans_compile_without_spills_or_load_hazards(name, sizes):
    w = graphs.build(name, **sizes)
    p = w.plan("fused")
    p.compile()
    fams = [p.kernel_info(k)[0] for k in range(p.num_kernels())]
    assert set(fams) <= {"row", "rowcol", "plane", "colreduce"} and (name[:3] != "mha" or "plane" in fams)
    for k in range(p.num_kernels()):
        code = p.kernel_code(k)
        for kernel, r in codeobj.kernel_resources(code).items():
            assert r["scratch"] == 0 and r["vgpr_spill"] == 0 and r["lds"] <= 160 * 1024, (kernel, r)
        loads, faults = lds_load_faults(disassemble(code))
        assert not faults, faults[:3]
        # plain products and sums only: packed fp32 arithmetic stays off
        assert not any(op.startswith("v_pk_") and op.endswith("_f32") for op, _ in disassemble(code))


def test_attention_is_one_kernel_and_its_gradient_evaluates_scores_twice():
    w = graphs.build("mha", n=300, heads=4, d=64, dtype="f16", causal=True)
    assert w.plan("fused").num_kernels() == 1
    w = graphs.build("mha_grad", n=300, heads=4, d=64, dtype="f16", causal=True)
    ks = w.plans["fused"]
    assert [sorted(o) for _, o in ks] == [["dQ", "delta"], ["dK", "dV"]]
    assert all("S0" in p for p, _ in ks)  # redundant execution
    assert w.plan("unfused").num_kernels() > 15


def test_rewritten_graphs_keep_their_results():
    """The graph transformations leave a masked attention's results as they are."""
    from paper_2406_09465_amd._abi import RW_ALL, RW_LAYOUT_VARIANTS
    sizes, x, _, want = cases._unpack(dict(dtype="f32", n=6, m=9, d=8, heads=4, kv_heads=2, causal=True, cap=2.0, slopes=True), grad=True)
    w = graphs.build("mha", **sizes)
    for rules in (RW_ALL, RW_LAYOUT_VARIANTS):
        g2, _ = w.graph.rewrite(rules)
        w2 = graphs.Workload("t", "f32", g2, {str(i): i for i in range(g2.num_nodes())}, [], [])
        o = _oracle_copy(w2)
        out = run_unfused(o, {str(i): x[k] for k, i in zip(w.input_names, g2.inputs())})
        for k, i in zip(w.output_names, g2.outputs()):
            assert np.allclose(out[str(i)], want[k][0], rtol=1e-9, atol=1e-11), (rules, k)


@pytest.mark.parametrize("case", cases.WIDE, ids=str)
def test_widest_gradients_compile(case):
    sizes = cases._unpack(case)[0]
    p = graphs.build("mha_grad", **sizes).plan("fused")
    p.compile()
    for k in range(p.num_kernels()):
        for kernel, r in codeobj.kernel_resources(p.kernel_code(k)).items():
            assert r["scratch"] == 0 and r["lds"] <= 160 * 1024, (kernel, r)


def test_a_masked_score_that_scores_may_lie_below():
    """The row maximum starts from the masked score: one of -100 is refused."""
    for low, family in ((-1e30, "plane"), (-100.0, "none")):
        w = cases._masked_rows(cases.MASKS["equal"][0], 60, 70, None, low)
        assert w.graph.family(*w.kernels("fused")[0]) == family


@pytest.mark.parametrize("cap", [float("inf"), float("nan")])
def test_caps_that_are_no_numbers(cap):
    with pytest.raises(ValueError):
        graphs.build("mha", n=8, heads=2, d=16, cap=cap)
