"""Group norm, rotary positions and gradient clipping at the edges of what they
take, without a GPU: what is no number, sizes that a kernel just takes or just
does not, and what the generated code needs."""

import numpy as np
import pytest

from oracle.graph import run_unfused
from paper_2406_09465_amd import codeobj, graphs, search
from paper_2406_09465_amd._abi import KorchError, Plan
from tests import test_gpu_vision_ops as cases
from tests import vision_ref as ref
from tests.test_layer_ops import _oracle_copy


def _oracle(name, x, **sizes):
    w = graphs.build(name, **sizes)
    return run_unfused(_oracle_copy(w), {k: x[k] for k in w.input_names})


# ---- what is no number ------------------------------------------------------------


def poisoned(dtype, hh, act):
    """Three images with a NaN in group 1 and an infinity in group 2 of the second; the
    plain results of what is not hit, and which elements of each result are."""
    x, s = cases._gn_inputs(dtype, 3, hh, hh, 48)
    want = ref.groupnorm(x["X"], x["gamma"], x["beta"], 4, 1e-5, act, dtype, x["dY"])
    s["X"] = s["X"].copy()
    x["X"] = x["X"].copy()
    for v, at in ((np.nan, (1, hh // 2, 3, 14)), (np.inf, (1, 0, 0, 30))):
        x["X"][at] = v
        s["X"][at] = ref.rounded(np.array([v]), dtype)[1][0]
    hit = np.zeros((3, 4), bool)
    hit[1, 1] = hit[1, 2] = True
    full = np.broadcast_to(np.repeat(hit, 12, axis=1)[:, None, None], x["X"].shape)
    chan = np.repeat(hit.any(0), 12)
    # without an activation dbeta is a sum of dY alone
    return x, s, want, dict(Y=full, dX=full, mu=hit, r=hit, dgamma=chan, dbeta=chan if act != "none" else np.zeros_like(chan))


def check_poisoned(out, want, hit, dtype):
    for k, bad in hit.items():
        v, b = want[k]
        if k == "mu":  # (a group with an infinity: its mean is infinite, or none where parts of it merge)
            assert np.isnan(out[k][1, 1]) and not np.isfinite(out[k][1, 2])
        else:
            assert np.all(np.isnan(out[k][bad])), k
        if not bad.all():
            assert ref.outside(out[k][~bad], v[~bad], b[~bad], "f32" if k in ("mu", "r") else dtype) <= 1.0, k


@pytest.mark.parametrize("act", graphs.ACTIVATIONS)
def test_a_group_that_is_no_number_stays_none(act):
    """Every result of such a group is NaN, the sums over its channels too, whatever the activation."""
    x, _, want, hit = poisoned("f32", 6, act)
    z = dict(batch=3, hh=6, ww=6, c=48, groups=4, act=act, dtype="f32")
    with np.errstate(invalid="ignore"):
        x.update(_oracle("groupnorm", x, **z))
        x.update(_oracle("groupnorm_grad", x, **z))
    check_poisoned(x, want, hit, "f32")


def test_relu_keeps_what_is_no_number_in_the_kernels():
    """The maximum instruction drops a NaN: the kernels compare and select."""
    for name in ("groupnorm", "groupnorm_grad"):
        w = graphs.build(name, batch=3, hh=6, ww=6, c=48, groups=4, act="relu", dtype="f16")
        for plan in ("fused", "layered"):
            for k in w.kernels(plan):
                body = w.graph.kernel_source(*k).split('extern "C"')[-1]
                assert "k_relu" not in body and "k_max" not in body


# ---- heads that no rotary kernel takes ----------------------------------------------

# neighbouring pairs in heads of odd width with grouped queries: the results differ in their heads
ODD_HEADS = [
    dict(dtype="f32", batch=1, heads=8, kv_heads=4, n=5, d=9, rot=4, interleaved=True),
    dict(dtype="f16", batch=2, heads=4, kv_heads=2, n=7, d=9, rot=8, interleaved=True, packed=True, axes=2),
    dict(dtype="bf16", batch=3, heads=6, kv_heads=2, n=1, d=33, rot=32, interleaved=True, axes=3, first=70000),
    dict(dtype="f32", batch=1, heads=2, kv_heads=2, n=3, d=5, rot=2, interleaved=True, packed=True),
]


@pytest.mark.parametrize("case", ODD_HEADS, ids=str)
def test_neighbours_in_odd_heads_have_a_fused_plan(case):
    c, x, _ = cases._rot_case(case)
    for name, want in zip(("rotary", "rotary_grad"), cases._rot_want(c, x)):
        w = graphs.build(name, **c)
        p = w.plan("fused").compile()
        assert p.num_kernels() <= len(w.output_names) and all(p.kernel_info(k)[0] == "pointwise" for k in range(p.num_kernels()))
        out = run_unfused(_oracle_copy(w), {k: x[k] for k in w.input_names})
        for k, (v, _) in want.items():
            assert np.allclose(out[k], v, rtol=1e-12, atol=1e-12), k


# ---- what a kernel needs of a compute unit -------------------------------------------


def _compiled(name, sizes, plan):
    """(family, resources) of every kernel of a plan."""
    p = graphs.build(name, **sizes).plan(plan).compile()
    return [(p.kernel_info(k)[0], r) for k in range(p.num_kernels()) for r in codeobj.kernel_resources(p.kernel_code(k)).values()]


@pytest.mark.parametrize("c,groups", [(8192, 8192), (8192, 4096), (8191, 8191), (8190, 2730)])
@pytest.mark.parametrize("dtype,batch,hh", [("f16", 1, 100), ("f32", 2, 64), ("bf16", 2, 64)])
def test_wide_maps_of_many_groups_compile(c, groups, dtype, batch, hh):
    """As many groups as channels, up to the widest maps: the groups' numbers fit LDS."""
    sizes = dict(batch=batch, hh=hh, ww=hh, c=c, groups=groups, dtype=dtype)
    for name in ("groupnorm", "groupnorm_grad"):
        for plan in ("fused", "layered"):
            for family, r in _compiled(name, sizes, plan):
                assert family == "group" and r["lds"] <= 160 * 1024


def test_sums_that_lds_does_not_hold_are_refused():
    """Five sums over the positions of 8192 channels (160 KiB of partial sums): no family, instead of an error of the compiler."""
    for c, family in ((8192, "none"), (4096, "group")):
        b = graphs._B("f32")
        prims, outs = [], []
        b.inp("X", (1, 3000, 1, c))
        b.inp("mu", (1, 1, 1, c))
        b.op("D", "sub", ["X", "mu"])
        prims.append("D")
        for i in range(5):
            b.op(f"x{i}", "mul", ["D"], scalar=float(i + 1))
            b.op(f"s{i}", "reduce_sum", [f"x{i}"], axis=1, keepdim=True)
            prims += [f"x{i}", f"s{i}"]
            outs.append(f"s{i}")
        w = graphs._finish(b, "sums", outs, {})
        kernel = [w.ids[p] for p in prims], [w.ids[o] for o in outs]
        assert w.graph.family(*kernel) == family
        assert w.graph.compile_candidate(*kernel) == (family != "none")


@pytest.mark.parametrize("name,dtype,batch,hh,ww,c,groups,act", [
    ("groupnorm", "f32", 1, 64, 64, 7200, 16, "silu"),
    ("groupnorm", "f32", 2, 64, 64, 4288, 2144, "relu"),       # more groups than threads
    ("groupnorm", "f32", 1, 64, 64, 6395, 6395, "none"),
    ("groupnorm", "f16", 1, 64, 64, 8191, 8191, "relu"),
    ("groupnorm_grad", "f32", 1, 64, 64, 4288, 32, "silu"),
    ("groupnorm_grad", "f32", 1, 64, 64, 6464, 32, "silu"),
    ("groupnorm_grad", "f32", 300, 16, 17, 4100, 10, "silu"),
    ("groupnorm_grad", "f32", 9, 64, 65, 7680, 32, "silu"),
    ("groupnorm_grad", "f32", 1, 100, 100, 8192, 4096, "silu"),
    ("groupnorm_grad", "f32", 300, 5, 3, 6395, 1, "relu"),
    ("groupnorm_grad", "f32", 1, 64, 64, 2606, 2606, "silu"),
    ("groupnorm_grad", "f16", 2, 64, 64, 6395, 5, "silu"),
    ("groupnorm_grad", "bf16", 300, 16, 17, 8191, 8191, "relu"),
    ("groupnorm_grad", "bf16", 300, 1, 7, 8191, 1, "silu"),
    ("groupnorm_grad", "f16", 9, 100, 100, 7285, 7285, "silu"),
    ("groupnorm_grad", "bf16", 1, 200, 150, 6395, 1279, "relu"),
    ("groupnorm", "f32", 300, 30, 41, 4288, 64, "silu"),
    ("groupnorm", "bf16", 2, 64, 64, 8192, 256, "silu"),
], ids=str)
def test_wide_maps_compile_without_spills(name, dtype, batch, hh, ww, c, groups, act):
    """Workgroups of 1024 threads have 128 registers for each."""
    sizes = dict(dtype=dtype, batch=batch, hh=hh, ww=ww, c=c, groups=groups, act=act)
    for plan in ("fused", "layered"):
        for family, r in _compiled(name, sizes, plan):
            assert family == "group" and r["scratch"] == 0 and r["vgpr_spill"] == 0


# ---- what is refused, exactly ---------------------------------------------------------


@pytest.mark.parametrize("c,groups,hh,first", [(8194, 2, 4, "none"), (8194, 2, 200, "none"), (8194, 34, 200, "none"), (8194, 34, 4, "group"), (8194, 8194, 4, "group"),
                                               (8192, 2, 4, "group")])
def test_past_the_widest_maps(c, groups, hh, first):
    """Past 8192 channels no kernel streams a map; a small map's groups still fit registers, in one kernel of all."""
    for name in ("groupnorm", "groupnorm_grad"):
        w = graphs.build(name, hh=hh, ww=hh, c=c, groups=groups)
        for plan in ("fused", "layered"):
            fams = [w.graph.family(*k) for k in w.kernels(plan)]
            if c == 8192:
                assert fams == ["group", "group"]
            elif plan == "fused" and first == "group":
                assert fams == ["group"]
            else:  # (what only applies statistics is a pointwise kernel's, too)
                assert fams == [first, "pointwise" if name == "groupnorm" else "none"]
            if "none" in fams:
                with pytest.raises(KorchError) as e:
                    w.plan(plan).compile()
                assert e.value.code == -20
        assert w.plan("unfused").num_kernels() > 15


def test_names_of_the_results():
    want = {"groupnorm": ["Y", "mu", "r"], "groupnorm_grad": ["dX", "dgamma", "dbeta"], "rotary": ["Qr", "Kr"], "rotary_grad": ["dQ", "dK"],
            "grad_clip": ["norm", "C0", "C1"]}
    for name, outs in want.items():
        w = graphs.build(name)
        assert w.output_names == outs
        for plan in w.plans:
            stored = [o for _, made in w.plans[plan] for o in made]
            assert set(outs) <= set(stored)
    assert graphs.build("rotary", packed=True).output_names == ["Qr", "Kr", "V"] and graphs.build("rotary_grad", packed=True).output_names == ["dQKV"]


@pytest.mark.parametrize("count", [199, 200, 201, 400, 401, 650])
def test_clipping_of_many_tensors(count):
    """A norm and a product for every 200 tensors, and the norm of the parts' norms."""
    w = graphs.build("grad_clip", shapes=[(3 + i % 5, 2) for i in range(count)], dtype="f16")
    fams = [w.graph.family(*k) for k in w.kernels("fused")]
    parts = -(-count // graphs.CLIP_TENSORS)
    assert len(fams) == (2 if parts == 1 else 2 * parts + 1)
    # (a product of one tensor alone is the pointwise family's)
    assert fams == ["multi"] * (len(fams) - 1) + ["pointwise" if count % graphs.CLIP_TENSORS == 1 else "multi"]


def split_plan(w, groups):
    """A plan whose kernels store the given results, each computed from the inputs and what earlier kernels stored."""
    view, stored, kernels = search.GraphView(w.graph), set(w.graph.inputs()), []

    def is_stored(v):
        return v in stored or (view.op[v] == "reshape" and is_stored(view.ins[v][0]))

    for outs in groups:
        outs = [w.ids[o] for o in outs]
        need, walk = set(), list(outs)
        while walk:
            v = walk.pop()
            if v not in need and not is_stored(v):
                need.add(v)
                walk += view.ins[v]
        kernels.append((sorted(need), outs))
        stored.update(outs)
    return kernels


PACKED = dict(dtype="f16", batch=2, heads=4, kv_heads=2, n=21, d=32, rot=24, axes=2, packed=True)
NEIGHBOURS = dict(dtype="f32", batch=3, heads=4, kv_heads=2, n=13, d=16, axes=3, interleaved=True, first=1000)
# (operator, sizes, results of each kernel, families)
SPLITS = [
    ("rotary", PACKED, [["co"], ["si"], ["Qr", "Kr", "V"]], ["pointwise", "pointwise", "rotary"]),
    ("rotary", PACKED, [["Qt"], ["Kt"], ["V"], ["Qr", "Kr"]], ["pointwise", "pointwise", "pointwise", "rotary"]),
    ("rotary", PACKED, [["Kr"], ["V"], ["Qr"]], ["rotary", "pointwise", "rotary"]),
    ("rotary", dict(PACKED, batch=1, heads=1, kv_heads=1), [["place"], ["V", "Kr", "Qr"]], ["pointwise", "rotary"]),
    ("rotary", NEIGHBOURS, [["place"], ["Qr", "Kr"]], ["pointwise", "rotary"]),
    ("rotary", NEIGHBOURS, [["co_i"], ["si_i"], ["Qr"], ["Kr"]], ["pointwise"] * 4),  # (stored angles of neighbours)
    ("rotary_grad", PACKED, [["dQ"], ["dK"], ["dQKV"]], ["rotary", "rotary", "pointwise"]),
    ("rotary_grad", dict(PACKED, interleaved=True), [["dQ", "dK"], ["dQKV"]], ["rotary", "pointwise"]),
    ("rotary_grad", dict(PACKED, interleaved=True), [["co"], ["si"], ["dQKV"]], ["pointwise"] * 3),
    ("rotary_grad", NEIGHBOURS, [["dQ"], ["dK"]], ["rotary", "rotary"]),
]


@pytest.mark.parametrize("name,case,groups,families", SPLITS, ids=str)
def test_turns_in_several_kernels_compile(name, case, groups, families):
    c = {k: v for k, v in case.items() if k != "first"}
    w = graphs.build(name, **c)
    p = Plan(w.graph, split_plan(w, groups)).compile()
    assert [p.kernel_info(k)[0] for k in range(p.num_kernels())] == families
