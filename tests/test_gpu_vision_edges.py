"""Group norm, rotary positions and gradient clipping on the GPU at the edges of
what they take, against plain float64 forms with bounds counted from the
definitions."""

import random

import numpy as np
import pytest

from paper_2406_09465_amd import graphs, search

from . import vision_ref as ref
from .test_gpu_vision_ops import _check, _clip_case, _gn_inputs, _gn_sizes, _rot_case, _rot_want, _run
from .test_vision_edges import ODD_HEADS, SPLITS, check_poisoned, poisoned, split_plan

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hh,dtype,plan", [(6, "f16", "fused"), (6, "f32", "layered"), (6, "f16", "unfused"), (100, "bf16", "fused"), (100, "f32", "fused")])
@pytest.mark.parametrize("act", graphs.ACTIVATIONS)
def test_a_group_that_is_no_number_stays_none(act, hh, dtype, plan):
    _, s, want, hit = poisoned(dtype, hh, act)
    z = dict(batch=3, hh=hh, ww=hh, c=48, groups=4, act=act, dtype=dtype)
    out = _run(graphs.build("groupnorm", **z), s, plan)
    g = {**s, "mu": out["mu"].astype(np.float32), "r": out["r"].astype(np.float32)}
    out.update(_run(graphs.build("groupnorm_grad", **z), g, plan))
    check_poisoned(out, want, hit, dtype)


@pytest.mark.parametrize("case", ODD_HEADS + [
    dict(dtype="f16", batch=7, heads=4, kv_heads=2, n=1, d=64, axes=2, first=3000),      # next tokens
    dict(dtype="f32", batch=2, heads=6, kv_heads=3, n=1, d=40, rot=24, packed=True),
    dict(dtype="f32", batch=3, heads=2, kv_heads=2, n=1, d=16, interleaved=True, axes=3),
], ids=str)
def test_rotary_and_gradient(case):
    """Heads that no rotary kernel takes, and single tokens of every type."""
    c, x, s = _rot_case(case)
    for name, want in zip(("rotary", "rotary_grad"), _rot_want(c, x)):
        out = _run(graphs.build(name, **c), s)
        assert set(out) == set(want)
        _check(out, want, c["dtype"])


WIDE = [
    ("f16", 1, 40, 41, 8192, 8192, "silu"),   # a channel to a group, split positions: the groups' numbers fill most of LDS
    ("f32", 2, 33, 40, 8192, 4096, "relu"),
    ("f32", 1, 50, 41, 8190, 8190, "none"),
    ("f32", 2, 40, 40, 4288, 2144, "silu"),   # 1024 threads, several vectors to each
    ("bf16", 1, 45, 41, 6395, 5, "relu"),     # and single elements
    ("f32", 30, 20, 21, 4288, 64, "silu"),    # an image to a workgroup
]


@pytest.mark.parametrize("case", WIDE, ids=str)
def test_wide_maps(case):
    z = _gn_sizes(case)
    x, s = _gn_inputs(*case[:5])
    want = ref.groupnorm(x["X"], x["gamma"], x["beta"], z["groups"], 1e-5, z["act"], z["dtype"], x["dY"])
    out = _run(graphs.build("groupnorm", **z), s, "layered")
    _check(out, want, z["dtype"], ("mu", "r"))
    g = {**s, "mu": out["mu"].astype(np.float32), "r": out["r"].astype(np.float32)}
    back = _run(graphs.build("groupnorm_grad", **z), g, "layered")
    _check(back, want, z["dtype"])
    assert set(out) | set(back) == set(want)


@pytest.mark.parametrize("case", [("f32", 2, 3, 5, 12, 4, "silu"), ("f32", 3, 70, 40, 12, 3, "relu"), ("f32", 3, 70, 40, 12, 3, "silu")], ids=str)
def test_gradients_with_an_activation_by_sampled_plans(case):
    """Random valid plans of the gradient's graph, of the group family's kernels and single primitives."""
    from paper_2406_09465_amd.runner import PlanRunner
    z = _gn_sizes(case)
    x, s = _gn_inputs(*case[:5])
    want = ref.groupnorm(x["X"], x["gamma"], x["beta"], z["groups"], 1e-5, z["act"], z["dtype"], x["dY"])
    s.update({k: want[k][0].astype(np.float32) for k in ("mu", "r")})
    w = graphs.build("groupnorm_grad", **z)
    cands = [c for c in w.graph.candidates(max_prims=6, max_outs=2, only_supported=True) if len(c[0]) == 1 or w.graph.family(*c) == "group"]
    wide, few = [c for c in cands if len(c[0]) > 3], [c for c in cands if len(c[0]) <= 2]
    view, rng = search.GraphView(w.graph), random.Random(7)
    for i in range(2):
        plan = search.random_plan(view, rng.sample(wide, min(len(wide), 60)) + few, rng)
        made = {o for _, outs in plan for o in outs}
        r = PlanRunner(w, kernels=plan + [([o], [o]) for o in w.graph.outputs() if o not in made])  # (views that are outputs)
        fams = [r.plan.kernel_info(k)[0] for k in range(r.plan.num_kernels())]
        print(f"\n[case] {case} plan {i}: {fams}", flush=True)
        assert "group" in fams
        out = r.run(s)
        assert set(out) == {"dX", "dgamma", "dbeta"}
        _check(out, want, z["dtype"])


@pytest.mark.parametrize("name,case,groups,families", SPLITS, ids=str)
def test_turns_in_several_kernels(name, case, groups, families):
    from paper_2406_09465_amd.runner import PlanRunner
    c, x, s = _rot_case(case)
    want = _rot_want(c, x)[name == "rotary_grad"]
    w = graphs.build(name, **c)
    out = PlanRunner(w, kernels=split_plan(w, groups)).run(s)
    assert set(out) == set(want)
    _check(out, want, c["dtype"])


def test_clipping_in_place_one_tensor_past_a_part():
    """201 gradients, the last one's product a kernel of its own, written over the gradients."""
    import torch
    from paper_2406_09465_amd.runner import PlanRunner
    case = dict(shapes=[(7 + i % 9, 3) for i in range(200)] + [(1001, 3)], dtype="f16")
    dt, x, s = _clip_case(case)
    want = ref.clipped(list(x.values()), dt, 0.5, 1e-6)
    r = PlanRunner(graphs.build("grad_clip", **case, max_norm=0.5), "fused")
    r.set_inputs(s)
    r.outs[1:] = r.ins
    r.launch()
    torch.cuda.synchronize()
    assert ref.outside(r.outs[0].double().cpu().numpy(), *want["norm"], "f32") <= 2.0  # (norms of parts are rounded too)
    for i, t in enumerate(r.outs[1:]):
        assert ref.outside(t.double().cpu().numpy(), *want[f"C{i}"], "f16") <= 1.0, i
