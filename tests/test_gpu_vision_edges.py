"""Group norm, rotary positions and gradient clipping on the GPU at the edges of
what they take, against plain float64 forms with bounds counted from the
definitions."""

import numpy as np
import pytest

from paper_2406_09465_amd import graphs

from .test_gpu_vision_ops import _run
from .test_vision_edges import check_poisoned, poisoned

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
