"""What the bounds of gradients are worth, on the CPU: g rounded to one part of 16 bits breaks those that hold where it has two."""
import numpy as np
import pytest

import step_ref as ref
from test_gpu_blocks import as_type, half_unit
from test_gpu_step import some, upstream
from test_gpu_step_parts import FINE, rounded as more


def rounded(name, parts, g):
    """g in so many parts of the type, scaled as the library says: by the first dloss in bfloat16, to the top of the range in half precision."""
    lift = 1.0 if name == "bf16" else 2.0 ** (14 - np.ceil(np.log2(np.abs(g).max())))
    left, kept = g * lift, 0.0
    for _ in range(parts):
        part = as_type(left, name)
        left, kept = left - part, kept + part
    return kept / lift


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("rows,classes,cols", [(16, 4099, 512), (1, 5000, 1030), (700, 2, 130), (63, 31, 65), (64, 257, 200), (21, 600, 300)])
def test_a_lost_second_part_breaks_the_bound(rows, classes, cols, name):
    u, w, target, live, rng = some(rows, classes, cols, name, seed=54)
    up = upstream(rng, rows, "both")
    lse = ref.loss(u, w, target, live)[1].astype(np.float32).astype(np.float64)
    least = 2.0 ** -38 * max(np.abs(up[0]).max(), np.abs(up[0] + up[1]).max()) if name == "f16" else 0.0
    du, dw, eu, ew = ref.gradients_by_the_parts(u, w, target, lse, *up, live, FINE[name], least)
    g = np.exp(u @ w.T - lse[:, None]) * (up[0] + up[1])[:, None]
    g[np.arange(rows), target] -= up[0]
    worst = {}
    for parts in (1, 2):
        of = rounded(name, parts, g)
        over = [np.abs(as_type(got, name) - want) - half_unit(name, want) * 1.01 - more(want, off, name) for got, want, off in ((of @ w, du, eu), (of.T @ u, dw, ew))]
        worst[parts] = max(x.max() for x in over)
    assert worst[2] <= 0 < worst[1]
