"""The loss over a table of classes and its gradients where numbers are far apart: loud rows, classes and columns, upstream gradients at the ends of the
range, padding in front, numbers that are no numbers beside padded rows."""
import numpy as np
import pytest

import paper_2206_08869_amd as iodf
import step_ref as ref
from test_gpu_blocks import as_type, dev, dtype, half_unit, host, near, on_gpu, torch
from test_gpu_step import NAMES, check_forward, long, on_card, some, spoiled, upstream

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def test_class_loss_rows_do_not_see_how_loud_others_are():
    """32 bits: a row's logits are as near as its own numbers make them."""
    u, w, target, _, _ = some(200, 300, 96, "f32", seed=31)
    for row, by in ((7, 1e8), (90, -1e8), (40, 1e-25)):
        u[row] = as_type(u[row] * by, "f32")
    check_forward(u, w, target, None, "f32")


def test_class_loss_classes_do_not_see_how_loud_others_are():
    """Some classes are loud in columns where half the rows have nothing, another is so everywhere and has no probability."""
    u, w, target, _, _ = some(200, 300, 96, "f32", seed=32)
    w[:, 5] = 0
    w[11, 5], w[250, 5] = 1e8, 3e7
    u[::2, 5] = 0
    u[1::2, 5] = -1
    target[np.isin(target, (11, 250))] = 3
    check_forward(u, w, target, None, "f32")
    u[:, 7], w[100], target[target == 100] = -1, 0, 101
    w[100, 7] = 1e30
    r = iodf.class_loss(dev(u), dev(w), long(target))
    rest = np.arange(300) != 100
    loss, lse, s = ref.loss(u, w[rest], target - (target > 100))
    slack = ref.logit_slack(u, w[rest]) + 64 * U * (1 + np.abs(lse) + np.abs(s).max(1))
    near(r.lse, lse, "f32", slack, "lse")
    near(r.loss, loss, "f32", 2 * slack, "loss")


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("classes", [300, 2000])
def test_class_loss_of_huge_logits(name, classes):
    """Logits whose 24 bits end above 1."""
    u, w, target, _, _ = some(200, classes, 96, name, seed=40)
    for row, by in ((7, 1e12), (90, 1e20), (199, 1e30)):
        u[row] = as_type(u[row] * by, name)
    check_forward(u, w, target, None, name)


def test_class_loss_loud_columns_of_small_weights():
    u, w, target, _, _ = some(150, 200, 96, "f32", seed=33)
    u[:, 3], w[:, 3] = as_type(u[:, 3] * 1e8, "f32"), as_type(w[:, 3] * 1e-8, "f32")
    check_forward(u, w, target, None, "f32")


def gradients(u, w, target, live, name, dloss, dlse):
    lse = ref.loss(u, w, target, live)[1].astype(np.float32)
    got = iodf.class_loss_backward(dev(u, name), dev(w, name), long(target), dev(lse), *(None if d is None else dev(d) for d in (dloss, dlse)), live=on_gpu(live))
    return got, lse.astype(np.float64)


@pytest.mark.parametrize("rows,classes,cols", [(150, 270, 96), (600, 900, 264), (20, 3000, 130), (300, 40, 520)])
def test_class_loss_gradients_of_loud_numbers(rows, classes, cols):
    """32 bits: one number of a row, one of a class and a whole column are far louder than all others, each where the other tensor has nothing or next to nothing: what they
    meet is exact, and what they do not meet is as near as its own numbers make it."""
    u, w, target, _, rng = some(rows, classes, cols, "f32", seed=34)
    w[:, 1], u[:, 2] = 0, 0
    u[rows // 2, 1], w[classes // 2, 2] = 1e10, 1e12
    u[:, 3], w[:, 3] = as_type(u[:, 3] * 1e9, "f32"), as_type(w[:, 3] * 1e-9, "f32")
    up = upstream(rng, rows, "both")
    up[0][rows // 3], up[1][rows // 3] = 1e6, 1e6
    got, lse = gradients(u, w, target, None, "f32", *up)
    du, dw, eu, ew = ref.gradients_by_the_parts(u, w, target, lse, *up, None, U)
    near(got[0], du, "f32", eu, "du")
    near(got[1], dw, "f32", ew, "dweight")


def test_class_loss_gradients_without_a_diverged_row():
    """32 bits: a live row whose upstream gradient is 0 may be as loud as it likes."""
    u, w, target, _, rng = some(200, 300, 96, "f32", seed=35)
    up = upstream(rng, 200, "both")
    for row, by in ((3, 1e8), (77, 1e25)):
        u[row] = as_type(u[row] * by, "f32")
        up[0][row] = up[1][row] = 0
    got, lse = gradients(u, w, target, None, "f32", *up)
    rest = np.ones(200, bool)
    rest[[3, 77]] = False
    du, dw, eu, ew = ref.gradients_by_the_parts(u[rest], w, target[rest], lse[rest], up[0][rest], up[1][rest], None, U)
    near(got[0][torch().from_numpy(rest).cuda()], du, "f32", eu, "du")
    near(got[1], dw, "f32", ew, "dweight")
    assert not got[0][[3, 77]].any()


@pytest.mark.parametrize("quiet", ["padded", "masked"])
@pytest.mark.parametrize("rows", [400, 2000])
def test_class_loss_gradient_s_rounding_is_not_the_same_in_all_rows(quiet, rows):
    """bfloat16, the same dloss in every row but the first hundred, half way between two neighbours: multiplied so that it is a power of two, gradients that are dloss
    itself are exact, and a result is off by its own rounding alone. The rows' targets have next to no probability and another class has next to all."""
    rng = np.random.default_rng(36)
    classes, cols, d = 400, 200, (1 + 2.0 ** -8) * 2.0 ** -9
    w = as_type(rng.standard_normal((classes, cols)), "bf16")
    sure, target = rng.integers(0, classes, rows), rng.integers(0, classes, rows)
    target = np.where(sure == target, (target + 1) % classes, target)
    u = as_type(w[sure], "bf16")  # a logit of 200, others far below
    dloss = np.full(rows, d)
    live = None
    if quiet == "padded":
        live = np.arange(rows) >= 100
    else:
        dloss[:100] = 0
    got, lse = gradients(u, w, target, live, "bf16", dloss, None)
    du, dw, _, _ = ref.loss_backward(u, w, target, lse, dloss, None, live, "f32")
    for a, b in zip(got, (du, dw)):
        assert np.linalg.norm(host(a) - b) <= 1.01 * np.linalg.norm(half_unit("bf16", b))


def test_class_loss_gradients_at_the_end_of_the_range():
    """bfloat16: dloss near the largest number of 32 bits."""
    u, w, target, _, _ = some(400, 300, 200, "bf16", seed=37)
    dloss = np.full(400, np.float64(np.float32(1e30)))
    dloss[5] = dloss[0] = np.float64(np.float32(2.5e38))
    w = as_type(w * 2.0 ** -10, "bf16")
    u = as_type(u * 2.0 ** -10, "bf16")
    (a, b), lse = gradients(u, w, target, None, "bf16", dloss, None)
    du, dw, eu, ew = ref.loss_backward(u, w, target, lse, dloss, None, None, "bf16")
    near(a, du, "bf16", eu, "du")
    near(b, dw, "bf16", ew, "dweight")


@pytest.mark.parametrize("rows,classes,cols", [(9, 300, 96), (150, 270, 96), (300, 513, 200), (40, 200, 4100)])
@pytest.mark.parametrize("name", NAMES)
def test_padded_rows_have_no_gradient_whatever_the_table_holds(rows, classes, cols, name):
    u, w, target, live, _ = some(rows, classes, cols, name, seed=38, dead=0.4)
    live[0], live[-1] = True, False
    w[classes // 2, 1], w[classes - 1, 2] = np.inf, np.nan
    t = torch()
    du, _ = iodf.class_loss_backward(dev(u, name), dev(w, name), long(target), t.ones(rows, device="cuda"), t.ones(rows, device="cuda"), live=on_gpu(live))
    assert not host(du)[~live].any() and not np.isfinite(host(du)[live]).all()


@pytest.mark.parametrize("rows", [12, 300])
@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_rows_without_upstream_gradient_stay_out_whatever_their_logits(name, rows):
    """Logits so large that the two passes' roundings of them lie a thousand apart: a probability is at most 1 for all that, and nothing times it is nothing."""
    u, w, target, _, rng = some(rows, 400, 200, name, seed=39)
    up = upstream(rng, rows, "both")
    rest = np.ones(rows, bool)
    for row, by in ((0, 1e10), (rows // 4, 1e15), (rows - 1, 1e25)):
        u[row] = as_type(u[row] * by, name)
        up[0][row] = up[1][row] = 0
        rest[row] = False
    got, lse = gradients(u, w, target, None, name, *up)
    du, dw, eu, ew = ref.loss_backward(u[rest], w, target[rest], lse[rest], up[0][rest], up[1][rest], None, name)
    near(got[0][torch().from_numpy(rest).cuda()], du, name, eu, "du")
    near(got[1], dw, name, ew, "dweight")
    assert not got[0][torch().from_numpy(~rest).cuda()].any()


@pytest.mark.parametrize("rows,classes,cols,name", [(2049, 3001, 768, "bf16"), (4096, 8192, 320, "bf16"), (600, 5003, 264, "f32"), (600, 5003, 264, "f16"),
                                                   (20, 9000, 130, "f32"), (5000, 40, 700, "bf16")])
def test_a_gradient_has_the_same_bits_with_the_other_and_without(rows, classes, cols, name):
    t = torch()
    u, w, target, d = on_card(rows, classes, cols, name, 41)
    lse = iodf.class_loss(u, w, target).lse
    both = iodf.class_loss_backward(u, w, target, lse, d)
    assert t.equal(iodf.class_loss_backward(u, w, target, lse, d, need=(True, False))[0], both[0])
    assert t.equal(iodf.class_loss_backward(u, w, target, lse, d, need=(False, True))[1], both[1])


def test_many_large_matrices_go_a_few_at_a_time():
    """2^26 elements at a time: the bits of calls with as many."""
    t = torch()
    gen = t.Generator("cuda").manual_seed(42)
    g = t.randn((5, 4096, 4096), generator=gen, device="cuda").bfloat16()
    got = iodf.orthogonalise(g)
    assert t.equal(got[:4], iodf.orthogonalise(g[:4])) and t.equal(got[4:], iodf.orthogonalise(g[4:]))
    w, m = [t.zeros_like(x) for x in g], [t.zeros((4096, 4096), device="cuda") for _ in g]
    iodf.muon_step(w, list(g), m, 1.0, beta=0.0, nesterov=False, scale=-1.0)
    assert all(t.equal(a, b) for a, b in zip(w, got)) and all(t.equal(a, b.float()) for a, b in zip(m, g))


@pytest.mark.parametrize("rows,classes,cols,name", [(300, 400, 200, "f32"), (300, 400, 200, "bf16"), (20, 5000, 130, "f32"), (1000, 80, 300, "f32"), (40, 90, 64, "bf16")])
def test_class_loss_gradients_of_classes_that_are_no_targets(rows, classes, cols, name):
    """Their gradients are probabilities alone, here 1e-8 to 1e-15 of the others', and as near in themselves as those are."""
    u, w, target, _, rng = some(rows, classes, cols, name, seed=43)
    rare = np.arange(classes) % 3 == 1
    u[:, 0], w[:, 0] = 1, 0
    w[rare, 0] = -as_type(rng.uniform(18, 34, rare.sum()), name)
    target[rare[target]] = 0
    up = (np.full(rows, np.float64(np.float32(1.0 / rows))), None)
    got, lse = gradients(u, w, target, None, name, *up)
    step = U if name == "f32" else 2.0 ** -16 if cols <= 128 else 2.0 ** -8
    du, dw, eu, ew = ref.gradients_by_the_parts(u, w, target, lse, *up, None, step)
    assert 0 < np.abs(dw[rare]).max() < 1e-6 * np.abs(dw[~rare]).max()
    for a, b, off in ((got[0], du, eu), (got[1], dw, ew)):
        near(a, b, name, off + 1.01 * (half_unit(name, np.abs(b) + off) - half_unit(name, b)), "gradient")
    assert np.linalg.norm(host(got[1])[rare] - dw[rare]) <= {"f32": 1e-5, "bf16": 2.0 ** -8}[name] * np.linalg.norm(dw[rare])


MASKED = [(9, 300, 96), (100, 300, 96), (30, 300, 96), (300, 513, 200), (40, 200, 4100), (500, 600, 264)]


@pytest.mark.parametrize("rows,classes,cols", MASKED)
@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("mask", ["infinity", "lowest"])
def test_classes_masked_through_a_column_of_ones(rows, classes, cols, name, mask):
    """A mask of minus infinity, or of the type's lowest number, in a column of the table that every row multiplies with 1: those classes have no probability and the others are as without
    them. An infinity times g, which is 0 there, makes that column of du NaN, and nothing else."""
    t = torch()
    u, w, target, live, rng = some(rows, classes, cols, name, seed=44, dead=0.2)
    live[0] = True
    masked = np.arange(classes) % 4 == 2
    masked[-1] = True
    target[masked[target]] = 0
    u[:, 5], w[:, 5] = 1, 0
    rest = np.flatnonzero(~masked)
    w[masked, 5] = -np.inf if mask == "infinity" else float(t.finfo(dtype(name)).min)
    place = np.cumsum(~masked) - 1
    loss, lse, s = ref.loss(u, w[rest], place[target], live)
    su, st = spoiled(u, target, live)
    r = iodf.class_loss(dev(su, name), dev(w, name), long(st), live=on_gpu(live))
    slack = ref.logit_slack(u, w[rest], live) + 64 * U * (1 + np.abs(lse) + np.abs(s).max(1))
    near(r.lse, lse, "f32", slack, "lse")
    near(r.loss, loss, "f32", 2 * slack, "loss")
    up = upstream(rng, rows, "both")
    lse32 = lse.astype(np.float32)
    got = iodf.class_loss_backward(dev(su, name), dev(w, name), long(st), dev(lse32), dev(up[0]), dev(up[1]), live=on_gpu(live))
    du, dw, eu, ew = ref.loss_backward(u, w[rest], place[target], lse32.astype(np.float64), *up, live, name)
    columns = np.arange(cols) != 5
    more = lambda b, off: off + 1.01 * (half_unit(name, np.abs(b) + off) - half_unit(name, b))  # noqa: E731
    near(got[0][:, t.from_numpy(columns).cuda()], du[:, columns], name, more(du, eu)[:, columns], "du")
    near(got[1][t.from_numpy(rest).cuda()], dw, name, more(dw, ew), "dweight")
    assert not got[1][t.from_numpy(masked).cuda()].any() and (mask == "infinity" or not got[0][:, 5].isnan().any())


@pytest.mark.parametrize("rows,classes,cols", [(10, 90, 64), (80, 90, 64), (300, 513, 200)])
@pytest.mark.parametrize("name", NAMES)
def test_a_row_that_is_no_number_has_a_gradient_that_is_none(rows, classes, cols, name):
    u, w, target, _, rng = some(rows, classes, cols, name, seed=45)
    u[4, 9] = np.nan
    t = torch()
    lse = iodf.class_loss(dev(u, name), dev(w, name), long(target)).lse
    du, dw = iodf.class_loss_backward(dev(u, name), dev(w, name), long(target), lse, t.full((rows,), 0.1, device="cuda"))
    rest = np.arange(rows) != 4
    assert np.isnan(host(du)[4]).all() and np.isfinite(host(du)[rest]).all() and np.isnan(host(dw)).all()
