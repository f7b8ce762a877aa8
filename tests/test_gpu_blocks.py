"""The training operators on the GPU against their plain forms in 64 bits (blocks_ref.py).

Tolerances come from the arithmetic: an output is the exact value, off by half a unit of its own type and by a few dozen roundings of
32-bit floats, each relative to what is added up at that place (SLACK units of 2^-24 of the terms' magnitudes; a sum over rows adds
its terms one after the other over at most a few hundred of them, and may be off by as many units). Codes of given numbers are exact; codes of
computed numbers may be one step off where the number lies on a border, so they are held to half a step and a hair."""
import ctypes

import numpy as np
import pytest

import blocks_ref as ref
import paper_2206_08869_amd as iodf

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SLACK = 64


def torch():
    import torch as t
    return t


def dtype(name):
    t = torch()
    return {"f32": t.float32, "bf16": t.bfloat16, "f16": t.float16}[name]


def half_unit(name, want):
    """Half the distance of the type's neighbouring numbers at `want`: the types have 24, 8 and 11 significant bits."""
    bits, least = {"f32": (24, -149), "bf16": (8, -133), "f16": (11, -24)}[name]
    return 0.5 * np.exp2(np.maximum(np.frexp(want)[1] - bits, least).astype(np.float64))


def dev(a, name="f32"):
    t = torch()
    return t.from_numpy(np.ascontiguousarray(a)).cuda().to(dtype(name))


def host(x):
    return x.detach().double().cpu().numpy()


def near(got, want, name, slack, what):
    """|got - want| within half a unit of the type, and slack (same shape or broadcast) more."""
    got = host(got)
    assert got.shape == want.shape, what
    assert np.isfinite(got).all(), what
    off = np.abs(got - want) - half_unit(name, want) * 1.01 - slack
    assert got.size == 0 or off.max() <= 0, (what, float(off.max()), np.unravel_index(off.argmax(), off.shape))


def codes_near(codes, want, what):
    """Codes of computed numbers: exponents as 64 bits give them or, on a border, one off; values within half a step and a hair of it."""
    q, e = codes.q.cpu().numpy(), codes.e.cpu().numpy().astype(np.int64)
    top = np.abs(ref.groups(want)).max(2) if want.size else np.zeros(e.shape)
    assert ((e == ref.exponents(top * (1 - 1e-5))) | (e == ref.exponents(top * (1 + 1e-5)))).all(), what
    step = np.repeat(np.exp2(e - 133.0), 32, 1)[:, :want.shape[1]]
    off = np.abs(ref.decode(q, e, want.shape[1]) - want)
    assert off.size == 0 or (off <= 0.5 * step * (1 + 1e-2)).all(), (what, float((off / step).max()))
    assert not q[:, want.shape[1]:].any(), what + ": columns past the last are 0"


def spread(rng, *shape):
    return rng.standard_normal(shape) * np.exp(0.5 * rng.standard_normal(shape[-1]))


def as_type(a, name):
    """a rounded to the type, as float64."""
    t = torch()
    return t.from_numpy(np.ascontiguousarray(a)).to(dtype(name)).double().numpy()


def some_live(rng, rows, mode):
    if mode == "all":
        return None
    if mode == "none":
        return np.zeros(rows, bool)
    live = rng.random(rows) < 0.7
    return live


def on_gpu(live):
    return None if live is None else torch().from_numpy(live).cuda()


# ---- checkpoints of given tensors: exact ----

SHAPES = [(1, 1), (1, 7), (3, 33), (65, 8), (130, 100), (33, 129), (5, 257), (1000, 40), (9, 513), (4, 1111), (2, 4097), (1, 65536), (0, 40)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("name", ["f32", "bf16", "f16"])
def test_pack_is_exact(rows, cols, name):
    rng = np.random.default_rng(rows * 7 + cols)
    v = as_type(spread(rng, rows, cols) * np.exp(2 * rng.standard_normal((rows, 1))), name)
    c = iodf.pack(dev(v, name))
    q, e = ref.encode(v)
    assert np.array_equal(c.q.cpu().numpy(), q) and np.array_equal(c.e.cpu().numpy(), e)
    want = ref.decode(q, e, cols)
    for out in ("bf16", "f32"):
        assert np.array_equal(host(iodf.unpack(c, dtype(out))), want)   # both types hold every value


def test_pack_at_the_edges():
    """Signed zeros, ties, the border of 127.5 steps, the smallest and largest numbers, infinities and NaN (only their own group)."""
    v = np.zeros((8, 96), np.float32)
    v[0, 0], v[0, 1] = -0.0, 0.0
    v[1, :5] = [127.0, 0.5, 1.5, -2.5, -127.0]
    v[2, 0], v[2, 40] = 127.5, np.nextafter(np.float32(127.5), np.float32(0))
    v[3, 0], v[3, 40], v[3, 80] = 1e-45, -1.1754944e-38, 1e-33
    v[4, 0], v[4, 40] = np.finfo(np.float32).max, -3.3895314e38   # the lowest bfloat16
    v[5, 3], v[5, 4] = np.inf, 1.0
    v[6, 70], v[6, 1] = np.nan, 2.0
    v[7, 95] = -np.inf
    x = torch().from_numpy(v).cuda()
    c = iodf.pack(x)
    q, e = ref.encode(v.astype(np.float64))
    assert np.array_equal(c.q.cpu().numpy(), q) and np.array_equal(c.e.cpu().numpy(), e)
    back = host(iodf.unpack(c))
    assert np.array_equal(np.isnan(back), np.repeat(e == 255, 32, 1)) and (e == 255).sum() == 3
    want = ref.decode(q, e, 96)
    assert np.array_equal(back[~np.isnan(back)], want[~np.isnan(want)])


def test_pack_leaves_padding_out():
    rng = np.random.default_rng(1)
    v = rng.standard_normal((50, 70)).astype(np.float32)
    live = rng.random(50) < 0.5
    v[~live] = np.nan
    c = iodf.pack(torch().from_numpy(v).cuda(), live=on_gpu(live))
    q, e = ref.encode(np.where(live[:, None], v, 0).astype(np.float64))
    assert np.array_equal(c.q.cpu().numpy(), q) and np.array_equal(c.e.cpu().numpy(), e)


@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_pack_takes_strided_rows_at_any_element(name):
    rng = np.random.default_rng(2)
    v = as_type(rng.standard_normal((40, 200)), name)
    for first, last in ((0, 64), (1, 66), (3, 200), (5, 6)):
        c = iodf.pack(dev(v, name)[:, first:last])
        q, e = ref.encode(v[:, first:last])
        assert np.array_equal(c.q.cpu().numpy(), q) and np.array_equal(c.e.cpu().numpy(), e)


# ---- join ----

def join_case(seed, rows, cols, stream, block, groups, mode, what="agpq"):
    rng = np.random.default_rng(seed)
    live = some_live(rng, rows, mode)
    p = dict(h=as_type(spread(rng, rows, cols), stream), f=as_type(0.3 * spread(rng, rows, cols), block),
             alpha=np.float32([0.7]) if "a" in what else None,
             gate=(rng.random((groups, cols)) if groups > 1 else rng.random(cols)).astype(np.float32) if "g" in what else None,
             w_post=(1 + 0.2 * rng.standard_normal(cols)).astype(np.float32) if "p" in what else None,
             w_pre=(1 + 0.2 * rng.standard_normal(cols)).astype(np.float32) if "q" in what else None)
    if live is not None:
        p["f"][~live] = np.nan
    return rng, p, live


def params_on_gpu(p):
    return [None if p[k] is None else dev(p[k]) for k in ("alpha", "gate", "w_post", "w_pre")]


JOINS = [  # rows, cols, stream, block, gate groups, live rows, which parameters there are
    (1, 1, "f32", "f32", 1, "all", "agpq"), (3, 7, "bf16", "bf16", 1, "all", "agpq"), (70, 33, "f32", "bf16", 1, "some", "agpq"),
    (65, 64, "f16", "f16", 5, "all", "agpq"), (90, 100, "f32", "f16", 90, "some", "agpq"), (64, 128, "bf16", "bf16", 4, "some", "agpq"),
    (33, 257, "f32", "f32", 1, "some", "agpq"), (40, 512, "bf16", "bf16", 1, "all", "agpq"), (21, 513, "f32", "f32", 21, "all", "agpq"),
    (36, 1000, "bf16", "bf16", 3, "some", "agpq"), (14, 1111, "f32", "f32", 7, "some", "agpq"), (5, 2049, "f32", "bf16", 1, "all", "agpq"),
    (8, 4096, "bf16", "bf16", 2, "some", "agpq"), (6, 4097, "f32", "f32", 1, "some", "agpq"), (3, 8193, "bf16", "bf16", 3, "all", "agpq"),
    (4, 16384, "f32", "bf16", 1, "some", "agpq"), (50, 96, "f32", "f32", 1, "none", "agpq"), (2, 5000, "f32", "f32", 1, "none", "agpq"),
    (40, 96, "bf16", "bf16", 1, "some", "agp"), (40, 96, "f32", "bf16", 1, "some", "agq"), (40, 640, "f32", "f32", 4, "some", "gq"),
    (40, 2100, "f32", "f32", 1, "some", "pq"), (40, 2100, "f32", "f32", 1, "all", "q"), (40, 64, "f32", "f32", 1, "all", "p"),
    (40, 64, "f32", "f32", 1, "all", ""), (3000, 24, "f32", "f32", 1, "some", "agpq"), (3000, 24, "f32", "f32", 1500, "some", "agpq"),
    (5000, 72, "bf16", "bf16", 2, "all", "agpq"), (0, 40, "f32", "f32", 1, "all", "agpq")]


@pytest.mark.parametrize("rows,cols,stream,block,groups,mode,what", JOINS)
def test_join_forward(rows, cols, stream, block, groups, mode, what):
    rng, p, live = join_case(rows + cols, rows, cols, stream, block, groups, mode, what)
    r = ref.join(live=live, eps=1e-5, **p)
    h, f = dev(p["h"], stream), dev(p["f"], block)
    h2, u, saved = iodf.join(h, f, *params_on_gpu(p), live=on_gpu(live), eps=1e-5)
    scale = np.abs(r["h"]).max(1, keepdims=True, initial=0) + np.abs(r["n"]).max(1, keepdims=True, initial=0)
    near(h2, r["h"], stream, SLACK * U * scale, "h'")
    near(saved.inv_post if "p" in what else dev(r["inv_post"]), r["inv_post"], "f32", SLACK * U * np.abs(r["inv_post"]), "inv_post")
    codes_near(saved.n, r["n"], "n")
    if "q" in what:
        near(u, r["u"], block, SLACK * U * np.abs(r["x"]).max(1, keepdims=True, initial=0) * 2, "u")
        near(saved.inv_pre, r["inv_pre"], "f32", SLACK * U * np.abs(r["inv_pre"]), "inv_pre")
        codes_near(saved.x, r["x"], "x")
    else:
        assert u is None and saved.x is None and saved.inv_pre is None
    # the form that keeps nothing, in place: the same numbers
    h3, u3, none = iodf.join(h, f, *params_on_gpu(p), live=on_gpu(live), eps=1e-5, save=False, h_out=h)
    assert none is None and h3 is h and torch().equal(h3, h2) and (u3 is None or torch().equal(u3, u))


@pytest.mark.parametrize("rows,cols,stream,block,groups,mode,what", JOINS)
def test_join_backward(rows, cols, stream, block, groups, mode, what):
    rng, p, live = join_case(rows + cols, rows, cols, stream, block, groups, mode, what)
    alive = np.ones(rows, bool) if live is None else live
    x, n = spread(rng, rows, cols), spread(rng, rows, cols)
    x[~alive], n[~alive] = 0, 0
    iq, ip = (0.5 + rng.random(rows)).astype(np.float32) * alive, (0.5 + rng.random(rows)).astype(np.float32) * alive
    dh, du = as_type(spread(rng, rows, cols), stream), as_type(spread(rng, rows, cols), block)
    du[~alive] = np.nan
    codes = [iodf.Codes(torch().from_numpy(q).cuda(), torch().from_numpy(e).cuda(), cols) for q, e in map(ref.encode, (x, n))]
    x, n = (ref.decode(*ref.encode(v), cols) for v in (x, n))
    saved = iodf.JoinSaved(codes[0], codes[1], dev(iq), dev(ip))
    gp = params_on_gpu(p)
    args = (saved, dev(dh, stream), dev(du, block) if "q" in what else None, *gp)
    g = iodf.join_backward(*args, live=on_gpu(live), block_dtype=dtype(block))
    al, wp, wq = (1 if p[k] is None else p[k].astype(np.float64) for k in ("alpha", "w_post", "w_pre"))
    r = ref.join_backward(x, n, iq.astype(np.float64), ip.astype(np.float64), dh, du, p["alpha"], p["gate"], p["w_post"], p["w_pre"], live)
    du0 = np.where(alive[:, None], du, 0)

    def row_mean(v):
        return np.abs(v).mean(1, keepdims=True) if cols else v

    # what is added up in dh: dh', dx, x mean(dx x); and behind the norm, from that
    mass = np.abs(dh) + (iq[:, None] * (np.abs(du0 * wq) + np.abs(x) * row_mean(du0 * wq * x)) if "q" in what else 0)
    near(g.dh, r["dh"], stream, SLACK * U * mass, "dh")
    coef = np.abs(al * wp * ref.per_row(p["gate"], rows, cols))
    mass_n = coef * mass * alive[:, None]
    mass_f = ip[:, None] * (mass_n + np.abs(n) * (mass_n * np.abs(n)).mean(1, keepdims=True)) if "p" in what else mass_n
    near(g.df, r["df"], block, SLACK * U * mass_f, "df")
    runs = min(rows, 512) + SLACK
    share = mass * np.abs(n) * alive[:, None]
    if "a" in what:
        near(g.dalpha, r["dalpha"], "f32", runs * U * (coef * share).sum() / abs(al), "dalpha")
    if "g" in what:
        near(g.dgate, r["dgate"], "f32", (runs * U * np.abs(al * wp) * share.reshape(groups, -1, cols).sum(1)).reshape(r["dgate"].shape), "dgate")
    if "p" in what:
        near(g.dw_post, r["dw_post"], "f32", runs * U * (np.abs(al) * ref.per_row(p["gate"], rows, cols) * share).sum(0), "dw_post")
    if "q" in what:
        near(g.dw_pre, r["dw_pre"], "f32", runs * U * np.abs(du0 * x).sum(0), "dw_pre")
    again = iodf.join_backward(*args, live=on_gpu(live), block_dtype=dtype(block))
    for a, b in zip(g, again):   # the same bits: no sum's order is left to chance
        assert (a is None) == (b is None) and (a is None or torch().equal(a, b))


@pytest.mark.parametrize("rows,cols,stream,block,groups,mode,what", [
    (600, 8200, "bf16", "bf16", 1, "some", "agpq"), (520, 9001, "f32", "f32", 2, "some", "agpq"), (530, 8201, "f16", "f16", 530, "some", "agpq"),
    (300, 8833, "f32", "bf16", 1, "some", "agp"), (3, 16383, "f32", "f16", 1, "all", "gq")])
def test_join_backward_of_rows_past_8192_columns(rows, cols, stream, block, groups, mode, what):
    """Rows that are not held but read twice: several to a run, padded ones between them."""
    test_join_backward(rows, cols, stream, block, groups, mode, what)


def test_join_backward_at_a_residual_scale_of_zero():
    """Where residual scales start: nothing of the block is in the stream, its gradients are 0, the scale's own is not."""
    rng, p, live = join_case(8, 60, 200, "f32", "bf16", 3, "some")
    p["alpha"] = np.float32([0.0])
    h2, u, saved = iodf.join(dev(p["h"]), dev(p["f"], "bf16"), *params_on_gpu(p), live=on_gpu(live))
    assert np.array_equal(host(h2), p["h"].astype(np.float32))
    dh, du = rng.standard_normal((60, 200)).astype(np.float32), as_type(rng.standard_normal((60, 200)), "bf16")
    g = iodf.join_backward(saved, dev(dh), dev(du, "bf16"), *params_on_gpu(p), live=on_gpu(live))
    x, n = (ref.decode(c.q.cpu().numpy(), c.e.cpu().numpy(), 200) for c in (saved.x, saved.n))
    r = ref.join_backward(x, n, host(saved.inv_pre), host(saved.inv_post), dh, du, p["alpha"], p["gate"], p["w_post"], p["w_pre"], live)
    assert not host(g.df).any() and not host(g.dgate).any() and not host(g.dw_post).any()
    mass = (np.abs(r["dh"]) * ref.per_row(p["gate"], 60, 200) * np.abs(p["w_post"] * n)).sum()
    assert abs(host(g.dalpha)[0] - r["dalpha"][0]) <= 2 * SLACK * U * mass and abs(r["dalpha"][0]) > 0


def test_join_backward_keeps_what_stands_in_padded_rows_to_itself():
    """NaN in dL/dh' of a padded row comes out where it went in, and reaches no gradient of a parameter."""
    rng, p, live = join_case(3, 40, 72, "f32", "f32", 4, "some")
    dh, du = rng.standard_normal((40, 72)), rng.standard_normal((40, 72))
    h2, u, saved = iodf.join(dev(p["h"]), dev(p["f"]), *params_on_gpu(p), live=on_gpu(live))
    clean = iodf.join_backward(saved, dev(dh), dev(du), *params_on_gpu(p), live=on_gpu(live))
    dh[~live], du[~live] = np.nan, np.inf
    dirty = iodf.join_backward(saved, dev(dh), dev(du), *params_on_gpu(p), live=on_gpu(live))
    assert np.isnan(host(dirty.dh)[~live]).all() and not host(dirty.df)[~live].any()
    assert np.array_equal(host(dirty.dh)[live], host(clean.dh)[live]) and np.array_equal(host(dirty.df), host(clean.df))
    for a, b in zip(clean[2:], dirty[2:]):
        assert torch().equal(a, b)


def test_join_backward_is_the_forward_s_slope():
    """Against differences of the forward form. Rows are chosen whose normalised values the checkpoint holds exactly, so that nothing but
    the formula is compared: for codes v with mean(v^2) < 1, f = v / r with r = sqrt((1 - mean(v^2)) / eps) has 1 / rms(f) = r."""
    rng = np.random.default_rng(11)
    rows, cols, eps = 6, 40, 0.25
    x, n = (np.rint(20 * rng.standard_normal((rows, cols))).clip(-60, 60) / 64 for _ in range(2))
    iq, ip = (np.sqrt((1 - (v * v).mean(1)) / eps) for v in (x, n))
    p = dict(alpha=np.float32([0.5]), gate=rng.random((2, cols)).astype(np.float32), w_post=rng.standard_normal(cols).astype(np.float32),
             w_pre=rng.standard_normal(cols).astype(np.float32))
    f = n / ip[:, None]
    h = x / iq[:, None] - p["alpha"] * ref.per_row(p["gate"], rows, cols) * p["w_post"] * n
    dh, du = (rng.standard_normal((rows, cols)).astype(np.float32) for _ in range(2))

    def loss(**q):
        r = ref.join(live=None, eps=eps, **q)
        return (dh * r["h"]).sum() + (du * r["u"]).sum()

    codes = [iodf.Codes(torch().from_numpy(q).cuda(), torch().from_numpy(e).cuda(), cols) for q, e in map(ref.encode, (x, n))]
    assert np.array_equal(ref.decode(*ref.encode(x), cols), x)
    g = iodf.join_backward(iodf.JoinSaved(*codes, dev(iq), dev(ip)), dev(dh), dev(du), *params_on_gpu(p))
    at = dict(h=h, f=f, **{k: v.astype(np.float64) for k, v in p.items()})
    for name, got in zip(("h", "f", "alpha", "gate", "w_post", "w_pre"), g):
        got = host(got)
        for _ in range(12):
            k = tuple(rng.integers(0, s) for s in at[name].shape)
            up, down = np.array(at[name]), np.array(at[name])
            up[k] += 1e-5
            down[k] -= 1e-5
            slope = (loss(**dict(at, **{name: up})) - loss(**dict(at, **{name: down}))) / 2e-5
            assert abs(slope - got[k]) < 1e-4 * max(1.0, np.abs(got).max()), (name, k)


# ---- gated activation ----

GLUS = [(1, 1, "f32"), (2, 31, "bf16"), (37, 520, "f16"), (130, 72, "bf16"), (9, 1365, "f32"), (3, 4097, "bf16"), (1, 65536, "bf16"), (600, 8, "f32"),
        (0, 16, "bf16")]


@pytest.mark.parametrize("rows,cols,name", GLUS)
@pytest.mark.parametrize("kind", ["relu", "silu", "gelu"])
@pytest.mark.parametrize("mode", ["all", "some"])
def test_glu(rows, cols, name, kind, mode):
    rng = np.random.default_rng(rows + cols)
    live = some_live(rng, rows, mode)
    alive = np.ones(rows, bool) if live is None else live
    ab = as_type(2 * spread(rng, rows, 2 * cols), name)
    ab[~alive] = np.nan
    g = dev(ab, name)
    y, saved = iodf.glu(g[:, :cols], g[:, cols:], kind, live=on_gpu(live))
    a, b = (np.where(alive[:, None], v, 0) for v in (ab[:, :cols], ab[:, cols:]))
    near(y, ref.act(a, kind)[0] * b, name, SLACK * U * np.abs(a * b), "y")
    for c, v in ((saved.a, a), (saved.b, b)):
        q, e = ref.encode(v)
        assert np.array_equal(c.q.cpu().numpy(), q) and np.array_equal(c.e.cpu().numpy(), e)
    y2, none = iodf.glu(g[:, :cols], g[:, cols:], kind, live=on_gpu(live), save=False)
    assert none is None and torch().equal(y, y2)
    dy = as_type(spread(rng, rows, cols), name)
    dy[~alive] = np.inf
    da, db, yc = iodf.glu_backward(saved, dev(dy, name), kind, live=on_gpu(live))
    a, b = (ref.decode(*ref.encode(v), cols) for v in (a, b))
    d = np.where(alive[:, None], dy, 0)
    f, slope = ref.act(a, kind)
    near(da, d * b * slope, name, SLACK * U * np.abs(d * b) * (1 + np.abs(a)), "da")
    near(db, d * f, name, SLACK * U * np.abs(d) * np.abs(a), "db")
    codes_near(yc, f * b, "y")
    assert iodf.glu_backward(saved, dev(dy, name), kind, live=on_gpu(live), rebuild=False)[2] is None


def test_activations_far_out():
    """Where exp overflows or vanishes: the activations' limits, and their slopes'."""
    v = np.float32([-1e30, -3e4, -200, -90, -30, 0, 30, 90, 200, 3e4, 1e30] * 3)[None]
    x, one = torch().from_numpy(v).cuda(), torch().ones((1, 33), device="cuda")
    for kind in ("relu", "silu", "gelu"):
        y, _ = iodf.glu(x, one, kind)
        with np.errstate(all="ignore"):
            want = np.where(v > 60, v, np.where(v < -190, 0, ref.act(np.clip(v, -190, 190).astype(np.float64), kind)[0]))
        near(y, want, "f32", 1e-6 * np.minimum(np.abs(v), 1), kind)
        c = iodf.pack(x)
        back = ref.decode(c.q.cpu().numpy(), c.e.cpu().numpy(), 33)
        da, db, _ = iodf.glu_backward(iodf.GluSaved(c, iodf.pack(one)), one, kind)
        near(da, (back > 0) + 0.0 * back if kind == "relu" else np.where(back == 0, 0.5, back > 0), "f32", 1e-6, kind + " slope")


# ---- weight gradient ----

WGRADS = [(1, 1, 1, "f32"), (1, 64, 64, "bf16"), (31, 33, 65, "bf16"), (1000, 72, 130, "bf16"), (129, 100, 7, "f16"), (257, 130, 129, "f32"),
          (2048, 128, 128, "bf16"), (5000, 40, 24, "bf16"), (5000, 40, 24, "f32"), (4099, 512, 264, "bf16"), (70000, 16, 16, "bf16"),
          (300, 1000, 520, "bf16"), (4100, 300, 1030, "f16"), (2100, 2056, 2051, "bf16"), (1025, 2048, 2048, "bf16"), (0, 40, 24, "bf16"),
          (3000, 1030, 1100, "f32")]


def wgrad_case(rows, cols, out, name, mode):
    rng = np.random.default_rng(rows + cols + out)
    live = some_live(rng, rows, mode)
    alive = np.ones(rows, bool) if live is None else live
    x, dy = spread(rng, rows, cols), as_type(rng.standard_normal((rows, out)) + 0.2, name)
    x[~alive] = 0
    dy[~alive] = np.nan
    q, e = ref.encode(x)
    codes = iodf.Codes(torch().from_numpy(q).cuda(), torch().from_numpy(e).cuda(), cols)
    return rng, codes, ref.decode(q, e, cols), dy, np.where(alive[:, None], dy, 0), live


@pytest.mark.parametrize("rows,cols,out,name", WGRADS)
@pytest.mark.parametrize("mode", ["all", "some"])
def test_weight_grad(rows, cols, out, name, mode):
    rng, codes, x, dy, d0, live = wgrad_case(rows, cols, out, name, mode)
    scale = (1 + 0.2 * rng.standard_normal(cols)).astype(np.float32)
    want = d0.T @ x
    # products are exact; the sum runs over the rows of a slice, sixteen at a time, at least, and may round at each step
    slack = (rows / 8 + SLACK) * U * (np.abs(d0).T @ np.abs(x))
    d = dev(dy, name)
    near(iodf.weight_grad(codes, d, live=on_gpu(live)), want, "f32", slack, "dw")
    before = rng.standard_normal((out, cols)).astype(np.float32)
    wide = torch().zeros((out, cols + 3), device="cuda")
    wide[:, :cols] = torch().from_numpy(before).cuda()
    got = iodf.weight_grad(codes, d, col_scale=dev(scale), live=on_gpu(live), out=wide[:, :cols], accumulate=True)
    near(got, before + scale * want, "f32", slack * np.abs(scale) + 4 * U * (np.abs(before) + np.abs(scale * want)), "dw, scaled and added")
    assert not wide[:, cols:].any()
    again = iodf.weight_grad(codes, d, col_scale=dev(scale), live=on_gpu(live))
    assert torch().equal(again, iodf.weight_grad(codes, d, col_scale=dev(scale), live=on_gpu(live)))


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_weight_grad_takes_strided_rows_at_any_element(name):
    rng, codes, x, dy, d0, live = wgrad_case(700, 264, 300, name, "all")
    d = dev(dy, name)
    for first, last in ((0, 256), (1, 258), (4, 300), (7, 8)):
        want = d0[:, first:last].T @ x
        near(iodf.weight_grad(codes, d[:, first:last]), want, "f32", (700 / 8 + SLACK) * U * (np.abs(d0[:, first:last]).T @ np.abs(x)), "dw")


def test_weight_grad_of_32_bits_loses_no_bit_of_dy():
    """One row: dw = dy x, to the bit, for values that need all 24 bits of dy (times a power of two)."""
    rng = np.random.default_rng(9)
    dy = rng.standard_normal((1, 70)).astype(np.float32)
    x = np.exp2(rng.integers(-3, 3, (1, 40))).astype(np.float64)
    q, e = ref.encode(x)
    x = ref.decode(q, e, 40)
    got = iodf.weight_grad(iodf.Codes(torch().from_numpy(q).cuda(), torch().from_numpy(e).cuda(), 40), torch().from_numpy(dy).cuda())
    assert np.array_equal(host(got), dy.astype(np.float64).T @ x)


@pytest.mark.parametrize("rows,cols,out", [(40001, 520, 1031), (33000, 1000, 257), (16384, 2048, 2048), (131073, 264, 392), (20000, 4095, 520),
                                           (9001, 2050, 2100)])
@pytest.mark.parametrize("mode", ["all", "some"])
def test_weight_grad_of_large_layers(rows, cols, out, mode):
    """Against a 64-bit product on the GPU: many rows, sides that are multiples of nothing, padding, a scale, added to what is there."""
    t = torch()
    gen = t.Generator("cuda").manual_seed(rows)
    live = t.rand(rows, generator=gen, device="cuda") < 0.8 if mode == "some" else None
    x = t.randn((rows, cols), generator=gen, device="cuda")
    d = (t.randn((rows, out), generator=gen, device="cuda") + 0.1).bfloat16()
    scale, before = (t.randn(n, generator=gen, device="cuda") for n in ((cols,), (out, cols)))
    d0 = d.double()
    if live is not None:
        d0[~live] = 0
        d[~live] = float("nan")
    codes = iodf.pack(x, live=live)
    v = iodf.unpack(codes).double()
    got = iodf.weight_grad(codes, d, col_scale=scale, live=live, out=before.clone(), accumulate=True).double()
    want = before.double() + scale.double() * (d0.t().contiguous() @ v)
    mass = before.double().abs() + scale.double().abs() * (d0.abs().t().contiguous() @ v.abs())
    # the sum of a slice takes sixteen rows at a time and may round at each step, slices are added in runs of a few
    assert ((got - want).abs() <= (min(rows, 1 << 14) / 16 + SLACK) * U * mass).all()


@pytest.mark.parametrize("rows,cols,out,name", [(40960, 512, 512, "bf16"), (8192, 1024, 1024, "bf16"), (30000, 136, 264, "bf16"), (20000, 64, 200, "f16")])
def test_weight_grad_of_operands_that_come_late(rows, cols, out, name):
    """Operands that other data has driven out of every cache, call after call without a wait between, against operands that a call has
    just read: the same bits, whatever the order in which loads land."""
    t = torch()
    gen = t.Generator("cuda").manual_seed(5)
    sets = []
    for _ in range(3):
        x = t.randn((rows, cols), generator=gen, device="cuda")
        d = t.randn((rows, out), generator=gen, device="cuda").to(dtype(name))
        codes = iodf.pack(x)
        want = iodf.weight_grad(codes, d)
        t.cuda.synchronize()
        want = iodf.weight_grad(codes, d)
        exact = t.matmul(d.double().t(), iodf.unpack(codes).double())
        assert (want.double() - exact).norm() <= 1e-5 * exact.norm()
        sets.append((codes, d, want))
    other = t.empty(1 << 29, dtype=t.uint8, device="cuda")   # twice the largest cache
    for _ in range(6):
        other.add_(1)
        got = [iodf.weight_grad(codes, d) for codes, d, _ in sets]
        for g, (_, _, want) in zip(got, sets):
            assert t.equal(g, want)


def test_weight_grad_spreads_an_infinity_no_further_than_its_column():
    rng, codes, x, dy, d0, _ = wgrad_case(100, 64, 40, "f32", "all")
    dy[17, 5] = np.inf
    got = host(iodf.weight_grad(codes, dev(dy)))
    keep = np.arange(40) != 5
    assert np.isfinite(got[keep]).all() and not np.isfinite(got[5]).any()


# ---- on the machine ----

def test_other_streams_and_graphs():
    """On a stream of the caller's, and captured into a graph: every replay gives what the eager calls gave."""
    t = torch()
    rng, p, live = join_case(4, 300, 264, "f32", "bf16", 1, "some")
    h, f, lv, par = dev(p["h"]), dev(p["f"], "bf16"), on_gpu(live), params_on_gpu(p)
    dy = dev(rng.standard_normal((300, 136)), "bf16")

    def all_of_it():
        h2, u, saved = iodf.join(h, f, *par, live=lv)
        g = iodf.join_backward(saved, h2, u, *par, live=lv)
        y, sv = iodf.glu(u, g.df, "silu", live=lv)
        da, db, yc = iodf.glu_backward(sv, y, "silu", live=lv)
        return [h2, u, *g, y, da, db, iodf.weight_grad(saved.x, dy, col_scale=par[3], live=lv), iodf.weight_grad(yc, dy, live=lv),
                iodf.unpack(iodf.pack(h, live=lv))]

    want = [x.clone() for x in all_of_it()]
    s = t.cuda.Stream()
    s.wait_stream(t.cuda.current_stream())
    with t.cuda.stream(s):
        side = all_of_it()
    s.synchronize()
    assert all(t.equal(a, b) for a, b in zip(want, side))
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        held = all_of_it()
    for _ in range(3):
        for x in held:
            x.zero_()
        graph.replay()
        t.cuda.synchronize()
        assert all(t.equal(a, b) for a, b in zip(want, held))
        all_of_it()


def test_offsets_past_32_bits():
    """More than 2^31 elements: the last rows are where they belong."""
    t = torch()
    rows, cols = (1 << 19) + 5, 4096
    x = t.zeros((rows, cols), dtype=t.bfloat16, device="cuda")
    x[-3:] = t.randn((3, cols), device="cuda", generator=t.Generator("cuda").manual_seed(1)).bfloat16()
    c = iodf.pack(x)
    q, e = ref.encode(host(x[-3:]))
    assert np.array_equal(c.q[-3:].cpu().numpy(), q) and np.array_equal(c.e[-3:].cpu().numpy(), e) and not c.q[:-3].any()
    assert t.equal(iodf.unpack(c)[-3:], t.from_numpy(ref.decode(q, e, cols)).cuda().bfloat16())
    small = iodf.pack(t.ones((rows, 8), device="cuda"))
    got = host(iodf.weight_grad(small, x))
    want = host(x[-3:]).sum(0)
    assert np.abs(got - want[:, None]).max() < 1e-5
    del c
    h, u, saved = iodf.join(x, x, w_post=t.ones(cols, device="cuda"), w_pre=t.ones(cols, device="cuda"))
    h1, u1, s1 = iodf.join(x[-3:].clone(), x[-3:].clone(), w_post=t.ones(cols, device="cuda"), w_pre=t.ones(cols, device="cuda"))
    assert t.equal(h[-3:], h1) and t.equal(u[-3:], u1) and t.equal(saved.x.q[-3:], s1.x.q) and t.equal(saved.n.e[-3:], s1.n.e)


def test_refusals_on_the_gpu():
    t = torch()
    x = t.zeros((6, 64), device="cuda")
    c = iodf.pack(x)
    v, bad = t.ones(64, device="cuda"), t.ones(63, device="cuda")
    for call in (lambda: iodf.pack(x.t()), lambda: iodf.pack(x.double()), lambda: iodf.pack(x[0]), lambda: iodf.pack(x[:1].expand(6, 64)),
                 lambda: iodf.pack(x, live=t.ones(5, dtype=t.bool, device="cuda")), lambda: iodf.pack(x, live=t.ones(6, device="cuda")),
                 lambda: iodf.pack(x, live=t.ones(6, dtype=t.bool)), lambda: iodf.unpack(c, t.float16),
                 lambda: iodf.unpack(iodf.Codes(c.q, c.e, 65)), lambda: iodf.join(x, x[:5]), lambda: iodf.join(x, x, w_post=bad),
                 lambda: iodf.join(x, x, w_post=v.bfloat16()), lambda: iodf.join(x, x, alpha=v), lambda: iodf.join(x, x, gate=t.ones((4, 64), device="cuda")),
                 lambda: iodf.join(x, x, h_out=x.bfloat16()), lambda: iodf.join(x, x, w_post=v.cpu()),
                 lambda: iodf.join_backward(iodf.JoinSaved(None, c, None, None), x, None, w_post=v),
                 lambda: iodf.join_backward(iodf.JoinSaved(c, c, None, None), x, x), lambda: iodf.glu(x, x, "tanh"), lambda: iodf.glu(x, x.bfloat16()),
                 lambda: iodf.glu_backward(iodf.GluSaved(c, c), x[:, :32]), lambda: iodf.weight_grad(c, x[:5]),
                 lambda: iodf.weight_grad(c, x, col_scale=bad), lambda: iodf.weight_grad(c, x, accumulate=True),
                 lambda: iodf.weight_grad(c, x, out=t.zeros((64, 63), device="cuda"))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: iodf.join(x.bfloat16(), x), lambda: iodf.join(x.half(), x.bfloat16()), lambda: iodf.join(x, x, eps=0.0),
                 lambda: iodf.join(t.zeros((1, 16385), device="cuda"), t.zeros((1, 16385), device="cuda"))):
        with pytest.raises(iodf.IodfError) as e:
            call()
        assert e.value.code == -1


@pytest.mark.parametrize("rows,cols,stream,block", [(37, 40, "f32", "bf16"), (20, 77, "bf16", "bf16"), (9, 1111, "f32", "f32"), (7, 600, "f16", "f16"),
                                                   (5, 8205, "f32", "f16")])
def test_join_and_glu_take_strided_rows_at_any_element(rows, cols, stream, block):
    """The columns of wider tensors, from an odd element on and up to the last one: the same bits as from tensors of their own, and what lies
    around an output stays."""
    t = torch()
    gen = t.Generator("cuda").manual_seed(cols)

    def apart(x, odd):
        wide = t.full((rows, cols + odd + 3), 7.0, dtype=x.dtype, device="cuda")
        part = wide.flatten()[odd + 3:].as_strided((rows, cols), (cols + odd + 3, 1), odd + 3)
        part.copy_(x)
        return wide, part

    def normal(name):
        return t.randn((rows, cols), generator=gen, device="cuda").to(dtype(name))

    def same(got, want):
        assert len(got) == len(want)
        for a, b in zip(got, want):
            assert t.equal(a, b)

    h, f, dh, du = normal(stream), normal(block), normal(stream), normal(block)
    par = [t.randn(n, generator=gen, device="cuda") for n in (1, cols, cols, cols)]
    h2, u, saved = iodf.join(h, f, *par)
    wide, out = apart(t.zeros_like(h), 8)
    g2, v, kept = iodf.join(apart(h, 0)[1], apart(f, 2)[1], *par, h_out=out)
    assert g2 is out and (wide[:, :11] == 7.0).all()
    same((out, v, *kept.x[:2], *kept.n[:2], kept.inv_pre, kept.inv_post), (h2, u, *saved.x[:2], *saved.n[:2], saved.inv_pre, saved.inv_post))
    same(iodf.join_backward(saved, apart(dh, 4)[1], apart(du, 6)[1], *par), iodf.join_backward(saved, dh, du, *par))
    y, gated = iodf.glu(f, du)
    z, kept = iodf.glu(apart(f, 2)[1], apart(du, 5)[1])
    same((z, *kept.a[:2], *kept.b[:2]), (y, *gated.a[:2], *gated.b[:2]))
    da, db, codes = iodf.glu_backward(gated, f)
    ea, eb, others = iodf.glu_backward(gated, apart(f, 3)[1])
    same((ea, eb, *others[:2]), (da, db, *codes[:2]))


# ---- as they are used together ----

def test_differentiable_calls():
    """One block, norms around it: gradients of the differentiable calls against autograd's own through plain 64-bit operations, as far as eight
    bits let them agree: a code is off by at most half a step, 1/128 of its group's largest value, at random, so gradients by about one percent."""
    t = torch()
    gen = t.Generator("cuda").manual_seed(7)
    rows, cols, hid = 600, 96, 160

    def leaf(*shape, by=1.0, plus=0.0):
        return (by * t.randn(shape, generator=gen, device="cuda") + plus).requires_grad_()

    h, f, w1, w2 = leaf(rows, cols), leaf(rows, cols), leaf(2 * hid, cols, by=0.1), leaf(cols, hid, by=0.1)
    par = [leaf(1, plus=0.5, by=0.0), leaf(cols, by=0.1, plus=0.7), leaf(cols, by=0.1, plus=1.0), leaf(cols, by=0.1, plus=1.0)]
    dy = t.randn((rows, cols), generator=gen, device="cuda")
    leaves = [h, f, w1, w2, *par]
    h2, u, codes = iodf.joined(h, f, *par)
    out = iodf.gated_projection(iodf.projection(u, w1, codes, col_scale=par[3].detach()), w2, "silu")
    got = t.autograd.grad((out * dy).sum() + (h2 * dy).sum(), leaves)
    wide = [x.detach().double().requires_grad_() for x in leaves]
    h, f, w1, w2, alpha, gate, w_post, w_pre = wide
    n = f * t.rsqrt((f * f).mean(1, keepdim=True) + 1e-6)
    z = h + alpha * gate * w_post * n
    x = z * t.rsqrt((z * z).mean(1, keepdim=True) + 1e-6)
    a, b = ((x * w_pre) @ w1.t()).chunk(2, 1)
    want = t.autograd.grad((((t.sigmoid(a) * a * b) @ w2.t()) * dy).sum() + (z * dy).sum(), wide)
    for g, w in zip(got, want):
        assert (g.double() - w).norm() <= 0.03 * w.norm()


def test_differentiable_calls_refuse_changed_parameters_and_second_derivatives():
    """The backward pass reads the parameters again, so a change in place between the passes is an error, as for torch's own operations; the
    gradients have no gradients of their own."""
    t = torch()
    gen = t.Generator("cuda").manual_seed(8)
    h, f, w = (t.randn(s, generator=gen, device="cuda").requires_grad_() for s in ((40, 32), (40, 32), (48, 32)))
    w_pre, w_out = t.ones(32, device="cuda", requires_grad=True), t.randn((32, 24), generator=gen, device="cuda").requires_grad_()

    def run():
        _, u, codes = iodf.joined(h, f, w_pre=w_pre)
        return iodf.gated_projection(iodf.projection(u, w, codes, col_scale=w_pre.detach()), w_out).square().sum()

    for changed in (w_pre, w, w_out):
        out = run()
        with t.no_grad():
            changed.mul_(2.0)
        with pytest.raises(RuntimeError, match="inplace"):
            out.backward()
    g, = t.autograd.grad(run(), f, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        g.sum().backward()


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_activations_keep_their_precision_in_the_tail(kind):
    """Where the logistic function is small, relative to the result itself: exp, a sum, a reciprocal and two products come to ten units of 2^-24 or
    so, a few more are allowed; gelu's argument 2 sqrt(2 / pi) (a + 0.044715 a^3) is rounded six times on its way (constants among them), half a unit
    of its last bit each, and exp turns that into as many units times the argument. A slope cancels near its zero: it is held to its terms."""
    a = np.linspace(-85, 85, 20001) if kind == "silu" else np.linspace(-7.6, 7.6, 20001)  # the argument within +-85
    a = a.astype(np.float32).reshape(-1, 1)
    x, one = dev(a), dev(np.ones_like(a))
    a = a.astype(np.float64)
    arg = np.abs(a if kind == "silu" else 2 * np.sqrt(2 / np.pi) * (a + 0.044715 * a ** 3))
    units = (16 + (0 if kind == "silu" else 6 * arg)) * U
    sig = 1 / (1 + np.exp(-(a if kind == "silu" else 2 * np.sqrt(2 / np.pi) * (a + 0.044715 * a ** 3))))
    y, _ = iodf.glu(x, one, kind)
    near(y, a * sig, "f32", units * np.abs(a * sig), kind)
    c = iodf.pack(x)
    v = ref.decode(c.q.cpu().numpy(), c.e.cpu().numpy(), 1)   # one number to a group: seven bits of it
    inner = v if kind == "silu" else 2 * np.sqrt(2 / np.pi) * (v + 0.044715 * v ** 3)
    grow = np.ones_like(v) if kind == "silu" else 2 * np.sqrt(2 / np.pi) * (1 + 3 * 0.044715 * v * v)
    up, down = 1 / (1 + np.exp(-inner)), 1 / (1 + np.exp(inner))
    units = (24 + (0 if kind == "silu" else 6 * np.abs(inner))) * U
    da, db, _ = iodf.glu_backward(iodf.GluSaved(c, iodf.pack(one)), one, kind)
    near(db, v * up, "f32", units * np.abs(v * up), kind + " again")
    # 1 - s is taken from s in 32 bits: where s is near 1 its own units count, not those of the small rest
    near(da, up + v * up * down * grow, "f32", units * (up + np.abs(v) * up * np.maximum(down, U) * grow) + 2 * U * np.abs(v) * grow * up * up, kind + " slope")


def test_weight_grad_of_the_largest_numbers_in_32_bits():
    """Up to the type's last number, which bfloat16 rounds to infinity: one row, to the bit. Infinities and NaN of any payload come out as such."""
    t = torch()
    top = np.finfo(np.float32).max
    dy = np.float32([[top, -top, np.nextafter(np.float32(3.3961775e38), top), 3.3895314e38, 1.0000001, 2.0 ** -100, 0, np.inf, -np.inf, 0]])
    dy.view(np.uint32)[0, 9] = 0x7f800001   # a NaN whose payload is in the lower half alone
    x = np.float64([[0.25, 0.5, 2.0 ** -20]])
    q, e = ref.encode(x)
    codes = iodf.Codes(t.from_numpy(q).cuda(), t.from_numpy(e).cuda(), 3)
    got = host(iodf.weight_grad(codes, t.from_numpy(dy).cuda()))
    x = ref.decode(q, e, 3)[:, :2]
    assert np.array_equal(got[:9, :2], dy[:, :9].astype(np.float64).T @ x) and np.isnan(got[9, :2]).all()


def test_what_is_no_tensor_or_was_not_saved_is_refused():
    t = torch()
    x = t.zeros((6, 64), device="cuda")
    c = iodf.pack(x)
    for call in (lambda: iodf.join(x, x, gate=0.5), lambda: iodf.join(x, x, gate=x[0, 0]), lambda: iodf.join(x, x, gate=x[None]),
                 lambda: iodf.join_backward(iodf.join(x, x, save=False)[2], x, None), lambda: iodf.join_backward((c, c, None, None), x, None),
                 lambda: iodf.join_backward(iodf.JoinSaved(None, c, None, None), x, None, block_dtype=t.float64),
                 lambda: iodf.join_backward(iodf.JoinSaved(c, c, x[:, 0].contiguous(), None), x, 1.0, w_pre=x[0]),
                 lambda: iodf.glu_backward(iodf.glu(x, x, save=False)[1], x), lambda: iodf.unpack(iodf.Codes(None, None, 64)),
                 lambda: iodf.unpack(iodf.Codes(c.q, None, 64)), lambda: iodf.weight_grad(iodf.Codes(None, c.e, 64), x),
                 lambda: iodf.unpack(iodf.Codes(c.q[0], c.e[0], 64))):
        with pytest.raises(ValueError, match="iodf"):
            call()


def test_the_binding_s_plain_entries_give_the_same_bits():
    """The C names with addresses and argument blocks, as a caller without torch's operators has them, on a stream of the caller's."""
    t = torch()
    rows, cols, out = 300, 200, 136
    rng, p, live = join_case(6, rows, cols, "f32", "bf16", 3, "some")
    h, f, lv = dev(p["h"]), dev(p["f"], "bf16"), on_gpu(live)
    alpha, gate, w_post, w_pre = par = params_on_gpu(p)
    dy, du, pitch = dev(rng.standard_normal((rows, out)), "bf16"), dev(rng.standard_normal((rows, cols)), "bf16"), 224
    h2, u, saved = iodf.join(h, f, *par, live=lv, eps=1e-5)
    grads = iodf.join_backward(saved, h, du, *par, live=lv)
    y, gated = iodf.glu(f, du, "gelu", live=lv)
    da, db, yc = iodf.glu_backward(gated, f, "gelu", live=lv)
    dw = iodf.weight_grad(saved.x, dy, col_scale=w_pre, live=lv)
    back = iodf.unpack(saved.x)
    st = t.cuda.Stream()
    st.wait_stream(t.cuda.current_stream())

    def codes():
        return iodf.Codes(t.full((rows, pitch), 99, dtype=t.int8, device="cuda"), t.full((rows, pitch // 32), 99, dtype=t.uint8, device="cuda"), cols)

    def at(**tensors):
        return {k: v.data_ptr() for k, v in tensors.items()}

    def same(got, want):
        for a, b in zip(got, want):
            assert t.equal(a, b)

    with t.cuda.stream(st):
        x, n, ipre, ipost = codes(), codes(), t.empty(rows, device="cuda"), t.empty(rows, device="cuda")
        o_h, o_u = t.empty_like(h), t.empty_like(f)
        a = iodf.JoinArgs(rows=rows, gate_rows=rows // 3, cols=cols, stream_type=iodf.IODF_T_F32, block_type=iodf.IODF_T_BF16, eps=1e-5,
                          in_stream_stride=cols, in_block_stride=cols, out_stream_stride=cols, out_block_stride=cols,
                          **at(alpha=alpha, gate=gate, w_post=w_post, w_pre=w_pre, live=lv, in_stream=h, in_block=f, out_stream=o_h, out_block=o_u,
                               xq=x.q, xe=x.e, nq=n.q, ne=n.e, inv_pre=ipre, inv_post=ipost))
        iodf.iodf_join_forward(a, st.cuda_stream)
        st.synchronize()
        same((o_h, o_u, *x[:2], *n[:2], ipre, ipost), (h2, u, *saved.x[:2], *saved.n[:2], saved.inv_pre, saved.inv_post))
        g = [t.empty_like(v) for v in (h, f, *par)]
        for name, v in at(in_block=du, out_stream=g[0], out_block=g[1], dalpha=g[2], dgate=g[3], dw_post=g[4], dw_pre=g[5]).items():
            setattr(a, name, v)
        work = t.empty(iodf.iodf_join_workspace(a), dtype=t.uint8, device="cuda")
        iodf.iodf_join_backward(a, work.data_ptr(), work.numel(), st.cuda_stream)
        st.synchronize()
        same(g, grads)
        ca, cb, cy, o_y, o_a, o_b = codes(), codes(), codes(), *(t.empty_like(f) for _ in range(3))
        a = iodf.GluArgs(rows=rows, cols=cols, type=iodf.IODF_T_BF16, act=iodf.IODF_ACT_GELU, a_stride=cols, b_stride=cols, y_stride=cols, dy_stride=cols,
                         da_stride=cols, db_stride=cols, **at(live=lv, a=f, b=du, y=o_y, dy=f, da=o_a, db=o_b, aq=ca.q, ae=ca.e, bq=cb.q, be=cb.e,
                                                              yq=cy.q, ye=cy.e))
        iodf.iodf_glu_forward(a, st.cuda_stream)
        iodf.iodf_glu_backward(a, st.cuda_stream)
        st.synchronize()
        same((o_y, *ca[:2], *cb[:2], o_a, o_b, *cy[:2]), (y, *gated.a[:2], *gated.b[:2], da, db, *yc[:2]))
        o_w = t.empty((out, cols), device="cuda")
        a = iodf.WgradArgs(rows=rows, cols=cols, out=out, dy_type=iodf.IODF_T_BF16, dy_stride=out, dw_stride=cols,
                           **at(dy=dy, q=x.q, e=x.e, col_scale=w_pre, live=lv, dw=o_w))
        work = t.empty(iodf.iodf_weight_grad_workspace(a) + 16, dtype=t.uint8, device="cuda")
        iodf.iodf_weight_grad(a, work.data_ptr(), work.numel(), st.cuda_stream)
        c, o_v = codes(), t.empty_like(f)
        iodf.iodf_pack(back.data_ptr(), iodf.IODF_T_BF16, cols, rows, cols, lv.data_ptr(), c.q.data_ptr(), c.e.data_ptr(), st.cuda_stream)
        iodf.iodf_unpack(x.q.data_ptr(), x.e.data_ptr(), rows, cols, o_v.data_ptr(), iodf.IODF_T_BF16, cols, st.cuda_stream)
        st.synchronize()
        again = iodf.pack(back, live=lv)
        same((o_w, o_v, *c[:2]), (dw, back, *again[:2]))
    for call, bad in ((iodf.iodf_weight_grad, iodf.WgradArgs(rows=-1)), (iodf.iodf_join_backward, iodf.JoinArgs(rows=-1))):
        with pytest.raises(iodf.IodfError):
            call(bad, 0, 0, 0)
    for call, bad in ((iodf.iodf_join_forward, iodf.JoinArgs(rows=-1)), (iodf.iodf_glu_forward, iodf.GluArgs(rows=-1)),
                      (iodf.iodf_glu_backward, iodf.GluArgs(rows=-1))):
        with pytest.raises(iodf.IodfError):
            call(bad, 0)
    for call, bad in ((iodf.iodf_join_workspace, iodf.JoinArgs(rows=-1)), (iodf.iodf_weight_grad_workspace, iodf.WgradArgs(rows=-1))):
        with pytest.raises(iodf.IodfError):
            call(bad)


@pytest.mark.parametrize("eps", [1e-6, 1e-30, 1.2e-38, 1e-38, 1e-40, 1.4e-45])
@pytest.mark.parametrize("cols", [5, 64, 1111])
def test_join_of_rows_of_zeros(cols, eps):
    """Whatever eps > 0 there is: zeros over sqrt(eps) are zeros, and the factors are finite."""
    t = torch()
    f, w = t.zeros((3, cols), device="cuda"), t.ones(cols, device="cuda")
    f[1] = 0.5
    h, u, saved = iodf.join(t.zeros_like(f), f, w_post=w, w_pre=w, eps=eps)
    root = np.float64(np.float32(eps)) ** -0.5
    for got in (saved.inv_post, saved.inv_pre):
        got = host(got)
        assert np.abs(got[[0, 2]] / root - 1).max() < 8 * U
    assert not host(h)[[0, 2]].any() and not host(u)[[0, 2]].any()
    near(u[1:2], np.full((1, cols), (1 + eps) ** -0.5), "f32", SLACK * U, "u")
