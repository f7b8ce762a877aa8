"""Plain 64-bit forms of the training operators, for the tests: written from the formulas in include/iodf.h, on the CPU."""
import numpy as np


def exponents(top):
    """Exponent byte of groups whose largest magnitudes are `top` (float64)."""
    top = np.asarray(top, np.float64)
    e = np.full(top.shape, 16, np.int64)
    big = top > 0
    m, k = np.frexp(top[big])                     # top = m 2^k, 0.5 <= m < 1
    e[big] = k - 1 + 127 + (np.rint(m * 128) >= 128)
    return np.clip(e, 16, 254)


def groups(v):
    rows, cols = v.shape
    pitch = -(-cols // 32) * 32
    g = np.zeros((rows, pitch))
    g[:, :cols] = v
    return g.reshape(rows, pitch // 32, 32)


def encode(v):
    """(q, e) of finite or non-finite v, exactly as the layout says."""
    g = groups(v)
    rows = g.shape[0]
    bad = ~np.isfinite(g).all(2)
    g = np.where(bad[:, :, None], 0.0, g)
    e = exponents(np.abs(g).max(2)) if g.size else np.zeros(g.shape[:2], np.int64)
    q = np.clip(np.rint(g * np.exp2(133.0 - e)[:, :, None]), -127, 127)
    e = np.where(bad, 255, e)
    return q.reshape(rows, 32 * g.shape[1]).astype(np.int8), e.astype(np.uint8)


def decode(q, e, cols):
    q, e = np.asarray(q), np.asarray(e).astype(np.int64)
    step = np.where(e == 255, np.nan, np.exp2(np.maximum(e, 7) - 133.0))
    return (q.astype(np.float64).reshape(*e.shape, 32) * step[:, :, None]).reshape(q.shape)[:, :cols]


def per_row(gate, rows, cols):
    if gate is None:
        return np.ones((rows, cols))
    gate = np.asarray(gate, np.float64).reshape(-1, cols)
    return np.repeat(gate, rows // gate.shape[0], 0) if rows else np.zeros((0, cols))


def join(h, f, alpha, gate, w_post, w_pre, live, eps):
    rows, cols = h.shape
    live = np.ones(rows, bool) if live is None else live
    f = np.where(live[:, None], f, 0.0)
    ip = (np.mean(f * f, 1) + eps) ** -0.5 if w_post is not None else np.ones(rows)
    n = f * ip[:, None]
    z = h + (1.0 if alpha is None else alpha) * per_row(gate, rows, cols) * (1.0 if w_post is None else w_post) * n
    iq = (np.mean(z * z, 1) + eps) ** -0.5
    x = np.where(live[:, None], z * iq[:, None], 0.0)
    return dict(h=z, n=n, x=x, u=None if w_pre is None else x * w_pre, inv_pre=np.where(live, iq, 0.0), inv_post=np.where(live, ip, 0.0))


def join_backward(x, n, iq, ip, dh, du, alpha, gate, w_post, w_pre, live):
    rows, cols = dh.shape
    live = np.ones(rows, bool) if live is None else live
    al, wp = (1.0 if alpha is None else alpha), (1.0 if w_post is None else w_post)
    g = per_row(gate, rows, cols)
    dz = np.array(dh)
    r = {}
    if w_pre is not None:
        du = np.where(live[:, None], du, 0.0)
        dx = du * w_pre
        dz = dz + np.where(live[:, None], iq[:, None] * (dx - x * np.mean(dx * x, 1, keepdims=True)), 0.0)
        r["dw_pre"] = (du * x).sum(0)
    alive = np.where(live[:, None], dz, 0.0)
    dn = al * g * wp * alive
    r["dh"] = dz
    r["df"] = ip[:, None] * (dn - n * np.mean(dn * n, 1, keepdims=True)) if w_post is not None else dn
    share = alive * n
    if alpha is not None:
        r["dalpha"] = (g * wp * share).sum().reshape(1)
    if w_post is not None:
        r["dw_post"] = (al * g * share).sum(0)
    if gate is not None:
        k = np.asarray(gate).reshape(-1, cols).shape[0]
        r["dgate"] = (al * wp * share.reshape(k, -1, cols).sum(1)).reshape(np.asarray(gate).shape)
    return r


def act(a, kind):
    """act(a) and its slope."""
    with np.errstate(over="ignore"):
        if kind == "relu":
            return np.maximum(a, 0), (a > 0).astype(np.float64)
        if kind == "silu":
            s = 1 / (1 + np.exp(-a))
            return a * s, s + a * s * (1 - s)
    c = np.sqrt(2 / np.pi)
    th = np.tanh(c * (a + 0.044715 * a ** 3))
    return 0.5 * a * (1 + th), 0.5 * (1 + th) + 0.5 * a * (1 - th * th) * c * (1 + 3 * 0.044715 * a * a)
