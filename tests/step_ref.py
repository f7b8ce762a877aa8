"""Plain 64-bit forms of the loss over a table of classes and of orthogonalised updates, for the tests: written from the formulas in include/iodf.h, on the
CPU, with what their roundings may amount to."""
import numpy as np

U = 2.0 ** -24
QUINTIC = (3.4445, -4.7750, 2.0315)
# Half a step, relative: of the 16-bit number that the gradient of a logit is rounded to (8 and 11 significant bits: the numbers behind 1 are 2^-7 and 2^-10
# away), and of two parts of 11 bits.
HALF = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -22}


def loss(u, w, target, live=None):
    """loss, lse, logits."""
    live = np.ones(len(u), bool) if live is None else live
    u = np.where(live[:, None], u, 0.0)
    s = u @ w.T
    top = s.max(1, keepdims=True)
    lse = (top + np.log(np.exp(s - top).sum(1, keepdims=True)))[:, 0]
    at = np.where(live, target, 0)
    return np.where(live, lse - s[np.arange(len(u)), at], 0.0), np.where(live, lse, 0.0), s


def logit_slack(u, w, live=None):
    """What a logit's sum may be off by, of each row: 64 roundings of the terms' magnitudes."""
    u = np.where(live[:, None], u, 0.0) if live is not None else u
    return 64 * U * (np.abs(u) @ np.abs(w).T).max(1) + 1e-37


def loss_backward(u, w, target, lse, dloss, dlse, live, name):
    """du, dw and what each may be off by besides its own rounding: of g the logit's error, 16 roundings of 32 bits and the half step it is stored with (in half
    precision and in two parts no finer than 2^-38 of the largest); 64 roundings of the sums."""
    rows, classes = len(u), len(w)
    live = np.ones(rows, bool) if live is None else live
    u = np.where(live[:, None], u, 0.0)
    up = np.where(live, 0.0 if dloss is None else dloss, 0.0)
    both = up + np.where(live, 0.0 if dlse is None else dlse, 0.0)
    s = u @ w.T
    p = np.exp(s - np.where(live, lse, 0.0)[:, None]) * both[:, None]
    g = p.copy()
    g[np.arange(rows), np.where(live, target, 0)] -= up
    off = np.abs(p) * (logit_slack(u, w)[:, None] + 16 * U * (1 + np.abs(s))) + np.abs(g) * HALF[name]
    if name != "bf16":
        off += 2.0 ** -38 * max(np.abs(up).max(initial=0.0), np.abs(both).max(initial=0.0)) * live[:, None]
    a, b = np.abs(u), np.abs(w)
    tiny = 2.0 ** -38 * (b.max(initial=0.0) if name == "f32" else 0.0), 2.0 ** -38 * (a.max(initial=0.0) if name == "f32" else 0.0)
    more = 64 * U * np.abs(g) + off
    return (g @ w, g.T @ u, more @ b + np.abs(g).sum(1, keepdims=True) * tiny[0], more.T @ a + np.abs(g).sum(0)[:, None] * tiny[1])


def gradients_by_the_parts(u, w, target, lse, dloss, dlse, live, step, least=0.0):
    """du, dw and what each may be off by besides its own rounding, where the numbers multiplied are exact but for g: that is stored with `step` of itself, or of
    `least` in its place. Nothing here goes by a tensor's largest number: a row or class does not see how large the others are."""
    rows, classes = len(u), len(w)
    live = np.ones(rows, bool) if live is None else live
    u = np.where(live[:, None], u, 0.0)
    up = np.where(live, 0.0 if dloss is None else dloss, 0.0)
    both = up + np.where(live, 0.0 if dlse is None else dlse, 0.0)
    s = u @ w.T
    p = np.exp(s - np.where(live, lse, 0.0)[:, None]) * both[:, None]
    g = p.copy()
    g[np.arange(rows), np.where(live, target, 0)] -= up
    a, b = np.abs(u), np.abs(w)
    off = np.abs(p) * (64 * U * (a @ b.T) + 16 * U * (1 + np.abs(s))) + np.abs(g) * (step + 64 * U) + least * live[:, None]
    return g @ w, g.T @ u, off @ b, off.T @ a


def steps_of(steps, coefficients):
    return [coefficients] * steps if np.isscalar(coefficients[0]) else list(coefficients)


def half(x, lift):
    """x in half precision times a power of two, as float64."""
    return np.float16(np.float32(x * lift)).astype(np.float64) / lift


def exactly(x, y):
    return x @ y


def of_halves(x, y):
    """A product of numbers rounded to half precision."""
    return half(x, 2.0 ** 12) @ half(y, 2.0 ** 12)


def of_two_halves(x, y):
    """A product of numbers in two parts of half precision: high high, high low and low high. The fourth product is left out: up to 2^-22 of each term."""
    xh, yh = half(x, 2.0 ** 12), half(y, 2.0 ** 12)
    return xh @ yh + xh @ half(y - yh, 2.0 ** 12) + half(x - xh, 2.0 ** 12) @ yh


def polynomial_steps(g, steps, coefficients, eps, product, stored, sums):
    """X <- a X + (b A + c A^2) X on the shorter side. product: of matrices as they are multiplied; stored: what a number is kept as between the products;
    sums: what a sum of products is kept as. Diagonals of A and of b A + c A^2 are sums."""
    tall = g.shape[0] > g.shape[1]
    x = (g.T if tall else g).astype(np.float64)
    x = stored(sums(x / (np.linalg.norm(x) + eps)), True)
    for a, b, c in steps_of(steps, coefficients):
        m = sums(product(x, x.T))
        d = np.diag(m).copy()
        o = stored(m - np.diag(d), False)
        q = sums(b * (o + np.diag(d)) + c * ((d[:, None] + d) * o + sums(product(o, o)) + np.diag(d * d)))
        e = np.diag(q).copy()
        x = stored(sums((a + e)[:, None] * x + sums(product(stored(q - np.diag(e), False), x))), True)
    return x.T if tall else x


def orthogonalise(g, steps=5, coefficients=QUINTIC, eps=1e-7, parts=True):
    """The result in 64 bits, and what its Frobenius norm may be off by: twice what the same steps are off by with their roundings put in (other sums round
    other numbers, by as much), and some half steps of the numbers multiplied for matrices so small that roundings happen to be kind."""
    def kept(v, x):  # X is always in two parts
        hi = half(v, 2.0 ** 12)
        return hi + half(v - hi, 2.0 ** 12) if x or parts else hi

    want = polynomial_steps(g, steps, coefficients, eps, exactly, lambda v, x: v, lambda v: v)
    put = polynomial_steps(g, steps, coefficients, eps, of_two_halves if parts else of_halves, kept, lambda v: v.astype(np.float32).astype(np.float64))
    return want, 2 * np.linalg.norm(put - want) + (2.0 ** -21 if parts else 2.0 ** -11) * 4 * np.linalg.norm(want)
