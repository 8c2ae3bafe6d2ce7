"""Plain float64 reference of the operators between ids, rows and gradients:
embedding sums and a table's gradient, norms around a block and their gradients,
the norm of all gradients.  Written from the definitions in include/stca.h; numpy
only.  Beside values, the magnitudes that rounding errors are relative to.
"""
import numpy as np


def embed(tables, ids, scale):
    """(out, sum of magnitudes) [n][d]"""
    out = np.zeros((len(ids[0]), tables[0].shape[1]))
    mag = np.zeros_like(out)
    for t, i in zip(tables, ids):
        for k, v in enumerate(i):
            if 0 <= v < len(t):
                out[k] += t[v]
                mag[k] += np.abs(t[v])
    return scale * out, np.abs(scale) * mag


def embed_grad(parts, n_rows, scale):
    """(distinct ids, their gradients, magnitudes, tokens of each)"""
    ids = np.concatenate([np.asarray(i, dtype=np.int64) for i, _ in parts])
    dout = np.concatenate([np.asarray(g, dtype=np.float64) for _, g in parts])
    keep = (ids >= 0) & (ids < n_rows)
    rows, at = np.unique(ids[keep], return_inverse=True)
    out = np.zeros((len(rows), dout.shape[1]))
    mag = np.zeros_like(out)
    np.add.at(out, at, dout[keep])
    np.add.at(mag, at, np.abs(dout[keep]))
    return rows, scale * out, np.abs(scale) * mag, np.bincount(at, minlength=len(rows))


U = 2.0 ** -24  # half a step of fp32


def unit(v, kind, eps, err):
    """Unit rows, r, and a bound on the error of the unit rows where v is off by err.

    Sums over a row are trees of at most 8 + 10 additions, r is within 13 U, and a
    layer norm's differences carry 2 U of their own and 18 U of the row's
    deviation: in all at most 40 U (|u| + 1).  What v is off by moves u by r err, the
    mean and the scale."""
    c = v
    for _ in range(4 if kind == "layer" else 0):  # (a mean that is rounded is not all of it)
        c = c - c.mean(-1, keepdims=True)
    with np.errstate(over="ignore", invalid="ignore"):
        r = 1.0 / np.sqrt((c * c).mean(-1, keepdims=True) + eps)
    u = c * r
    e = r * err
    bound = e + np.abs(u) * (e * np.abs(u)).mean(-1, keepdims=True) + 40 * U * (np.abs(u) + 1)
    if kind == "layer":
        bound += e.mean(-1, keepdims=True)
    return u, r, bound


def unit_grad(a, a_err, u, u_err, r, kind):
    """Gradient of a row from a, that of its unit row, and a bound on its error (r is
    off by what u is, relative to a deviation of 1)."""
    def mean(x):
        return x.mean(-1, keepdims=True)
    m = mean(a * u)
    g = a - u * m
    mag = np.abs(a) + np.abs(u) * mean(np.abs(a * u))
    err = a_err + np.abs(u) * mean(a_err * np.abs(u) + np.abs(a) * u_err) + u_err * np.abs(m)
    if kind == "layer":
        g = g - mean(a)
        mag = mag + mean(np.abs(a))
        err = err + mean(a_err)
    r_err = mean(u_err * np.abs(u)) + 40 * U
    return r * g, r * (err + 40 * U * mag + np.abs(g) * r_err)


def affine(u, u_err, w, b, d):
    w = np.ones(d) if w is None else w
    b = np.zeros(d) if b is None else b
    return u * w + b, u_err * np.abs(w) + 2 * U * (np.abs(u * w) + np.abs(b)), w


def sum_depth(n, d):
    """Additions behind one another in a gradient of [d]: a lane's rows (of teams of
    d / 8 lanes, 256 lanes a workgroup or a team, two workgroups a CU of 256), its
    workgroup's teams, and two roundings more: the residual scale, the fp64 sum's."""
    lanes = max(8, 1 << (-(-d // 8) - 1).bit_length())
    teams = 256 // lanes if lanes <= 64 else 1
    groups = min(-(-n // teams), 512)
    return -(-n // max(1, groups * teams)) + teams + 2


def norm(x, kind, eps, scale, block=None, gate=None, act=None, pre=(None, None), post=None, ls=None, dy=None, dh=None):
    """dict of values and (name + "_err") bounds on the error before rounding."""
    out, d = {}, x.shape[1]
    h, h_err = x, np.zeros_like(x)
    if block is not None:
        n, n_err = block, np.zeros_like(block)
        if post is not None:
            uo, ro, uo_err = unit(block, kind, eps, n_err)
            n, n_err, pw = affine(uo, uo_err, *post, d)
        s, s_err, slope, slope_err = np.ones_like(x), 0.0, 0.0, 0.0
        if act:
            p = np.where(gate >= 0, 1 / (1 + np.exp(-np.abs(gate))), np.exp(-np.abs(gate)) / (1 + np.exp(-np.abs(gate))))
            rest = np.where(gate >= 0, np.exp(-np.abs(gate)) / (1 + np.exp(-np.abs(gate))), 1 / (1 + np.exp(-np.abs(gate))))
            # the exponential is off by 2 U of exp2, U of its correction and 0.05 U |g| of what that leaves (4 U
            # at the end of fp32), the small one of s and 1 - s by U of 1 + it, 2 U of the reciprocal and U of a
            # product more, of which the first is nothing at |g| > 17, and a SiLU by another product's: below 12 U.
            # An exponential below 2^-126 may be zero.
            rel = 12 * U
            none = (1 + np.abs(gate)) * 2.0 ** -126
            s = p * gate if act == "silu" else p
            slope = p + gate * p * rest if act == "silu" else p * rest
            s_err = rel * np.abs(s) + none
            slope_err = 2 * rel * (p + np.abs(gate) * p * rest if act == "silu" else p * rest) + none
        t, t_err = n * s, n_err * np.abs(s) + np.abs(n) * s_err + U * np.abs(n * s)
        k = scale * (np.ones(d) if ls is None else ls)
        h = x + k * t
        h_err = np.abs(k) * t_err + 2 * U * np.abs(k * t) + U * np.abs(h)
        out["h"], out["h_err"] = h, h_err
    if pre is not False:
        u, r, u_err = unit(h, kind, eps, h_err)
        out["y"], out["y_err"], w = affine(u, u_err, *pre, d)
    if dy is None and dh is None:
        return out
    depth = sum_depth(*x.shape) * U
    def total(name, term, err):
        out[name], out[name + "_err"] = term.sum(0), err.sum(0) + depth * np.abs(term).sum(0)
    g = np.zeros_like(x) if dh is None else dh
    g_err = np.zeros_like(x)
    if pre is not False:
        total("pre_w", dy * u, np.abs(dy) * u_err)
        total("pre_b", dy, 0 * dy)
        v, v_err = unit_grad(dy * w, U * np.abs(dy * w), u, u_err, r, kind)
        g, g_err = g + v, v_err + U * np.abs(g + v)
    out["dx"], out["dx_err"] = g, g_err
    if block is None:
        return out
    total("ls", scale * g * t, np.abs(scale) * (g_err * np.abs(t) + np.abs(g) * t_err + U * np.abs(g * t)))
    e, e_err = g * k, np.abs(k) * g_err + 2 * U * np.abs(g * k)
    if act:
        out["dgate"] = e * n * slope
        out["dgate_err"] = (e_err * np.abs(n * slope) + np.abs(e) * n_err * np.abs(slope) + np.abs(e * n) * slope_err +
                            2 * U * np.abs(e * n * slope))
    o, o_err = e * s, e_err * np.abs(s) + np.abs(e) * s_err + U * np.abs(e * s)
    if post is not None:
        total("post_w", o * uo, o_err * np.abs(uo) + np.abs(o) * uo_err)
        total("post_b", o, o_err)
        o, o_err = unit_grad(o * pw, o_err * np.abs(pw) + U * np.abs(o * pw), uo, uo_err, ro, kind)
    out["dblock"], out["dblock_err"] = o, o_err
    return out


def clip(grads, max_norm):
    """(norm, factor)"""
    norm = float(np.sqrt(np.sum([np.sum(np.square(g.astype(np.longdouble))) for g in grads])))
    return norm, (max_norm / norm if np.isfinite(norm) and norm > max_norm else 1.0)
