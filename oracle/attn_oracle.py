"""Float64 oracle of the stand-alone attention, its gradients and the 8-bit
cache, written from the definitions with numpy, one request and head at a time.
Shares no code with the HIP path.

Beside each result stands the sum of absolute values that its roundings are
relative to (the same products with every factor replaced by its magnitude), so
that a test can bound an error instead of guessing a tolerance.
"""
from __future__ import annotations

import numpy as np


def bucket(dist, edges):
    """Number of edges that are at most max(dist, 0)."""
    d = np.maximum(dist, 0)
    b = np.zeros(d.shape, dtype=np.int64)
    for e in edges:
        b += d >= e
    return b


def attention(q, k, v, hoff, toff, *, scale, cap=0.0, edges=None, bias=None, masked=False, tgt_pos=None,
              hist_pos=None, dout=None):
    """q [n_tgt][H][dh], k, v [n_hist][Hk][dh], float64.  Returns a dict: out and,
    with dout, dq, dk, dv, dbias; "<name>_abs" the magnitudes; "score" the
    largest sum of |scale q k| and "x" the largest finite score magnitude."""
    H, Hk, dh = q.shape[1], k.shape[1], q.shape[2]
    nb = 0 if edges is None else len(edges) + 1
    r = {n: np.zeros(x.shape) for n, x in (("out", q), ("dq", q), ("dk", k), ("dv", v), ("dbias", np.zeros((H, nb))))}
    r.update({n + "_abs": np.zeros(x.shape) for n, x in list(r.items())})
    r["score"] = r["x"] = 0.0
    for i in range(len(hoff) - 1):
        ts, js = slice(toff[i], toff[i + 1]), slice(hoff[i], hoff[i + 1])
        m, L = toff[i + 1] - toff[i], hoff[i + 1] - hoff[i]
        if m == 0 or L == 0:
            continue
        dist = None
        if tgt_pos is not None:
            p = np.arange(L) if hist_pos is None else hist_pos[js].astype(np.int64)
            dist = np.clip(tgt_pos[ts].astype(np.int64)[:, None] - p[None, :], -2 ** 31, 2 ** 31 - 1)
        b = bucket(dist, edges) if nb else None
        for h in range(H):
            g = h * Hk // H
            kg, vg, qh = k[js, g], v[js, g], q[ts, h]
            vis = np.ones((m, L), dtype=bool)
            if masked:
                vis &= dist >= 0
            if nb:
                vis &= bias[h][b] != -np.inf
            with np.errstate(invalid="ignore", over="ignore"):
                z = scale * (qh @ kg.T)
                th = np.tanh(z / cap) if cap else None
                x = cap * th if cap else z
                if nb:
                    x = x + np.where(vis, bias[h][b], 0.0)
            x = np.where(vis, x, -np.inf)
            some = vis.any(axis=1, keepdims=True)
            top = np.where(some, x.max(axis=1, keepdims=True), 0.0)
            with np.errstate(invalid="ignore"):
                w = np.where(vis, np.exp(x - top), 0.0)
                w = np.divide(w, w.sum(axis=1, keepdims=True), out=np.zeros_like(w), where=vis)  # (0 / NaN is not 0)
            fin = np.isfinite(x)
            if fin.any():
                r["score"] = max(r["score"], float(np.nanmax(np.where(vis, abs(scale) * (abs(qh) @ abs(kg).T), 0.0))))
                r["x"] = max(r["x"], float(np.max(np.abs(x - top)[fin], initial=0.0, where=np.abs(x - top)[fin] < 1e30)))

            def over_rows(a, b):  # a [m][L] times b [L][dh], hidden pairs left out
                if np.isfinite(b).all():
                    return a @ b
                with np.errstate(invalid="ignore"):
                    return np.stack([(a[t][vis[t], None] * b[vis[t]]).sum(0) for t in range(m)])

            def over_targets(a, b):  # a [m][L]^T times b [m][dh]
                if np.isfinite(b).all():
                    return a.T @ b
                with np.errstate(invalid="ignore"):
                    return np.stack([(a[vis[:, j], j, None] * b[vis[:, j]]).sum(0) for j in range(L)])

            o = over_rows(w, vg)
            r["out"][ts, h] = o
            r["out_abs"][ts, h] = over_rows(w, abs(vg))
            if dout is None:
                continue
            go = dout[ts, h]
            with np.errstate(invalid="ignore"):
                dp, D = go @ vg.T, (go * o).sum(axis=1, keepdims=True)
                dx = np.where(vis, w * (dp - D), 0.0)
                slope = 1 - th * th if cap else np.ones_like(dx)
                dz = np.where(vis, dx * slope, 0.0) * scale
                ax = np.where(vis, w * (abs(go) @ abs(vg).T + (abs(go) * r["out_abs"][ts, h]).sum(1, keepdims=True)), 0.0)
            r["dq"][ts, h] = over_rows(dz, kg)
            r["dk"][js, g] += over_targets(dz, qh)
            r["dv"][js, g] += over_targets(w, go)
            r["dq_abs"][ts, h] = over_rows(ax * abs(scale), abs(kg))
            r["dk_abs"][js, g] += over_targets(ax * abs(scale), abs(qh))
            r["dv_abs"][js, g] += over_targets(w, abs(go))
            if nb:
                np.add.at(r["dbias"][h], b, dx)
                np.add.at(r["dbias_abs"][h], b, ax)
    return r


def quantise(x):
    """x [..][dh] float64 -> (n int, e int [..]): step 2^(e - 127) per row."""
    top = np.abs(x).max(axis=-1)
    ok = np.isfinite(top)
    e = np.full(top.shape, 255, dtype=np.int64)
    exp = np.frexp(np.where(ok & (top > 0), top, 1.0))[1] - 1
    e[ok] = np.where(top > 0, np.maximum(exp - 6, -126), -126)[ok] + 127
    n = np.zeros(x.shape, dtype=np.int64)
    n[ok] = np.clip(np.rint(np.ldexp(x[ok], -(e[ok][..., None] - 127).astype(int))), -127, 127)
    return n, e


def held(n, e):
    """The values that quantised rows stand for."""
    y = np.ldexp(n.astype(np.float64), (e[..., None] - 127).astype(int))
    return np.where(e[..., None] == 255, np.nan, y)
