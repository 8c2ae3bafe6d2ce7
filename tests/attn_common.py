"""Inputs and error bounds shared by the tests of the stand-alone attention."""
import numpy as np

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}  # half a step of the storage type, relative


def rounded(torch, a, dtype):
    """Float64 array -> (tensor of the storage type on the CPU, its exact float64 values)."""
    t = torch.from_numpy(np.asarray(a, dtype=np.float64)).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    return t, t.double().numpy()


def offsets(n):
    return np.concatenate([[0], np.cumsum(n)]).astype(np.int32)


def rel(dtype, dh, n, ref, cap):
    """Relative error of a weight or a product of the kernels, worst case.

    u = 2^-24.  A score: dh products summed in fp32, each at most (dh + 2) u off
    relative to sum |q k|, and a few roundings of its own size; a cap adds the
    error of tanh, at most 8 u relative to the cap.  exp of a difference d: 4 u
    |d| and 4 u.  The sum of n weights and of n products: n u.  A weight moves by
    the errors of its own score and of the sum, hence twice.  bf16 storage: the
    two-term split leaves 2^-16 of a weight, once for the weight and once for
    the gradient of its score."""
    u = 2.0 ** -24
    score = (dh + 6) * u * ref["score"] + 8 * u * cap + 4 * u * (1 + ref["x"])
    return 2 * score + 2 * (n + 2 * dh + 8) * u + (2.0 ** -15 if dtype == "bf16" else 0.0)


def worst(got, want, mag, dtype, c):
    """Largest error over its bound; NaN and infinities have to agree."""
    got, want = np.asarray(got, dtype=np.float64), np.asarray(want)
    assert got.shape == want.shape
    odd = ~np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), "NaN in other places"
    assert np.array_equal(got[odd & ~np.isnan(want)], want[odd & ~np.isnan(want)])
    with np.errstate(invalid="ignore"):
        bound = HALF[dtype] * np.abs(want) * (1 + c) + c * mag + 1e-37
        e = np.abs(got - want) / bound
    e = e[~odd]
    return float(e.max()) if e.size else 0.0


# ---- long histories in which every block of 32 rows counts

def deep(dtype, dh, L, ref, cap=0.0):
    """rel with the depth that sums over a long history have: a wave takes at most
    512 rows of a chunk (fewer than 2^20 rows times kv heads in all), and at most
    one chunk in 64 rows is joined one after the other (a bucket's in fp64)."""
    return rel(dtype, dh, 512 + -(-int(max(L)) // 64), ref, cap)


def spread(rng, L, m, H, Hk, dh, buckets=128):
    """Inputs as float64 arrays, options and offsets: block b of a request's rows has
    its K and V mostly in feature b % dh, so that each feature of out and dq is a sum
    over few blocks; buckets of equal width, so that each is one over few as well (the
    short requests', whose weights are larger, in a bucket beyond the longest)."""
    rows, off = int(np.sum(L)), offsets(L)
    row = np.arange(rows) - np.repeat(off[:-1], L)
    f = dict(q=rng.standard_normal((int(np.sum(m)), H, dh)), dout=rng.standard_normal((int(np.sum(m)), H, dh)))
    for n, gain in (("k", 1.0), ("v", 2.0)):
        x = 0.002 * rng.standard_normal((rows, Hk, dh))
        x[np.arange(rows), :, row // 32 % dh] += gain
        f[n] = x
    edges = np.unique(np.linspace(1, max(L) - 1, buckets - 1).astype(np.int32))
    far = [l + (max(L) if l < 1000 else 0) for l in L]
    tgt_pos = np.repeat(far, m).astype(np.int32) + rng.integers(0, 9, size=int(np.sum(m)), dtype=np.int32)
    bias = rng.standard_normal((H, len(edges) + 1)).astype(np.float32)
    return f, dict(edges=edges, bias=bias, tgt_pos=tgt_pos)


SPREAD = [  # Hk = H, d_head, history lengths, targets: several kv heads a workgroup, backward tiles 1, 2 and 4
    (4, 32, [40000, 0, 33, 27000, 17], [3, 3, 1, 5, 5]),
    (4, 32, [40000, 0, 33, 27000, 17], [20, 3, 1, 3, 5]),
    (4, 32, [66000], [40]),
    (6, 32, [30000, 1, 20000], [7, 2, 4]),
    (4, 64, [34000, 100, 32000], [16, 4, 2]),
    (2, 128, [80000, 500, 52000], [5, 17, 2]),
]
