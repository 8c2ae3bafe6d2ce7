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
