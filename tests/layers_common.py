"""Shared by the tests of the operators between ids, rows and gradients."""
import numpy as np

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}  # half a step of the storage type, relative


def dtype_of(torch, name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def rounded(torch, a, dtype):
    """Float64 array -> (tensor of the storage type on the GPU, its exact float64 values)."""
    t = torch.from_numpy(np.asarray(a, dtype=np.float64)).to(dtype_of(torch, dtype))
    return t.cuda(), t.double().numpy()


def strided(torch, t, pad=8):
    """The same rows inside wider ones whose other columns are NaN."""
    wide = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype, device=t.device)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def worst(got, want, err, dtype):
    """Largest error over its bound: half a step of the rounded result (which may sit
    on the other side of a step by err), err, and fp32's smallest numbers."""
    got = got.double().cpu().numpy() if hasattr(got, "cpu") else np.asarray(got, dtype=np.float64)
    assert got.shape == np.shape(want), (got.shape, np.shape(want))
    assert np.isfinite(got).all(), "not finite"
    bound = HALF[dtype] * (np.abs(want) + err) + err + 1e-37
    e = np.abs(got - want) / bound
    return float(e.max()) if e.size else 0.0
