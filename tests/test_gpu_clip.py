"""The norm of many gradients and clipping on the GPU against long sums on the host:
odd sizes and alignments, many tensors, counts of rows, values at the ends of fp32."""
import numpy as np
import pytest

from layers_common import HALF, dtype_of
from oracle import layers_oracle as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available(), "GPU tests need a GPU"
    return t


def make(torch, sizes, seed=0, gain=1.0):
    rng = np.random.default_rng(seed)
    return [torch.from_numpy(gain * rng.standard_normal(n)).to(torch.bfloat16 if b else torch.float32).cuda() for n, b in sizes]


def host(gs):
    return [g.double().cpu().numpy() for g in gs]


def close(norm, want):
    # fp64 sums of exact squares: at most 2^-40 off, then fp32, whose range a norm may leave
    # (7.3e38 rounds to infinity: the largest fp32 is 3.4e38)
    if want > 3.5e38:
        assert float(norm) == float("inf")
        return
    assert abs(float(norm) - want) <= (HALF["f32"] + 2.0 ** -40) * want, (float(norm), want)


def scaled(got, want, dtype):
    e = np.abs(got.double().cpu().numpy() - want)
    # rounded from fp64 to fp32, and to bf16 from there; half a step of the smallest numbers
    # is 2^-150 of fp32 (steps of 2^-149) and 2^-134 of bf16 (steps of 2^-133)
    least = 2.0 ** -134 + 2.0 ** -150 if dtype == "bf16" else 2.0 ** -150
    assert (e <= (HALF[dtype] + (HALF["f32"] if dtype == "bf16" else 2.0 ** -50)) * np.abs(want) + 1.0001 * least).all()


LISTS = {
    "one": [(1, False)],
    "odd": [(1, False), (7, True), (8, False), (9, True), (4097, False), (8191, True), (8193, False), (0, False), (33, True)],
    "pieces": [(8192, False), (8192 * 3, True), (8192 * 5 + 1, False)],
    "many": [(1 + 37 * i % 4000, i % 3 == 0) for i in range(200)],
    "launch_borders": [(100, False)] * 64,
    "launch_borders_1": [(100, False)] * 65,
    "large": [(20_000_003, False), (5_000_001, True)],
}


@pytest.mark.parametrize("max_norm", [0.5, 1e9, float("inf")])
@pytest.mark.parametrize("name", list(LISTS))
def test_clip(torch, name, max_norm):
    from paper_2511_06077_amd.layers import GradientNorm
    gs = make(torch, LISTS[name])
    f = host(gs)
    want, factor = O.clip(f, max_norm)
    plan = GradientNorm(max_norm)
    close(plan.norm(gs), want)
    assert all(np.array_equal(a, b) for a, b in zip(host(gs), f))
    out = [torch.zeros_like(g, dtype=torch.float32 if i % 2 else torch.bfloat16) for i, g in enumerate(gs)]
    close(plan.clip(gs, out=out), want)
    assert all(np.array_equal(a, b) for a, b in zip(host(gs), f))
    for i, (o, x) in enumerate(zip(out, f)):
        scaled(o, x * factor, "f32" if i % 2 else "bf16")
    again = [torch.zeros_like(o) for o in out]
    plan.clip(gs, out=again)
    assert all(torch.equal(a, b) for a, b in zip(again, out))
    close(plan.clip(gs), want)
    for g, x in zip(gs, f):
        scaled(g, x * factor, "bf16" if g.dtype == torch.bfloat16 else "f32")


@pytest.mark.parametrize("at", [1, 2, 3, 5])
def test_unaligned_views(torch, at):
    """Gradients and results at any element, and what lies around them."""
    from paper_2511_06077_amd.layers import GradientNorm
    base = [torch.full((30000,), 7.0, device="cuda"), torch.full((30000,), 7.0, dtype=torch.bfloat16, device="cuda")]
    gs = [b[at:at + 20001 + i] for i, b in enumerate(base)]
    for i, g in enumerate(gs):
        g.copy_(make(torch, [(g.numel(), False)], seed=i)[0])
    f = host(gs)
    want, factor = O.clip(f, 1.0)
    outs = [torch.full((30000,), 7.0, device="cuda") for _ in gs]
    views = [o[at + 1:at + 1 + g.numel()] for o, g in zip(outs, gs)]
    close(GradientNorm(1.0).clip(gs, out=views), want)
    for o, v, x in zip(outs, views, f):
        scaled(v, x * factor, "f32")
        assert bool((o[:at + 1] == 7).all()) and bool((o[at + 1 + v.numel():] == 7).all())
    close(GradientNorm(1.0).clip(gs), want)
    for b, g in zip(base, gs):
        assert bool((b[:at] == 7).all()) and bool((b[at + g.numel():] == 7).all())


@pytest.mark.parametrize("used", [0, 1, 37, 500, 501, -3])
def test_rows_in_use(torch, used):
    """What lies behind the count is neither read nor written."""
    from paper_2511_06077_amd.layers import GradientNorm
    a, b = make(torch, [(500 * 72, False), (1000, False)])
    a = a.view(500, 72)
    live = min(max(used, 0), 500)
    a[live:] = float("nan")
    f = [a[:live].double().cpu().numpy(), b.double().cpu().numpy()]
    want, factor = O.clip(f, 2.0)
    count = torch.tensor([used], dtype=torch.int32, device="cuda")
    out = [torch.full_like(a, 7.0), torch.full_like(b, 7.0)]
    close(GradientNorm(2.0).clip([a, b], out=out, counts=[count, None]), want)
    scaled(out[0][:live], f[0] * factor, "f32")
    assert bool((out[0][live:] == 7).all())
    close(GradientNorm(2.0).clip([a, b], counts=[count, None]), want)
    scaled(a[:live], f[0] * factor, "f32")
    assert bool(torch.isnan(a[live:]).all())


def test_ends_of_fp32(torch):
    """Squares and factors that fp32 could not hold."""
    from paper_2511_06077_amd.layers import GradientNorm
    for gain in (1e37, 1e-37, 1e-20, 1e25):
        gs = make(torch, [(5000, False), (300, True)], gain=gain)
        f = host(gs)
        for max_norm in (1.0, 1e-30, 1e-3 * gain):
            want, factor = O.clip(f, max_norm)
            out = [torch.zeros_like(g) for g in gs]
            close(GradientNorm(max_norm).clip(gs, out=out), want)
            for o, x in zip(out, f):
                scaled(o, x * factor, "bf16" if o.dtype == torch.bfloat16 else "f32")


@pytest.mark.parametrize("odd", [float("nan"), float("inf"), -float("inf")])
def test_a_norm_that_is_not_finite_changes_nothing(torch, odd):
    from paper_2511_06077_amd.layers import GradientNorm
    gs = make(torch, [(5000, False), (300, True)])
    gs[0][17] = odd
    keep = [g.clone() for g in gs]
    out = [torch.zeros_like(g) for g in gs]
    norm = GradientNorm(0.1).clip(gs, out=out)
    assert not torch.isfinite(norm)
    GradientNorm(0.1).clip(gs)
    for g, o, k in zip(gs, out, keep):
        assert torch.equal(g.nan_to_num(1.5), k.nan_to_num(1.5)) and torch.equal(o.nan_to_num(1.5), k.nan_to_num(1.5))


def test_nothing_to_clip(torch):
    from paper_2511_06077_amd.layers import GradientNorm
    assert float(GradientNorm(1.0).clip([])) == 0.0
    assert float(GradientNorm(1.0).clip([torch.zeros(0, device="cuda"), torch.zeros((4, 3), device="cuda")])) == 0.0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("at", [0, 1])
def test_bf16_results_are_rounded_once(torch, dtype, at):
    """Products a little beside the middle of two bf16 numbers, nearer to it than fp32 can
    tell: rounded to fp32 they are the middle, and from there to the even number, which is
    the wrong one.  Aligned views and others."""
    from paper_2511_06077_amd.layers import GradientNorm
    k = np.arange(2, 128, dtype=np.float64)
    if dtype == "f32":
        # factors of 1 -+ 2^-40 of an odd multiple of half a step (2^-8), k even and odd
        g = np.concatenate([1 + (2 * k + 1) * 2.0 ** -8, -(1 + (2 * k + 1) * 2.0 ** -8)])
        factors = [1 - 2.0 ** -40]
    else:
        # 128 * factor is the middle of 65 + 66 halves, or of 64 and 64.5, and a little more or less
        g = np.concatenate([np.full(100, 128.0), np.full(27, -128.0)])
        factors = [m / 128 * (1 + s * 2.0 ** -40) for m in (64.25, 64.75, 65.25, 97.25) for s in (1, -1)]
    store = torch.zeros(len(g) + at, dtype=dtype_of(torch, dtype), device="cuda")
    t = store[at:]
    t.copy_(torch.from_numpy(g))
    assert np.array_equal(host([t])[0], g)
    norm = float(np.sqrt(np.sum(g.astype(np.longdouble) ** 2)))
    for f in factors:
        out = torch.zeros(len(g) + at, dtype=torch.bfloat16, device="cuda")[at:]
        GradientNorm(norm * f).clip([t], out=[out])
        # in fp64 exact to 2^-52, twice; the middles are 2^-41 away
        want = g * f
        step = 2.0 ** (np.floor(np.log2(np.abs(want))) - 7)
        assert np.array_equal(host([out])[0], np.rint(want / step) * step), f
