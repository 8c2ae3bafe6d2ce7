"""Norms around a block on the GPU against the float64 oracle: every form, odd
widths, rows far from zero and of the largest values, strides, rows in place."""
import numpy as np
import pytest

from layers_common import rounded, strided, worst
from oracle import layers_oracle as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available(), "GPU tests need a GPU"
    return t


FORMS = {
    "pre": dict(),
    "pre_plain": dict(pre=()),
    "block": dict(block=True),
    "block_only": dict(block=True, pre=False),
    "sigmoid": dict(block=True, gate="sigmoid", post=("w",), ls=True),
    "silu": dict(block=True, gate="silu", post=("w", "b"), pre=("w", "b"), ls=True),
    "gate_only": dict(block=True, gate="silu", pre=False),
    "post_plain": dict(block=True, post=(), pre=(), ls=True),
    "bias_only": dict(block=True, post=("", "b"), pre=("", "b")),
}


def vectors(torch, rng, d, names):
    """((tensors), (float64)) of a norm's parameters"""
    got = [None if not n else rounded(torch, (1.0 if n == "w" else 0.0) + 0.3 * rng.standard_normal(d), "f32") for n in names]
    return tuple(None if g is None else g[0] for g in got), [None if g is None else g[1] for g in got] + [None] * (2 - len(got))


def build(torch, n, d, dtype, kind, form, seed=0, spread=None, eps=1e-6):
    """Tensors and arguments of a call, and the oracle's results for it."""
    rng = np.random.default_rng([n, d, seed])
    f = dict(FORMS[form])
    block, gate = f.get("block", False), f.get("gate")
    t, a = {}, {}
    for name in ["x", "dy", "dh"] + (["block"] if block else []) + (["gate"] if gate else []):
        v = rng.standard_normal((n, d))
        if spread is not None and name in ("x", "block"):
            v = spread(rng, v)
        t[name], a[name] = rounded(torch, v, dtype)
    given, want = {}, {}
    pre = f.get("pre", ("w",))
    if pre is False:
        given["pre"] = want["pre"] = False
        t["dy"] = a["dy"] = None
    else:
        given["pre"], want["pre"] = vectors(torch, rng, d, pre)
    if f.get("post") is not None:
        given["post"], want["post"] = vectors(torch, rng, d, f["post"])
    if f.get("ls"):
        given["layer_scale"], want["ls"] = rounded(torch, 0.5 + 0.2 * rng.standard_normal(d), "f32")
    scale = float(np.float32(0.7))
    with np.errstate(over="ignore"):
        ref = O.norm(a["x"], kind, float(np.float32(eps)), scale, a.get("block"), a.get("gate"), gate, dy=a["dy"], dh=a["dh"], **want)
    from paper_2511_06077_amd.layers import BlockNorm
    plan = BlockNorm(d, kind=kind, gate=gate, scale=scale, eps=eps, dtype=t["x"].dtype, backward=True)
    for name in ("block", "gate"):
        if name in t:
            given[name] = t[name]
    return plan, t, given, ref


def check(got, ref, dtype, block):
    h, y, g = got
    e = {}
    if block:
        e["h"] = worst(h, ref["h"], ref["h_err"], dtype)
    if y is not None:
        e["y"] = worst(y, ref["y"], ref["y_err"], dtype)
    for name, v, kind in (("dx", g.x, dtype), ("dblock", g.block, dtype), ("dgate", g.gate, dtype), ("pre_w", g.pre[0], "f32"),
                          ("pre_b", g.pre[1], "f32"), ("post_w", g.post[0], "f32"), ("post_b", g.post[1], "f32"),
                          ("ls", g.layer_scale, "f32")):
        if v is not None:
            e[name] = worst(v, ref[name], ref[name + "_err"], kind)
    assert max(e.values()) <= 1.0, e


def both(plan, t, given):
    h, y = plan.forward(t["x"], **given)
    return h, y, plan.backward(t["dy"], t["x"], dh=t["dh"], **given)


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("n,d", [(1, 256), (5, 8), (33, 72), (9, 264), (7, 1000), (3, 2000), (2, 4096)])
def test_forms(torch, n, d, form, dtype, kind):
    plan, t, given, ref = build(torch, n, d, dtype, kind, form)
    check(both(plan, t, given), ref, dtype, "block" in given)


@pytest.mark.parametrize("n,d", [(20000, 32), (9001, 64), (5000, 128), (9000, 256), (3000, 512), (2500, 1024)])
def test_many_rows(torch, n, d):
    """More rows than one round of the workgroups has, and the sums over them."""
    plan, t, given, ref = build(torch, n, d, "bf16", "layer", "silu")
    got = both(plan, t, given)
    check(got, ref, "bf16", True)
    again = plan.backward(t["dy"], t["x"], dh=t["dh"], **given)
    for a, b in ((got[2].x, again.x), (got[2].pre[0], again.pre[0]), (got[2].post[1], again.post[1]),
                 (got[2].layer_scale, again.layer_scale)):
        assert torch.equal(a, b)


SPREADS = {
    "far_from_zero": lambda rng, v: 1000.0 + v,
    "one_large": lambda rng, v: v * np.where(np.arange(v.shape[1]) == 3, 1e4, 1.0),
    "scales_by_row": lambda rng, v: v * 2.0 ** rng.integers(-40, 40, size=(len(v), 1)),
    "squares_leave_fp32": lambda rng, v: v * 2.0 ** np.where(np.arange(len(v)) % 3 == 0, 100.0, 0.0)[:, None],
    "tiny": lambda rng, v: v * 1e-30,
    "zeros": lambda rng, v: v * (np.arange(len(v)) % 2)[:, None],
}


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("name", list(SPREADS))
@pytest.mark.parametrize("d", [64, 72, 256, 264, 1000])  # (teams of 8, 16, 32, 64 and 128 lanes)
def test_values(torch, d, name, kind):
    for form in ("pre", "sigmoid"):
        plan, t, given, ref = build(torch, 13, d, "f32", kind, form, spread=SPREADS[name], seed=3)
        check(both(plan, t, given), ref, "f32", "block" in given)


@pytest.mark.parametrize("d", [64, 264, 1000])
def test_odd_values_stay_in_their_rows(torch, d):
    for kind in ("rms", "layer"):
        plan, t, given, ref = build(torch, 11, d, "f32", kind, "sigmoid", seed=5)
        clean = both(plan, t, given)
        t["x"][3, 1], given["block"][6, 2], given["gate"][8, 0] = float("nan"), float("inf"), float("nan")
        h, y, g = both(plan, t, given)
        for a, b in ((h, clean[0]), (y, clean[1]), (g.x, clean[2].x), (g.block, clean[2].block), (g.gate, clean[2].gate)):
            keep = [i for i in range(11) if i not in (3, 6, 8)]
            assert torch.equal(a[keep], b[keep])
        for row in (3, 6, 8):
            assert torch.isnan(y[row]).any()


def test_strides_and_no_gradient_of_h(torch):
    plan, t, given, _ = build(torch, 70, 200, "bf16", "layer", "silu")
    want = both(plan, t, given)
    loose = {k: strided(torch, v) if k in ("block", "gate") else v for k, v in given.items()}
    got = both(plan, {k: strided(torch, v) for k, v in t.items()}, loose)
    for a, b in zip(got[2][:3], want[2][:3]):
        assert torch.equal(a, b)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    none = plan.backward(t["dy"], t["x"], dh=None, **given)
    zero = plan.backward(t["dy"], t["x"], dh=torch.zeros_like(t["x"]), **given)
    assert torch.equal(none.x, zero.x) and torch.equal(none.block, zero.block) and torch.equal(none.layer_scale, zero.layer_scale)


def test_results_on_their_inputs(torch):
    """h on x, y on block; dx on dh, dblock on dy, dgate on gate, with wider rows around."""
    from paper_2511_06077_amd import stca
    for n, d in ((2500, 64), (300, 1000)):
        plan, t, given, _ = build(torch, n, d, "bf16", "rms", "sigmoid")
        h, y, g = both(plan, t, given)
        m = plan._forms[True, True]
        fresh = {k: v.clone() for k, v in {**t, **{k: given[k] for k in ("block", "gate")}}.items()}
        inp = stca.norm_in(fresh["x"], fresh["block"], fresh["gate"], pre_w=given["pre"][0], post_w=given["post"][0],
                           layer_scale=given["layer_scale"])
        s = plan.stream()
        stca.stca_norm_forward(m, inp, n, fresh["x"], 0, fresh["block"], 0, s)
        assert torch.equal(fresh["x"], h) and torch.equal(fresh["block"], y)
        fresh["x"].copy_(t["x"]), fresh["block"].copy_(given["block"])
        stca.stca_norm_backward(m, inp, n, fresh["dh"], 0, fresh["dy"], 0,
                                stca.norm_grads(fresh["dh"], fresh["dy"], fresh["gate"]), plan.ws, plan.ws_bytes, s)
        assert torch.equal(fresh["dh"], g.x) and torch.equal(fresh["dy"], g.block) and torch.equal(fresh["gate"], g.gate)


def test_no_rows(torch):
    from paper_2511_06077_amd.layers import BlockNorm
    plan = BlockNorm(64, gate="silu", backward=True, dtype=torch.float32)
    none, w = torch.empty((0, 64), device="cuda"), torch.ones(64, device="cuda")
    h, y = plan.forward(none, block=none, gate=none, post=(w,), pre=(w,))
    assert h.shape == y.shape == (0, 64)
    g = plan.backward(none, none, dh=none, block=none, gate=none, post=(w, w), pre=(w,), layer_scale=w)
    assert g.x.shape == (0, 64) and all(bool((v == 0).all()) for v in (g.pre[0], *g.post, g.layer_scale))


def test_gradients_against_differences(torch):
    """fp32 central differences of the forward at some coordinates of every input."""
    plan, t, given, ref = build(torch, 3, 24, "f32", "layer", "silu", seed=9)
    g = plan.backward(t["dy"], t["x"], dh=t["dh"], **given)
    def f():
        h, y = plan.forward(t["x"], **given)
        return float((h.double() * t["dh"].double()).sum() + (y.double() * t["dy"].double()).sum())
    size = 3 * 24 * 4.0  # of f's terms: each at most a few, off by some 40 U
    for where, grad in ((t["x"], g.x), (given["block"], g.block), (given["gate"], g.gate), (given["pre"][0], g.pre[0]),
                        (given["pre"][1], g.pre[1]), (given["post"][0], g.post[0]), (given["post"][1], g.post[1]),
                        (given["layer_scale"], g.layer_scale)):
        flat, gf = where.view(-1), grad.reshape(-1)
        for i in (0, 7, flat.numel() - 1):
            keep, step = float(flat[i]), 2.0 ** -7
            flat[i] = keep + step
            up, hi = f(), float(flat[i])
            flat[i] = keep - step
            down, lo = f(), float(flat[i])
            flat[i] = keep
            # rounding of f over the step, and the third derivative times step^2 / 6
            bound = 80 * O.U * size / (hi - lo) + step * step * 20
            assert abs((up - down) / (hi - lo) - float(gf[i])) <= bound


def doubles(t):
    return None if t is None else t.double().cpu().numpy()


def oracle(t, given, kind, act, eps=1e-6, rows=slice(None)):
    """The oracle's results for rows of a call's tensors."""
    def pair(p):
        return p if p is None or p is False else tuple(map(doubles, (*p, None, None)[:2]))
    def some(v):
        return None if v is None else doubles(v[rows])
    return O.norm(some(t["x"]), kind, float(np.float32(eps)), float(np.float32(0.7)), some(given.get("block")),
                  some(given.get("gate")), act, pre=pair(given["pre"]), post=pair(given.get("post")),
                  ls=doubles(given.get("layer_scale")), dy=some(t["dy"]), dh=some(t["dh"]))


@pytest.mark.parametrize("act", ["sigmoid", "silu"])
@pytest.mark.parametrize("form", ["full", "gate_only"])
@pytest.mark.parametrize("d", [72, 1000])
def test_gates_far_from_zero(torch, d, form, act):
    """Gates up to where the sigmoid leaves fp32, of either sign: the small one of s and
    1 - s, and a SiLU's slope, keep fp32's accuracy."""
    from paper_2511_06077_amd.layers import BlockNorm
    _, t, given, _ = build(torch, 29, d, "f32", "rms", "sigmoid" if form == "full" else "gate_only", seed=4)
    plan = BlockNorm(d, kind="rms", gate=act, scale=float(np.float32(0.7)), dtype=torch.float32, backward=True)
    rng = np.random.default_rng(d)
    gate = rng.uniform(-95, 95, size=(29, d))
    gate[:, :8] = [0.0, -0.0, 88.0, -88.0, 87.3, -87.3, 1e-30, -20.0]
    given["gate"], _ = rounded(torch, gate, "f32")
    if form == "full":
        # nothing else in the way of what is small: h is the gated block's alone
        t["x"].zero_()
        t["dh"].zero_()
    check(both(plan, t, given), oracle(t, given, "rms", act), "f32", True)


def test_gates_without_end(torch):
    """sigmoid(inf) = 1 and sigmoid(-inf) = 0, with no slope; silu(inf) stays infinite; a NaN stays one."""
    from paper_2511_06077_amd.layers import BlockNorm
    x, o = torch.zeros((4, 64), device="cuda"), torch.ones((4, 64), device="cuda")
    gate = torch.tensor([float("inf"), -float("inf"), float("nan"), 3e38], device="cuda")[:, None].repeat(1, 64)
    sig = BlockNorm(64, gate="sigmoid", dtype=torch.float32, backward=True)
    h, _ = sig.forward(x, block=o, gate=gate, pre=False)
    assert bool((h[[0, 3]] == 1).all()) and bool((h[1] == 0).all()) and bool(torch.isnan(h[2]).all())
    g = sig.backward(None, x, dh=o, block=o, gate=gate, pre=False)
    assert bool((g.gate[[0, 1, 3]] == 0).all()) and bool(torch.isnan(g.gate[2]).all())
    h, _ = BlockNorm(64, gate="silu", dtype=torch.float32).forward(x, block=o, gate=gate, pre=False)
    assert bool(torch.isposinf(h[0]).all()) and bool(torch.isnan(h[2]).all()) and bool((h[3] == gate[3]).all())


# ---- more rows than the workgroups take at once

def launched(torch, d):
    """(rows a workgroup takes at once, rows of a forward's and of a backward's first turn)"""
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    rows = 256 // max(8, 1 << (-(-d // 8) - 1).bit_length()) if d <= 512 else 1
    return rows, 16 * cus * rows, 2 * cus * rows


WIDE = [(64, "bf16"), (72, "f32"), (256, "bf16"), (512, "bf16"), (520, "f32"), (1000, "bf16"), (2000, "bf16"), (2000, "f32"),
        (4096, "bf16"), (4096, "f32")]  # (teams of 8, 16, 32, 64, 128, 256 and 512 lanes)


def large(torch, n, d, dtype, seed=0):
    """Tensors of n rows, drawn on the GPU, for the form with everything in it."""
    gen = torch.Generator(device="cuda").manual_seed(1000 * seed + d)
    kind = torch.bfloat16 if dtype == "bf16" else torch.float32
    def normal(shape, middle=0.0, gain=1.0):
        return middle + gain * torch.randn(shape, generator=gen, device="cuda")
    t = {k: normal((n, d)).to(kind) for k in ("x", "dy", "dh")}
    given = {k: normal((n, d)).to(kind) for k in ("block", "gate")}
    given.update(pre=(normal(d, 1.0, 0.3), normal(d, 0.0, 0.3)), post=(normal(d, 1.0, 0.3), normal(d, 0.0, 0.3)),
                 layer_scale=normal(d, 0.5, 0.2))
    return t, given


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("d,dtype", WIDE)
def test_rows_of_later_turns(torch, d, dtype, kind):
    """A workgroup's second turn of rows, forward and backward, gives bit for bit what a call
    of those rows alone gives, and some of them are compared with the oracle."""
    from paper_2511_06077_amd.layers import BlockNorm
    rows, first, _ = launched(torch, d)
    n = first + 37 * rows + min(rows - 1, 3)
    t, given = large(torch, n, d, dtype)
    plan = BlockNorm(d, kind=kind, gate="silu", scale=float(np.float32(0.7)), dtype=t["x"].dtype, backward=True)
    h, y, g = both(plan, t, given)
    whole = (h, y, g.x, g.block, g.gate)
    def part(at):
        cut = {**given, **{k: given[k][at] for k in ("block", "gate")}}
        ph, py, pg = both(plan, {k: v[at] for k, v in t.items()}, cut)
        return ph, py, pg.x, pg.block, pg.gate
    for at in (slice(0, first // 2), slice(first // 2, first), slice(first, n)):  # (each a forward's one turn)
        for a, b in zip(whole, part(at)):
            assert torch.equal(a[at], b)
    # single turns of the backward too: where its second one begins, and the last rows
    for a0 in (launched(torch, d)[2] - 5, n - 11):
        at = slice(a0, a0 + 11)
        for a, b in zip(whole, part(at)):
            assert torch.equal(a[at], b)
        ref = oracle(t, given, kind, "silu", rows=at)
        for name, v in zip(("h", "y", "dx", "dblock", "dgate"), whole):
            assert worst(v[at], ref[name], ref[name + "_err"], dtype) <= 1.0, name


@pytest.mark.parametrize("d,dtype", [(64, "f32"), (256, "bf16"), (512, "f32"), (1000, "f32"), (1000, "bf16"), (2000, "bf16"),
                                     (4096, "f32")])
def test_results_on_their_inputs_in_later_turns(torch, d, dtype):
    """h on x, y on block, and y on gate; dx on dh, dblock on dy, dgate on gate: with the
    next row of a team on its way while this one is written."""
    from paper_2511_06077_amd import stca
    from paper_2511_06077_amd.layers import BlockNorm
    rows, first, _ = launched(torch, d)
    n = first + 5 * rows + 1
    t, given = large(torch, n, d, dtype, seed=1)
    plan = BlockNorm(d, kind="layer", gate="sigmoid", dtype=t["x"].dtype, backward=True)
    h, y, g = both(plan, t, given)
    m, s = plan._forms[True, True], plan.stream()
    for y_on in ("block", "gate"):
        f = {k: v.clone() for k, v in {**t, **{k: given[k] for k in ("block", "gate")}}.items()}
        inp = stca.norm_in(f["x"], f["block"], f["gate"], 0, 0, 0, *given["pre"], *given["post"], given["layer_scale"])
        stca.stca_norm_forward(m, inp, n, f["x"], 0, f[y_on], 0, s)
        assert torch.equal(f["x"], h) and torch.equal(f[y_on], y)
    f = {k: v.clone() for k, v in {**t, **{k: given[k] for k in ("block", "gate")}}.items()}
    inp = stca.norm_in(f["x"], f["block"], f["gate"], 0, 0, 0, *given["pre"], *given["post"], given["layer_scale"])
    stca.stca_norm_backward(m, inp, n, f["dh"], 0, f["dy"], 0, stca.norm_grads(f["dh"], f["dy"], f["gate"]), plan.ws,
                            plan.ws_bytes, s)
    assert torch.equal(f["dh"], g.x) and torch.equal(f["dy"], g.block) and torch.equal(f["gate"], g.gate)


@pytest.mark.parametrize("n,d", [(1100, 2000), (1100, 4096), (2100, 512), (17000, 64)])
def test_sums_over_later_turns(torch, n, d):
    """The gradients of [d] where workgroups of the backward have a second turn and more."""
    assert n > launched(torch, d)[2]
    plan, t, given, ref = build(torch, n, d, "bf16", "layer", "silu", seed=6)
    check(both(plan, t, given), ref, "bf16", True)


@pytest.mark.parametrize("n,d", [(200000, 520), (1500000, 64)])
def test_sums_at_their_bound(torch, n, d):
    """A long sum whose every term but the first of a workgroup's is half a step of it, and lost."""
    from paper_2511_06077_amd.layers import BlockNorm
    first = launched(torch, d)[2]
    dy = torch.full((n, d), 2.0 ** -24, dtype=torch.bfloat16, device="cuda")
    dy[:first] = 1.0
    x = torch.ones((n, d), dtype=torch.bfloat16, device="cuda")
    plan = BlockNorm(d, backward=True)
    got = plan.backward(dy, x, pre=(None, torch.zeros(d, device="cuda"))).pre[1]
    want = np.full(d, first + (n - first) * 2.0 ** -24)
    assert worst(got, want, O.sum_depth(n, d) * O.U * want, "f32") <= 1.0


@pytest.mark.parametrize("d", [72, 264, 1000, 2000])
def test_rows_of_one_value(torch, d):
    """A layer norm of rows whose values are all the same, and of such rows with one that is a
    step of fp32 off: far from zero, where the mean's rounding is more than the deviation."""
    values = np.float32([1.0, -300.0, 1e4, 1e5, 1e6 + 0.25, -3e7, 1e8, 7e12, 1e18, -3e19, 1e30, 3e38])
    def spread(rng, v):
        v[:] = np.repeat(values, 2)[:, None]
        v[1::2, 1] = np.nextafter(values, np.float32(0)).astype(np.float64)
        return v
    for form in ("pre", "sigmoid"):
        plan, t, given, ref = build(torch, 2 * len(values), d, "f32", "layer", form, spread=spread, seed=8)
        if form == "sigmoid":  # (the block's rows are such, and the next norm's are others)
            t["x"].copy_(t["dh"])
            ref = oracle(t, given, "layer", "sigmoid")
        check(both(plan, t, given), ref, "f32", "block" in given)
