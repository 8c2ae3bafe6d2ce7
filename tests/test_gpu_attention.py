"""Stand-alone attention on the GPU against the float64 oracle: forward and
gradients over types, head layouts, lengths and masks, with worst-case error
bounds (attn_common.rel), and the calls around it: strides, streams, captured
graphs, missing host offsets, guard regions, bitwise repeats."""
import numpy as np
import pytest

from attn_common import HALF, offsets, rel, rounded, worst
from oracle import attn_oracle as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available(), "GPU tests need a GPU"
    return t


def edges_of(n, top=600):
    from paper_2511_06077_amd.attention import bias_edges
    return bias_edges(n, max(1, n // 3), max(top, n)) if n > 1 else np.zeros(0, dtype=np.int32)


class Case:
    """Seeded inputs of a ragged batch, the plan's options and the oracle's view."""

    def __init__(self, torch, L, m, *, dtype="bf16", H=2, Hk=None, dh=32, cap=0.0, nb=0, masked=False, time=False,
                 seed=0, q_gain=1.0, bias_at=None):
        rng = np.random.default_rng([seed, dh, H])
        self.torch, self.dtype, self.dh, self.H, self.Hk = torch, dtype, dh, H, Hk or H
        self.hoff, self.toff = offsets(L), offsets(m)
        nh, nt = int(self.hoff[-1]), int(self.toff[-1])
        self.t, self.f = {}, {}
        for n, rows, heads, gain in (("q", nt, H, q_gain), ("k", nh, self.Hk, 1.0), ("v", nh, self.Hk, 1.0),
                                     ("dout", nt, H, 1.0)):
            self.t[n], self.f[n] = rounded(torch, gain * rng.standard_normal((rows, heads, dh)), dtype)
        self.edges = edges_of(nb) if nb else None
        self.bias = rng.standard_normal((H, nb)).astype(np.float32) if nb else None
        if bias_at is not None:
            for b, x in bias_at.items():
                self.bias[:, b] = x
        self.masked, self.cap, self.scale = masked, cap, float(np.float32(1.0 / np.sqrt(dh)))
        self.hist_pos = self.tgt_pos = None
        if nb or masked:
            tp, hp = [], []
            for l, n in zip(L, m):
                p = np.cumsum(rng.integers(0, 9, size=l)) if time else np.arange(l)
                hp.append(rng.permutation(p) if time else p)
                hi = int(p[-1]) if l else 0
                tp.append(rng.integers(-1 if masked else hi, hi + 5, size=n))
            self.tgt_pos = np.concatenate(tp).astype(np.int32)
            self.hist_pos = np.concatenate(hp).astype(np.int32) if time else None

    def opts(self):
        return dict(n_kv_heads=self.Hk, dtype=self.t["q"].dtype, scale=self.scale, softcap=self.cap, edges=self.edges,
                    masked=self.masked)

    def given(self):
        def dev(a):
            return None if a is None else self.torch.from_numpy(a).cuda()
        return dict(tgt_pos=dev(self.tgt_pos), hist_pos=dev(self.hist_pos), bias=dev(self.bias))

    def plan(self, **kw):
        from paper_2511_06077_amd.attention import CrossAttention
        return CrossAttention(self.hoff, self.toff, self.H, self.dh, **{**self.opts(), **kw})

    def oracle(self, grads=True):
        return O.attention(self.f["q"], self.f["k"], self.f["v"], self.hoff, self.toff, scale=self.scale, cap=self.cap,
                           edges=self.edges, bias=None if self.bias is None else self.bias.astype(np.float64),
                           masked=self.masked, tgt_pos=self.tgt_pos, hist_pos=self.hist_pos,
                           dout=self.f["dout"] if grads else None)

    def dev(self, *names):
        return [self.t[n].cuda() for n in names]

    def compare(self, got, ref):
        """got: dict of device tensors; prints and returns the worst error over its bound."""
        n = int(max(np.diff(self.hoff).max(initial=1), np.diff(self.toff).max(initial=1) * self.H // self.Hk))
        c = rel(self.dtype, self.dh, n, ref, self.cap)
        e = {}
        for name, y in got.items():
            if name == "dbias":  # a sum over every pair, fp32 whatever the storage type
                c_sum = c + 2.0 ** -24 * np.diff(self.hoff).max(initial=1) * len(self.hoff)
                e[name] = worst(y.cpu().numpy(), ref[name], ref[name + "_abs"], "f32", c_sum)
            else:
                e[name] = worst(y.double().cpu().numpy(), ref[name], ref[name + "_abs"], self.dtype, c)
        print("[attention]", {k: round(x, 3) for k, x in e.items()}, f"c={c:.1e}", flush=True)
        return e

    def step(self, plan=None):
        plan = plan or self.plan(backward=True)
        q, k, v, dout = self.dev("q", "k", "v", "dout")
        given = self.given()
        out = plan.forward(q, k, v, **given)
        dq, dk, dv, dbias = plan.backward(dout, q, k, v, **given)
        assert plan.device_status() == 0
        got = dict(out=out, dq=dq, dk=dk, dv=dv)
        if dbias is not None:
            got["dbias"] = dbias
        return got


RAGGED_L, RAGGED_M = [1, 7, 31, 32, 33, 64, 65, 0, 300, 513, 40], [1, 17, 16, 3, 0, 33, 1, 4, 15, 5, 70]
CASES = {
    "one_row": dict(L=[1], m=[1]),
    "one_target": dict(L=[1000], m=[1], nb=16),
    "ragged": dict(L=RAGGED_L, m=RAGGED_M),
    "bias": dict(L=RAGGED_L, m=RAGGED_M, nb=32, H=4),
    "mask": dict(L=RAGGED_L, m=RAGGED_M, masked=True),
    "mask_bias_cap": dict(L=RAGGED_L, m=RAGGED_M, masked=True, nb=8, cap=2.0, H=4),
    "times_any_order": dict(L=RAGGED_L, m=RAGGED_M, masked=True, nb=64, time=True),
    "many_buckets": dict(L=[600, 90], m=[20, 40], nb=128, time=True),
    "one_bucket": dict(L=[70], m=[5], nb=1),
    "shared_heads": dict(L=[40, 0, 257, 1], m=[3, 2, 18, 40], H=6, Hk=2, nb=16, masked=True, dh=64),
    "one_kv_head": dict(L=[100, 333], m=[1, 9], H=8, Hk=1, cap=5.0, dh=64),
    "wide": dict(L=[33, 200, 1], m=[20, 3, 33], dh=128, nb=8, masked=True, time=True),
    "wide_shared": dict(L=[90, 300], m=[5, 40], dh=128, H=4, Hk=2, cap=30.0),
    "peaked": dict(L=[500, 64], m=[16, 30], q_gain=12.0),
    "many_targets": dict(L=[130], m=[200], nb=16, masked=True),
    "many_requests": dict(L=[(i * 7) % 20 for i in range(200)], m=[(i * 5) % 4 for i in range(200)], nb=8, masked=True),
    "long": dict(L=[4100], m=[3], nb=32),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", list(CASES))
def test_forward_and_gradients(torch, name, dtype):
    c = Case(torch, **CASES[name], dtype=dtype)
    e = c.compare(c.step(), c.oracle())
    assert max(e.values()) <= 1.0, e


@pytest.mark.parametrize("host", [True, False])
@pytest.mark.parametrize("dtype,dh", [("bf16", 32), ("f32", 64)])
def test_forward_alone_and_without_host_offsets(torch, host, dtype, dh):
    c = Case(torch, [3000, 0, 17, 900], [3, 1, 20, 9], dtype=dtype, dh=dh, nb=16, masked=True)
    plan = c.plan(host_offsets=host)
    out = plan.forward(*c.dev("q", "k", "v"), **c.given())
    assert plan.device_status() == 0
    assert max(c.compare(dict(out=out), c.oracle(grads=False)).values()) <= 1.0
    if not host:
        assert max(c.compare(c.step(c.plan(host_offsets=False, backward=True)), c.oracle()).values()) <= 1.0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_targets_that_see_nothing(torch, dtype):
    """Every position before the history, a bias of minus infinity in every
    bucket that occurs, an empty history: output 0 and no part in a gradient."""
    c = Case(torch, [50, 80, 0], [5, 6, 3], dtype=dtype, nb=8, masked=True)
    c.tgt_pos[:5] = -7
    c.tgt_pos[7] = -1
    got = c.step()
    assert max(c.compare(got, c.oracle()).values()) <= 1.0
    for rows in (slice(0, 5), slice(7, 8), slice(11, 14)):
        assert not got["out"][rows].any() and not got["dq"][rows].any()
    assert not got["dk"][:50].any() and not got["dv"][:50].any()
    c = Case(torch, [50], [5], dtype=dtype, nb=4, bias_at={i: -np.inf for i in range(4)})
    got = c.step()
    assert not any(x.any() for x in got.values())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("low", [-np.inf, float(np.finfo(np.float32).min)])
def test_buckets_of_the_lowest_value(torch, dtype, low):
    """A bucket masked by its bias; where a target sees no other, the lowest
    value still is an ordinary (equal) score and minus infinity hides."""
    c = Case(torch, [200, 3], [9, 4], dtype=dtype, nb=6, bias_at={0: low, 3: low})
    c.tgt_pos[9:] = 2  # the short request: distances 0..2
    c.bias[:, 1] = low
    c.bias[:, 2] = low
    ref = c.oracle()
    assert max(c.compare(c.step(), ref).values()) <= 1.0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh,time", [(32, False), (64, True)])
@pytest.mark.parametrize("what", ["k", "v", "q", "dout"])
def test_odd_values_in_hidden_places(torch, dtype, dh, time, what):
    """NaN and infinities in rows that some targets may not see reach only
    those that do."""
    c = Case(torch, [90, 70], [20, 7], dtype=dtype, dh=dh, masked=True, nb=8, time=time, seed=3)
    n = c.t[what].shape[0]
    for row, x in ((1, float("nan")), (n - 2, float("nan")), (n // 2, float("inf") if what == "v" else float("nan"))):
        c.t[what][row, :, 3] = x
        c.f[what][row, :, 3] = x
    got, ref = c.step(), c.oracle()
    # (the magnitudes that bounds are relative to, of what is finite)
    for k in list(ref):
        if k.endswith("_abs"):
            ref[k] = np.nan_to_num(ref[k], nan=0.0, posinf=0.0)
    for name, y in got.items():
        y, w = y.double().cpu().numpy(), ref[name]
        fin = np.isfinite(w)
        assert np.isfinite(y[fin]).all(), f"{name}: an odd value where none is due"
        assert not np.isfinite(y[~fin]).any(), f"{name}: a finite value where an odd one is due"
        mag = np.where(fin, ref[name + "_abs"], 0.0)
        e = worst(np.where(fin, y, 0.0), np.where(fin, w, 0.0), mag, "f32" if name == "dbias" else dtype,
                  rel(dtype, dh, 400, ref, 0.0))
        assert e <= 1.0, (name, e)


def test_positions_saturate(torch):
    """Distances beyond int32 count as its ends: far in the past, or hidden."""
    c = Case(torch, [40], [4], nb=8, masked=True, time=True)
    c.hist_pos[:20] = -2 ** 31
    c.hist_pos[30:] = 2 ** 31 - 1
    c.tgt_pos[:] = [2 ** 31 - 1, -2 ** 31, 0, 5]
    assert max(c.compare(c.step(), c.oracle()).values()) <= 1.0


def test_strided_rows(torch):
    """q, k, v as slices of wider rows; the gap holds NaN."""
    c = Case(torch, RAGGED_L, RAGGED_M, nb=16, masked=True, H=4, Hk=2)
    want = c.step()
    q, k, v, dout = c.dev("q", "k", "v", "dout")
    wide_q = torch.full((q.shape[0], 4 * 32 + 24), float("nan"), dtype=q.dtype, device="cuda")
    kv = torch.full((k.shape[0], 2, 2 * 32 + 8), float("nan"), dtype=q.dtype, device="cuda")
    wide_q[:, 8:136] = q.flatten(1)
    kv[:, 0, :64], kv[:, 1, :64] = k.flatten(1), v.flatten(1)
    plan, given = c.plan(backward=True), c.given()
    args = (wide_q[:, 8:136], kv[:, 0, :64], kv[:, 1, :64])
    got = (plan.forward(*args, **given), *plan.backward(dout, *args, **given))
    for x, name in zip(got, ("out", "dq", "dk", "dv", "dbias")):
        assert torch.equal(x, want[name]), name


def test_gradients_repeat_bitwise_and_stay_inside(torch):
    """Two runs, the second through strided gradient buffers inside a pattern."""
    from paper_2511_06077_amd import stca
    c = Case(torch, RAGGED_L, RAGGED_M, nb=16, masked=True, H=4, Hk=2)
    a = c.step()
    plan, given = c.plan(backward=True), c.given()
    q, k, v, dout = c.dev("q", "k", "v", "dout")
    plan.forward(q, k, v, **given)
    big = {n: torch.full((a[n].shape[0] + 8, w), 7.0, dtype=q.dtype, device="cuda")
           for n, w in (("dq", 160), ("dk", 72), ("dv", 96))}
    db = torch.full((4 * 16 + 64,), 7.0, device="cuda")
    view = {n: x[4:-4] for n, x in big.items()}
    stca.stca_attn_backward(plan.attn, plan.batch, plan._in(q, k, v, **given), plan.saved, dout,
                            stca.attn_grads(view["dq"], view["dk"], view["dv"], 160, 72, 96, db[32:]), plan.ws,
                            plan.ws_bytes, plan.stream())
    torch.cuda.synchronize()
    for n, w in (("dq", 128), ("dk", 64), ("dv", 64)):
        assert torch.equal(view[n][:, :w].reshape(a[n].shape), a[n]), n
        assert (view[n][:, w:] == 7).all() and (big[n][:4] == 7).all() and (big[n][-4:] == 7).all(), n
    assert torch.equal(db[32:96].view(4, 16), a["dbias"]) and (db[:32] == 7).all() and (db[96:] == 7).all()


@pytest.mark.parametrize("L,m", [([0, 0], [3, 2]), ([5, 9], [0, 0]), ([4, 0], [0, 2])])
def test_empty_sides(torch, L, m):
    c = Case(torch, L, m, nb=4, masked=True)
    got = c.step()
    assert max(c.compare(got, c.oracle()).values()) <= 1.0
    assert not any(x.any() for x in got.values())


def test_other_stream_and_captured_graph(torch):
    """The step on a stream of its own, captured and replayed with other work
    between the replays, gives the eager bits."""
    c = Case(torch, [900, 33, 0, 400], [5, 40, 2, 16], nb=16, masked=True, H=4, Hk=2)
    want = c.step()
    plan, given = c.plan(backward=True), c.given()
    q, k, v, dout = c.dev("q", "k", "v", "dout")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = (plan.forward(q, k, v, **given), *plan.backward(dout, q, k, v, **given))
    side.synchronize()
    for x, n in zip(got, want):
        assert torch.equal(x, want[n]), n
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = plan.forward(q, k, v, **given)
        grads = plan.backward(dout, q, k, v, **given)
    for i in range(3):
        for t in (out, *grads):
            t.fill_(5.0)
        c.step()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for x, n in zip((out, *grads), want):
            assert torch.equal(x, want[n]), (i, n)


def test_gradients_against_differences(torch):
    """Central differences of the GPU's own forward in fp32 storage along random
    directions: the step's error is O(h^2), its rounding about 2^-24 / h."""
    c = Case(torch, [40, 9], [6, 3], dtype="f32", nb=8, masked=True, cap=4.0, time=True)
    q, k, v, dout = c.dev("q", "k", "v", "dout")
    given, plan = c.given(), c.plan(backward=True)
    got = c.step(plan)
    gen = torch.Generator(device="cuda").manual_seed(4)
    for name, x, g in (("q", q, "dq"), ("k", k, "dk"), ("v", v, "dv"), ("bias", given["bias"], "dbias")):
        d = torch.randn(x.shape, generator=gen, device="cuda")
        d /= d.norm()

        def f(s):
            at = dict(q=q, k=k, v=v, bias=given["bias"])
            at[name] = x + s * d
            y = plan.forward(at["q"], at["k"], at["v"], given["tgt_pos"], given["hist_pos"], at["bias"])
            return float((y.double() * dout.double()).sum())

        h = 2.0 ** -6
        num, ana = (f(h) - f(-h)) / (2 * h), float((got[g].double() * d.double()).sum())
        # third derivatives of f along a unit direction are below 40 for these sizes; sum |out dout| is below 600
        assert abs(num - ana) <= 40 * h * h / 6 + 600 * 2.0 ** -20 / h, (name, num, ana)


def test_bad_device_offsets_are_reported(torch):
    """Offsets that only the device can check: the status says so, no work is
    done outside the buffers and the call after it is whole."""
    from paper_2511_06077_amd import stca
    c = Case(torch, [40, 60], [3, 5])
    plan = c.plan(host_offsets=False)
    q, k, v = c.dev("q", "k", "v")
    good = plan.hoff.clone()
    plan.hoff.copy_(torch.tensor([0, 140, 100], dtype=torch.int32))
    plan.forward(q, k, v)
    assert plan.device_status() == stca.STCA_ERR_INVALID_ARG
    plan.hoff.copy_(good)
    out = plan.forward(q, k, v)
    assert plan.device_status() == 0
    assert max(c.compare(dict(out=out), c.oracle(grads=False)).values()) <= 1.0


def test_more_than_4_gib_of_rows(torch):
    """Row offsets past 2^32 bytes: the last request of a long batch is the
    same as alone."""
    H, dh, ld = 2, 32, 8192
    L = [270000, 300]
    k = torch.empty((sum(L), ld), dtype=torch.bfloat16, device="cuda")
    assert k.numel() * 2 > 2 ** 32
    c = Case(torch, [300], [7], H=H, nb=8)
    q1, k1, v1, dout = c.dev("q", "k", "v", "dout")
    want = c.step()
    k[:L[0], :2 * H * dh] = 0.25
    k[L[0]:, :H * dh], k[L[0]:, H * dh:2 * H * dh] = k1.flatten(1), v1.flatten(1)
    from paper_2511_06077_amd.attention import CrossAttention
    plan = CrossAttention(offsets(L), offsets([0, 7]), H, dh, backward=True, **{**c.opts(), "n_kv_heads": H})
    given = c.given()
    args = (q1, k[:, :H * dh], k[:, H * dh:2 * H * dh])
    out = plan.forward(*args, **given)
    dq, dk, dv, dbias = plan.backward(dout, *args, **given)
    ref = c.oracle()
    got = dict(out=out, dq=dq, dk=dk[L[0]:], dv=dv[L[0]:], dbias=dbias)
    assert max(c.compare(got, ref).values()) <= 1.0
    assert torch.equal(want["dv"].isnan(), got["dv"].isnan()) and not dk[:L[0]].any()
