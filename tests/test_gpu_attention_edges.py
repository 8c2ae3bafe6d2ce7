"""The stand-alone attention at the ends of what its calls allow: device offsets
that are not the host's, the largest tables and values, what is left of weights."""
import numpy as np
import pytest

import attn_common
from attn_common import offsets
from test_gpu_attention import Case, torch  # noqa: F401  (a fixture)
from test_gpu_guards import Guarded

pytestmark = pytest.mark.gpu


# Host lengths of one chunk (no partials) and of several, one pass over the
# targets and several; the device copies show a longer request, or one of more
# targets.  What the launches were planned for takes more rows than the host's
# longest request where chunks end later, and any number of targets forward.
@pytest.mark.parametrize("dtype,dh,H,Hk", [("bf16", 32, 2, 2), ("bf16", 64, 4, 1), ("f32", 32, 2, 2)])
@pytest.mark.parametrize("L,m,dev_L,dev_m,forward,backward", [
    ([50, 50], [3, 6], [90, 10], [3, 6], False, False),
    ([50, 50], [3, 6], [100, 0], [9, 0], False, False),
    ([40000, 40000], [2, 2], [79990, 10], [2, 2], False, False),
    ([50, 50], [3, 6], [60, 40], [6, 3], True, True),
    ([50, 50], [16, 16], [50, 50], [32, 0], True, None),  # (shared heads go in several passes, any number of them)
    ([5000] + [40] * 30, [2] * 31, [5000] + [40] * 30, [2] * 29 + [4, 0], False, False),  # (partials by unit)
])
def test_stale_host_offsets(torch, dtype, dh, H, Hk, L, m, dev_L, dev_m, forward, backward):  # noqa: F811
    """Nothing is written outside the buffers, and a request that was not taken
    whole is reported."""
    from paper_2511_06077_amd import stca
    c = Case(torch, dev_L, dev_m, dtype=dtype, dh=dh, H=H, Hk=Hk, nb=4, masked=True)  # what the device's offsets say
    c.hoff, c.toff = offsets(L), offsets(m)
    plan = c.plan(backward=True)
    plan.hoff.copy_(torch.from_numpy(offsets(dev_L)))
    plan.toff.copy_(torch.from_numpy(offsets(dev_m)))
    q, k, v, dout = c.dev("q", "k", "v", "dout")
    places = c.given()
    given = plan._in(q, k, v, **places)
    es = q.element_size()
    size = dict(out=q.numel() * es, saved=plan.saved.numel(), dq=q.numel() * es, dk=k.numel() * es, dv=v.numel() * es,
                dbias=4 * H * 4)
    fwd_ws = stca.stca_attn_workspace_size(plan.attn, plan.batch, False)
    bwd_ws = stca.stca_attn_workspace_size(plan.attn, plan.batch, True)
    backward = H != Hk if backward is None else backward
    status = {True: stca.STCA_OK, False: stca.STCA_ERR_INVALID_ARG}
    g = {n: Guarded(torch, x) for n, x in size.items()}
    ws = Guarded(torch, fwd_ws)
    stca.stca_attn_forward(plan.attn, plan.batch, given, g["out"].ptr, g["saved"].ptr, ws.ptr, fwd_ws, plan.stream())
    got = stca.stca_device_status(ws.ptr, plan.stream())
    assert ws.intact() and all(x.intact() for x in g.values())
    assert got == status[forward]
    ws = Guarded(torch, bwd_ws)
    stca.stca_attn_backward(plan.attn, plan.batch, given, g["saved"].ptr, dout,
                            stca.attn_grads(*(g[n].ptr for n in ("dq", "dk", "dv")), dbias=g["dbias"].ptr), ws.ptr,
                            bwd_ws, plan.stream())
    got = stca.stca_device_status(ws.ptr, plan.stream())
    assert ws.intact() and all(x.intact() for x in g.values())
    assert got == status[backward]
    # what was taken whole is right
    c.hoff, c.toff = offsets(dev_L), offsets(dev_m)
    ref = c.oracle()
    if forward:
        e = c.compare(dict(out=g["out"].view(torch, q.dtype, q.shape)), ref)
        assert max(e.values()) <= 1.0, e
    if backward:
        e = c.compare(dict(dq=g["dq"].view(torch, q.dtype, q.shape), dk=g["dk"].view(torch, q.dtype, k.shape),
                           dv=g["dv"].view(torch, q.dtype, v.shape),
                           dbias=g["dbias"].view(torch, torch.float32, (H, 4))), ref)
        assert max(e.values()) <= 1.0, e


def some_heads(c, heads):
    """The case with the given query heads of each kv head's group alone."""
    import copy
    G = c.H // c.Hk
    pick = [g * G + h for g in range(c.Hk) for h in heads]
    s = copy.copy(c)
    s.f = {n: x[:, pick] if n in ("q", "dout") else x for n, x in c.f.items()}
    s.H, s.bias = len(pick), c.bias[pick]
    return s, pick


@pytest.mark.parametrize("dh,G,nb", [(32, 2, 16), (128, 64, 128), (128, 32, 128)])
def test_tables_of_several_heads_a_workgroup(torch, dh, G, nb):  # noqa: F811
    """Four kv heads a workgroup where their groups' biases fit the LDS, else
    fewer; forward, the first and the last head of every group."""
    c = Case(torch, [40000, 0, 33, 26000], [2, 3, 1, 2], H=4 * G, Hk=4, dh=dh, nb=nb, masked=True)
    plan = c.plan()
    out = plan.forward(*c.dev("q", "k", "v"), **c.given())
    assert plan.device_status() == 0
    s, pick = some_heads(c, (0, G - 1))
    e = s.compare(dict(out=out[:, pick]), s.oracle(grads=False))
    assert max(e.values()) <= 1.0, e


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_largest_tables_without_targets(torch, dtype):  # noqa: F811
    c = Case(torch, [60000, 6000], [0, 0], H=256, Hk=4, dh=128, nb=128, dtype=dtype)
    got = c.step()
    assert not any(x.any() for x in got.values())


def balanced(plus, minus):
    """An order of len(plus) + len(minus) terms whose running sum stays small:
    indices of plus, and len(plus) + those of minus."""
    order, total, i, j = [], 0.0, 0, 0
    while i < len(plus) or j < len(minus):
        if j == len(minus) or (i < len(plus) and total <= 0):
            order.append(i)
            total += plus[i]
            i += 1
        else:
            order.append(len(plus) + j)
            total -= minus[j]
            j += 1
    return np.array(order)


# What two bf16 terms leave of a weight may lie on either side of it.  N weights
# whose low bits are spread evenly, against exact ones (1, or 1/2) of the other
# sign: what is left of the N adds up to no more than Hoeffding's bound for N
# values within +-2^-16 of their power of two (chance 1e-9), beside 6e-7 of each
# for exp2, the sum and its reciprocal (some ulps); cut to one side it is N 2^-16
# of that power of two at the mean, four times as much.
N_LOW = 4096
HOEFFDING = np.sqrt(N_LOW * np.log(2e9) / 2)


def test_weights_are_not_low_forward(torch):  # noqa: F811
    rng = np.random.default_rng(0)
    c = Case(torch, [1], [1], H=1, Hk=1)
    k = np.zeros((N_LOW, 32))
    k[:, :2] = torch.from_numpy(-rng.uniform(0.01, 0.68, size=(N_LOW, 2))).to(torch.bfloat16).double().numpy()
    q = np.zeros((1, 1, 32))
    q[0, 0, :2] = 1.0, 2.0 ** -8
    w = np.exp(k @ q[0, 0])  # within 1/2 .. 1
    ones = int(round(w.sum()))
    at = balanced(np.ones(ones), w)
    k = np.concatenate([np.zeros((ones, 32)), k])[at]
    v = np.concatenate([np.ones(ones), -np.ones(N_LOW)])[at][:, None] * np.ones(32)
    c.hoff, c.toff, c.scale = offsets([len(at)]), offsets([1]), 1.0
    for n, x in (("q", q), ("k", k[:, None]), ("v", v[:, None])):
        c.f[n], c.t[n] = x, torch.from_numpy(x).to(torch.bfloat16)
        assert np.array_equal(c.t[n].double().numpy(), x)
    out = c.plan().forward(*c.dev("q", "k", "v")).double().cpu().numpy()[0, 0]
    want, total = (ones - w.sum()) / (ones + w.sum()), ones + w.sum()
    bound = (HOEFFDING * 2.0 ** -16 + 6e-7 * total) / total + 2.0 ** -8 * abs(want)
    print("[low]", np.abs(out - want).max() / bound)
    assert (np.abs(out - want) <= bound).all()


def test_weights_are_not_low_backward(torch):  # noqa: F811
    rng = np.random.default_rng(1)
    q = np.zeros((N_LOW, 1, 32))
    q[:, 0, :2] = torch.from_numpy(rng.uniform(0.01, 1.0, size=(N_LOW, 2))).to(torch.bfloat16).double().numpy()
    k = np.zeros((2, 1, 32))
    k[1, 0, :2] = 1.0, 2.0 ** -8
    w = 1 / (1 + np.exp(q[:, 0] @ k[1, 0]))  # of row 0: within 1/4 .. 1/2
    halves = int(round(2 * w.sum()))
    at = balanced(np.full(halves, 0.5), w)
    q = np.concatenate([np.zeros((halves, 1, 32)), q])[at]
    dout = np.concatenate([np.ones(halves), -np.ones(N_LOW)])[at][:, None, None] * np.ones((1, 1, 32))
    c = Case(torch, [2], [len(at)], H=1, Hk=1)
    c.scale = 1.0
    for n, x in (("q", q), ("k", k), ("dout", dout)):
        c.f[n], c.t[n] = x, torch.from_numpy(x).to(torch.bfloat16)
        assert np.array_equal(c.t[n].double().numpy(), x)
    dv = c.step()["dv"][0, 0].double().cpu().numpy()
    want = 0.5 * halves - w.sum()
    bound = HOEFFDING * 2.0 ** -17 + 6e-7 * 0.5 * len(at) + 2.0 ** -8 * abs(want)
    print("[low]", np.abs(dv - want).max() / bound)
    assert (np.abs(dv - want) <= bound).all()


# The largest V of the types: equal signs and nearly equal scores, so that every
# sum before the division is the number of rows times larger.  (Rows are taken a
# second time, with scores up to 8 + log2(rows) < 26 from their maximum: 26 u of a
# weight, which the bounds' 2 (rows + ..) u hold many times over.)
TOP = 3.3e38


def large(torch, c, dtype):  # noqa: F811
    from attn_common import rounded
    rng = np.random.default_rng(5)
    v = TOP * rng.uniform(0.5, 1.0, size=c.f["v"].shape)
    return rounded(torch, v, dtype)


@pytest.mark.parametrize("L,m", [([5000, 40, 1, 0], [3, 20, 2, 1]), ([300, 2000], [33, 5]), ([70000], [2])])
@pytest.mark.parametrize("dtype,dh,H,Hk,masked", [("bf16", 32, 4, 4, True), ("bf16", 64, 2, 1, False),
                                                  ("bf16", 128, 2, 2, False), ("f32", 32, 4, 4, False), ("f32", 64, 2, 2, True)])
def test_the_largest_values(torch, dtype, dh, H, Hk, masked, L, m):  # noqa: F811
    c = Case(torch, L, m, dtype=dtype, dh=dh, H=H, Hk=Hk, masked=masked, nb=8 if masked else 0, q_gain=0.1)
    c.t["v"], c.f["v"] = large(torch, c, dtype)
    c.t["dout"], c.f["dout"] = c.t["dout"] * 2.0 ** -90, c.f["dout"] * 2.0 ** -90
    ref = c.oracle()
    e = c.compare(dict(out=c.plan().forward(*c.dev("q", "k", "v"), **c.given())), ref)
    assert max(e.values()) <= 1.0, e
    e = c.compare(c.step(), ref)
    assert max(e.values()) <= 1.0, e


@pytest.mark.parametrize("fmt", ["int8", "bf16"])
@pytest.mark.parametrize("page,dh,m,H", [(16, 32, [1, 20, 2, 1], 2), (64, 64, [3, 1, 9, 1], 8), (256, 128, [2, 30, 1, 1], 2)])
def test_the_largest_values_cached(torch, fmt, page, dh, m, H):  # noqa: F811
    from test_gpu_cache import Users, serve
    u = Users(torch, [6000, 300, 1, 0], [0] * 4, page, dh=dh, fmt=fmt, gain=1.0)
    u.t["v"], u.f["v"] = large(torch, u, "bf16")
    u.write()
    plan, _, e = serve(u, torch, m, H, nb=8, masked=True, q_gain=0.1)
    assert plan.device_status() == 0 and e <= 1.0


# Partials by the chunk and target of each request, where one history is much
# longer than the others; and longer chunks where one request has most of the
# targets as well (the 64 MB that are always taken are passed by 8 heads of 128).
@pytest.mark.parametrize("dtype,dh,H,Hk,L,m", [
    ("bf16", 32, 2, 2, [40] * 30 + [5000, 0] + [40] * 20, [2] * 52),
    ("bf16", 64, 4, 1, [40] * 30 + [5000, 0] + [40] * 20, [i % 4 for i in range(52)]),
    ("f32", 32, 2, 2, [3000] + [7] * 60, [3] * 61),
    ("bf16", 128, 8, 4, [20] * 500 + [5000], [3, 60] + [3] * 499),
    ("f32", 128, 8, 4, [5000] + [20] * 500, [3, 60] + [3] * 499),
])
def test_one_long_history_among_short_ones(torch, dtype, dh, H, Hk, L, m):  # noqa: F811
    c = Case(torch, L, m, dtype=dtype, dh=dh, H=H, Hk=Hk, nb=8, masked=True)
    ref = c.oracle()
    plan = c.plan()
    e = c.compare(dict(out=plan.forward(*c.dev("q", "k", "v"), **c.given())), ref)
    assert plan.device_status() == 0 and max(e.values()) <= 1.0, e
    e = c.compare(c.step(), ref)
    assert max(e.values()) <= 1.0, e


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nb", [34, 35, 70, 71, 128])
def test_lanes_that_share_a_bucket_sum(torch, nb, dtype):  # noqa: F811
    """Up to 34 buckets every lane has sums of its own, up to 70 two lanes share
    one, above four; every row of a step in a bucket of its own or all in one, so
    that the sharing lanes meet; the same bits each time."""
    c = Case(torch, [400, 90], [40, 7], H=4, Hk=2, dtype=dtype, nb=nb, masked=True, time=True, seed=nb)
    c.edges = np.arange(1, nb, dtype=np.int32)
    c.hist_pos[200:400] = 50
    ref = c.oracle()
    got = [c.step() for _ in range(3)]
    e = c.compare(got[0], ref)
    assert max(e.values()) <= 1.0, e
    for g in got[1:]:
        assert torch.equal(g["dbias"], got[0]["dbias"])


def test_results_of_a_given_stream(torch):  # noqa: F811
    """A call with stream= takes no memory that the current stream has freed but
    still uses; its results are those of the current stream."""
    from paper_2511_06077_amd.attention import CacheAttention
    from test_gpu_cache import Users
    c = Case(torch, [900, 33, 0, 400], [50, 40, 2, 16], nb=16, masked=True, H=4, Hk=2)
    want = c.step()
    plan, given = c.plan(backward=True), c.given()
    q, k, v, dout = c.dev("q", "k", "v", "dout")
    u = Users(torch, [300, 20, 65], [0, 0, 0], 64, gain=1.0)
    u.write()
    cq, lens, table = torch.randn((9, 4, 32), device="cuda").bfloat16(), u.dev(u.n.astype(np.int32)), u.dev(u.table)
    serve = CacheAttention(u.cache, offsets([7, 1, 1]), 4, 300)
    where = u.where()
    cached = (serve.forward(cq, lens, table), *u.cache.read(*where, n_rows=385))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    calls = (
        (lambda s: [plan.forward(q, k, v, **given, stream=s)], [want["out"]]),
        (lambda s: plan.backward(dout, q, k, v, **given, stream=s), [want[n] for n in ("dq", "dk", "dv", "dbias")]),
        (lambda s: [serve.forward(cq, lens, table, stream=s)], [cached[0]]),
        (lambda s: u.cache.read(*where, n_rows=385, stream=s), cached[1:]))
    for call, expect in calls:
        held = [torch.full_like(x, 7.0) for x in expect]
        seen = [torch.empty_like(x) for x in expect]
        torch.cuda.synchronize()
        torch.cuda._sleep(50_000_000)  # the current stream is behind
        for a, b in zip(seen, held):
            a.copy_(b)
        del b
        held.clear()  # freed, and still to be read
        got = call(side.cuda_stream)
        side.synchronize()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, expect))
        assert all((x == 7.0).all() for x in seen)
    assert plan.device_status(side.cuda_stream) == 0 and u.cache.device_status(side.cuda_stream) == 0


def test_gradients_of_a_given_stream(torch):  # noqa: F811
    """The layer stack's gradients likewise."""
    from paper_2511_06077_amd import workload as W
    from paper_2511_06077_amd.device import DeviceBatch, to_device
    b = W.make_custom_batch("stream", [300, 45, 1], [5, 33, 2], d_model=128, n_heads=4, n_layers=1, dtype="bf16", seed=7,
                            with_grad=True)
    db = DeviceBatch(b, backward=True)
    dout = to_device(b.grad_out, "cuda")
    want = db.backward(dout)
    side = torch.cuda.Stream()
    held = [torch.full_like(x, 7.0) for x in want.values()]
    seen = [torch.empty_like(x) for x in held]
    torch.cuda.synchronize()
    torch.cuda._sleep(50_000_000)
    for x, y in zip(seen, held):
        x.copy_(y)
    del y
    held.clear()
    got = db.backward(dout, stream=side.cuda_stream)
    side.synchronize()
    torch.cuda.synchronize()
    assert all(torch.equal(got[n], want[n]) for n in want)
    assert all((x == 7.0).all() for x in seen)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cap", [1e4, 1e30])
def test_a_cap_far_above_the_scores(torch, cap, dtype):  # noqa: F811
    """tanh is relative to small values there: the results of no cap (at 1e4 what
    it takes off, x^3 / (3 cap^2), is about 2^-23 of a score)."""
    c = Case(torch, [200, 33], [9, 20], dtype=dtype, nb=8, masked=True)
    ref = c.oracle()
    c.cap = cap
    got = c.step()
    c.cap = 0.0
    e = c.compare(got, ref)
    assert max(e.values()) <= 1.0, e


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hk,dh,L,m", attn_common.SPREAD)
def test_every_block_of_a_long_history(torch, Hk, dh, L, m, dtype):  # noqa: F811
    """Several kv heads a workgroup, with bounds that a lost block exceeds."""
    c = Case(torch, L, m, dtype=dtype, H=Hk, dh=dh, masked=True)
    f, opts = attn_common.spread(np.random.default_rng(7), L, m, Hk, Hk, dh)
    for n, x in f.items():
        c.t[n], c.f[n] = attn_common.rounded(torch, x, dtype)
    c.scale, c.edges, c.bias, c.tgt_pos = 1.0, opts["edges"], opts["bias"], opts["tgt_pos"]
    ref, got = c.oracle(), c.step()
    bound = attn_common.deep(dtype, dh, L, ref)
    e = {n: attn_common.worst(x.double().cpu().numpy(), ref[n], ref[n + "_abs"], "f32" if n == "dbias" else dtype, bound)
         for n, x in got.items()}
    print("[spread]", {n: round(x, 3) for n, x in e.items()}, f"c={bound:.1e}", flush=True)
    assert max(e.values()) <= 1.0, e


@pytest.mark.parametrize("page,dh,H,nb", [(16, 32, 4, 8), (64, 64, 8, 0), (128, 128, 2, 16)])
def test_eight_bit_rows_of_many_steps(torch, page, dh, H, nb):  # noqa: F811
    """K rows from 2^-12 to 2 and V rows from 2^-20 to 2^20: neighbours in a block
    have steps of their own, and the largest rows' do not spill into the others."""
    from test_gpu_cache import Users, serve
    u = Users(torch, [1500, 70, 33, 1], [0] * 4, page, dh=dh, gain=1.0, seed=8)
    rng = np.random.default_rng(3)
    for n, lo, hi in (("k", -12, 2), ("v", -20, 21)):
        f = 2.0 ** rng.integers(lo, hi, size=u.f[n].shape[:2])[..., None]
        u.f[n] = u.f[n] * f
        u.t[n] = torch.from_numpy(u.f[n]).to(torch.bfloat16)
        assert np.array_equal(u.t[n].double().numpy(), u.f[n])
    u.write()
    plan, _, e = serve(u, torch, [3, 20, 1, 2], H, nb=nb, masked=nb > 0, cap=20.0 if nb == 16 else 0.0)
    assert plan.device_status() == 0 and e <= 1.0
