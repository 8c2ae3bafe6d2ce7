"""The stand-alone attention where its work is divided otherwise than in small
batches: several kv heads a workgroup, passes whose sums wait in the workspace,
many partials, the largest tables, buckets of long distances, plans that run
side by side."""
import numpy as np
import pytest

from attn_common import offsets
from test_gpu_attention import Case, torch  # noqa: F401  (a fixture)
from test_gpu_cache import Users

pytestmark = pytest.mark.gpu


# 2^18 rows of kv heads on a card of 256 CUs are the fewest that give a
# workgroup several heads; targets choose the tiles of the backward: 1, 2 and 4.
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hk,dh,L,m", [
    (4, 32, [40000, 0, 33, 27000, 17], [9, 3, 1, 16, 5]),
    (4, 32, [40000, 0, 33, 27000, 17], [20, 3, 1, 30, 5]),
    (4, 32, [66000], [40]),
    (6, 32, [30000, 1, 20000], [7, 2, 16]),
    (4, 64, [34000, 100, 32000], [16, 40, 20]),
    (2, 128, [80000, 500, 52000], [5, 17, 12]),
])
def test_several_heads_a_workgroup(torch, Hk, dh, L, m, dtype):  # noqa: F811
    c = Case(torch, L, m, dtype=dtype, H=Hk, dh=dh, nb=16, masked=True)
    e = c.compare(c.step(), c.oracle())
    assert max(e.values()) <= 1.0, e


@pytest.mark.parametrize("dtype,dh,H,Hk,m", [("bf16", 32, 2, 2, 70), ("bf16", 64, 2, 1, 20), ("f32", 32, 4, 2, 5),
                                             ("f32", 128, 2, 1, 17), ("bf16", 128, 1, 1, 66)])
def test_passes_over_a_long_history(torch, dtype, dh, H, Hk, m):  # noqa: F811
    """More than 512 chunks of one step a wave: dk and dv of a pass wait in fp32."""
    c = Case(torch, [33000, 100], [m, 5], dtype=dtype, H=H, Hk=Hk, dh=dh, nb=8, masked=True)
    e = c.compare(c.step(), c.oracle())
    assert max(e.values()) <= 1.0, e


@pytest.mark.parametrize("dtype,dh", [("bf16", 32), ("bf16", 128), ("f32", 64), ("f32", 128)])
def test_the_largest_tables(torch, dtype, dh):  # noqa: F811
    """64 query heads of one kv head, 128 buckets."""
    c = Case(torch, [150, 0, 40], [3, 2, 18], dtype=dtype, H=64, Hk=1, dh=dh, nb=128, masked=True, time=True)
    e = c.compare(c.step(), c.oracle())
    assert max(e.values()) <= 1.0, e


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh,H,Hk,cap", [(32, 2, 2, 0.0), (64, 4, 1, 3.0), (128, 2, 2, 0.0)])
def test_a_single_visible_row_has_no_gradient(torch, dtype, dh, H, Hk, cap):  # noqa: F811
    """Its weight is 1 whatever its score: dq, dk and dbias are 0, not what
    rounding leaves of a difference; a value that is not finite still shows."""
    c = Case(torch, [1, 700, 1], [3, 18, 40], dtype=dtype, dh=dh, H=H, Hk=Hk, nb=8, masked=True, cap=cap)
    c.tgt_pos[:] = 0
    got = c.step()
    assert max(c.compare(dict(out=got["out"], dv=got["dv"]), c.oracle()).values()) <= 1.0
    assert not any(got[n].any() for n in ("dq", "dk", "dbias"))
    c.t["dout"][1, 0, 5] = float("nan")
    got = c.step()
    assert got["dq"][1, 0].isnan().all() and not got["dq"][2:].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m", [3, 16, 37, 90])
def test_infinite_scores_under_a_cap(torch, dtype, m):  # noqa: F811
    """An infinite K is the cap's end as a score: out, dv and dbias stay finite,
    also where a tile of targets is not full; dq is 0 times infinity."""
    c = Case(torch, [70, 40], [m, 2], dtype=dtype, nb=4, cap=3.0)
    c.t["q"], c.f["q"] = c.t["q"].abs(), np.abs(c.f["q"])
    for row in (5, 69):
        c.t["k"][row, 0, 7] = float("inf")
        c.f["k"][row, 0, 7] = np.inf
    with np.errstate(invalid="ignore"):
        ref = c.oracle()
    got = c.step()
    # (an infinite score has no error under the cap: the largest finite one counts)
    k = np.where(np.isfinite(c.f["k"]), np.abs(c.f["k"]), 0.0)
    score = max(float((c.scale * c.f["q"][:, h] @ k[:, h].T).max()) for h in range(2))
    assert max(c.compare({n: got[n] for n in ("out", "dv", "dbias")}, {**ref, "score": score}).values()) <= 1.0
    assert got["dq"][:m, 0, 7].isnan().all() and bool(got["dk"].isfinite().all())


def test_backward_needs_a_forward(torch):  # noqa: F811
    c = Case(torch, [9], [2])
    q, k, v, dout = c.dev("q", "k", "v", "dout")
    with pytest.raises(ValueError, match="no forward"):
        c.plan(backward=True).backward(dout, q, k, v)
    with pytest.raises(ValueError, match="without backward"):
        c.plan().backward(dout, q, k, v)


@pytest.mark.parametrize("m,H", [(1, 2), (530, 8)])
def test_many_partials(torch, m, H):  # noqa: F811
    """Partials of few rows are joined by more lanes than those of many."""
    c = Case(torch, [4500], [m], H=H, nb=8)
    plan = c.plan()
    out = plan.forward(*c.dev("q", "k", "v"), **c.given())
    assert plan.device_status() == 0
    assert max(c.compare(dict(out=out), c.oracle(grads=False)).values()) <= 1.0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("edges", [
    [1, 2, 3, 1000000, 1000001, 1000003, 2 ** 30, 2 ** 30 + 1, 2 ** 31 - 2],
    [2 ** 31 - 2], list(range(70, 190)), [16 * i + 5 for i in range(1, 120)],
])
def test_edges_close_together(torch, edges, dtype):  # noqa: F811
    """Several edges within what one cell of the look-up spans, and the ends."""
    c = Case(torch, [130, 70], [20, 33], dtype=dtype, nb=len(edges) + 1, masked=True, time=True)
    c.edges = np.asarray(edges, dtype=np.int32)
    rng = np.random.default_rng(9)
    tp = rng.integers(2 ** 30, 2 ** 31 - 1, size=len(c.tgt_pos))
    tp[0], tp[-1] = 2 ** 31 - 1, 2 ** 31 - 1
    near = rng.choice(edges, size=len(c.hist_pos)) + rng.integers(-2, 3, size=len(c.hist_pos))
    hp = rng.choice(tp, size=len(near)) - near
    hp[5], hp[-5] = 1, 2 ** 31 - 1
    c.tgt_pos, c.hist_pos = tp.astype(np.int32), np.clip(hp, -2 ** 31, 2 ** 31 - 1).astype(np.int32)
    e = c.compare(c.step(), c.oracle())
    assert max(e.values()) <= 1.0, e


def test_two_plans_at_once(torch):  # noqa: F811
    """Two plans on two streams, their launches interleaved, and graphs of both."""
    cases = [Case(torch, [900, 33, 700], [5, 40, 16], nb=16, masked=True, H=4, Hk=2, seed=s) for s in (1, 2)]
    want = [c.step() for c in cases]
    plans = [c.plan(backward=True) for c in cases]
    ins = [(c.dev("q", "k", "v", "dout"), c.given()) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = []
    for _ in range(4):
        got = []
        for p, (x, given), s in zip(plans, ins, streams):
            with torch.cuda.stream(s):
                got.append((p.forward(*x[:3], **given), *p.backward(x[3], *x[:3], **given)))
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        for x, n in zip(g, w):
            assert torch.equal(x, w[n]), n
    graphs, outs = [], []
    for p, (x, given) in zip(plans, ins):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append((p.forward(*x[:3], **given), *p.backward(x[3], *x[:3], **given)))
        graphs.append(g)
    for _ in range(3):
        for o in outs:
            for t in o:
                t.fill_(5.0)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            for x, n in zip(o, w):
                assert torch.equal(x, w[n]), n


@pytest.mark.parametrize("fmt", ["int8", "bf16"])
def test_cache_on_another_stream(torch, fmt):  # noqa: F811
    """Write, read and attend on a stream that is not the current one, and as a
    replayed graph: the same bits."""
    from paper_2511_06077_amd.attention import CacheAttention
    u = Users(torch, [300, 20, 65], [0, 7, 64], 64, fmt=fmt, gain=1.0, seed=4)
    v = Users(torch, [300, 20, 65], [0, 7, 64], 64, fmt=fmt, gain=1.0, seed=4)
    k, val, where = u.t["k"].cuda(), u.t["v"].cuda(), u.where()
    lens, q = u.dev(np.array([300, 0, 0], dtype=np.int32)), torch.randn((9, 4, 32), device="cuda").to(torch.bfloat16)
    toff = offsets([7, 1, 1])

    def step(cache, plan):
        cache.write(k, val, *where)
        return (*cache.read(*where, n_rows=385), plan.forward(q, lens, where[2]))

    a, b = (CacheAttention(x.cache, toff, 4, 300) for x in (u, v))
    want = step(u.cache, a)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step(v.cache, b)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert v.cache.device_status() == 0 and b.device_status() == 0
    v.check()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step(v.cache, b)
    for _ in range(3):
        for t in (v.cache.k, v.cache.v, *got):
            t.fill_(3)
        step(u.cache, a)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("fmt", ["int8", "bf16"])
@pytest.mark.parametrize("page,H,Hk,dh", [(16, 64, 1, 128), (64, 12, 6, 64), (32, 16, 16, 32)])
def test_cache_of_many_heads(torch, fmt, page, H, Hk, dh):  # noqa: F811
    from test_gpu_cache import serve
    u = Users(torch, [700, 33, 0, 9], [0] * 4, page, Hk=Hk, dh=dh, fmt=fmt, gain=1.0, seed=7, positions=True)
    u.write()
    plan, _, e = serve(u, torch, [1, 20, 2, 3], H, nb=128 if Hk == 1 else 12, masked=True, cap=70.0)
    assert plan.device_status() == 0 and e <= 1.0
    assert all(torch.equal(x.double().cpu(), torch.from_numpy(u.expect()[1][n]).to(torch.bfloat16).double())
               for n, x in zip(("k", "v"), u.cache.read(*u.where(), n_rows=742)))
