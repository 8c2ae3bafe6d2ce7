"""Arguments of the operators between ids, rows and gradients that are refused on
the host (nothing is launched), sizes, and the oracle's own pins; runs without a
GPU."""
import numpy as np
import pytest

from oracle import layers_oracle as O
from paper_2511_06077_amd import stca

BAD, NO, SMALL, OK = stca.STCA_ERR_INVALID_ARG, stca.STCA_ERR_UNSUPPORTED, stca.STCA_ERR_WORKSPACE, stca.STCA_OK
F32, BF16 = stca.STCA_F32, stca.STCA_BF16
INF, NAN = float("inf"), float("nan")


# ---- embedding

def field(table=0x100000, n_rows=10, ld=0, ids=0x200000):
    return table, n_rows, ld, ids


def look_up(e=None, fields=None, n=5, out=0x300000, ldo=0, ws=0x400000):
    e = e or stca.embed(64, BF16, BF16)
    return stca.stca_embed_forward(e, stca.embed_fields([field()] if fields is None else fields), n, out, ldo, ws, None,
                                   check=False)


@pytest.mark.parametrize("args,status", [
    ((0, BF16, BF16), BAD), ((-8, BF16, BF16), BAD), ((12, BF16, BF16), NO), ((8200, BF16, BF16), NO), ((64, 2, BF16), BAD),
    ((64, BF16, -1), BAD), ((64, BF16, BF16, NAN), BAD), ((64, BF16, BF16, INF), BAD)])
def test_embed_is_checked(args, status):
    assert look_up(stca.embed(*args)) == status


def test_embed_arguments():
    for kw in (dict(table=0), dict(table=0x100008), dict(ids=0), dict(ids=0x200002), dict(n_rows=0), dict(ld=63), dict(ld=68),
               dict(ld=1 << 23), dict(ld=-64)):
        assert look_up(fields=[field(), field(**kw)]) == BAD, kw
    assert look_up(fields=[field(n_rows=1 << 31)]) == NO and look_up(fields=[field()] * 9) == NO
    assert look_up(fields=[]) == BAD and look_up(n=-1) == BAD and look_up(n=1 << 31) == NO
    assert look_up(out=0) == BAD and look_up(out=0x300004) == BAD and look_up(ldo=32) == BAD and look_up(ws=0x400001) == BAD
    assert look_up(n=0, out=0, ws=0, fields=[field(ids=0)]) == OK  # (nothing to launch)


def grad(d=64, dtype=F32, n_rows=1000, scale=1.0):
    return stca.embed_grad(d, dtype, n_rows, scale)


def part(ids=0x100000, dout=0x200000, ld=0, n=50):
    return ids, dout, ld, n


def both(g=None, parts=None, **kw):
    """Status of the dense and of the sparse form, which have to agree."""
    a = dict(dtable=0x300000, ld=0, rows=0x400000, values=0x500000, count=0x600000, ws=0x700000, ws_bytes=1 << 50)
    a.update(kw)
    p = stca.embed_parts([part()] if parts is None else parts)
    g = g or grad()
    s = (stca.stca_embed_grad_dense(g, p, a["dtable"], a["ld"], False, a["ws"], a["ws_bytes"], None, check=False),
         stca.stca_embed_grad_sparse(g, p, a["rows"], a["values"], a["count"], a["ws"], a["ws_bytes"], None, check=False))
    return s


@pytest.mark.parametrize("kw,status", [
    (dict(d=0), BAD), (dict(d=20), NO), (dict(d=8200), NO), (dict(dtype=2), BAD), (dict(n_rows=0), BAD), (dict(n_rows=-5), BAD),
    (dict(n_rows=2 ** 31 - 2 ** 16 + 1), NO), (dict(scale=NAN), BAD), (dict(scale=-INF), BAD)])
def test_embed_grad_is_checked(kw, status):
    assert both(grad(**kw)) == (status, status)
    assert stca.stca_embed_grad_workspace_size(grad(**kw), 50) == 0


def test_embed_grad_arguments():
    for kw in (dict(ids=0), dict(dout=0), dict(ids=0x100001), dict(dout=0x200008), dict(ld=32), dict(ld=66), dict(n=-1)):
        assert both(parts=[part(), part(**kw)]) == (BAD, BAD), kw
    assert both(parts=[]) == (BAD, BAD) and both(parts=[part()] * 5) == (BAD, BAD)
    assert both(parts=[part(n=1 << 30)] * 2) == (NO, NO)
    assert both(ws=0) == (BAD, BAD) and both(ws=0x700008) == (BAD, BAD)
    assert both(dtable=0, rows=0) == (BAD, BAD) and both(dtable=8, values=8) == (BAD, BAD)
    assert both(ld=32, count=0) == (BAD, BAD)
    need = stca.stca_embed_grad_workspace_size(grad(), 100)
    assert both(parts=[part()] * 2, ws_bytes=need - 1) == (SMALL, SMALL)
    # a call of fewer rows never needs more than the object's workspace
    for d, dtype, rows in ((8, F32, 5), (64, BF16, 300), (256, F32, 1 << 20), (8192, BF16, 1 << 30)):
        size = [stca.stca_embed_grad_workspace_size(grad(d, dtype, rows), n) for n in
                (0, 1, 100, 4095, 4096, 4097, 4200, 8000, 20000, 99999, 100000, 3000000)]
        assert size == sorted(size) and size[0] > 0, (d, size)


# ---- norms

def norm_in(**kw):
    a = dict(x=0x100000, block=0x200000, gate=0x300000, pre_w=0x400000, pre_b=0x400100, post_w=0x400200, post_b=0x400300,
             layer_scale=0x400400)
    a.update(kw)
    return stca.norm_in(**a)


def norm(**kw):
    a = dict(d=64, dtype=BF16, kind=stca.STCA_NORM_LAYER, gate=stca.STCA_GATE_SILU, post=True, pre=True, scale=1.0, eps=1e-6)
    a.update(kw)
    return stca.norm(**a)


def norm_forward(m=None, g=None, n=5, h=0x500000, ldh=0, y=0x600000, ldy=0):
    return stca.stca_norm_forward(m or norm(), g or norm_in(), n, h, ldh, y, ldy, None, check=False)


def norm_backward(m=None, g=None, n=5, dh=0x700000, dy=0x800000, ws=0x900000, ws_bytes=1 << 50, lddh=0, lddy=0, **kw):
    a = dict(dx=0xa00000, dblock=0xb00000, dgate=0xc00000, dpre_w=0xd00000, dpost_b=0xd10000, dlayer_scale=0xd20000)
    a.update(kw)
    return stca.stca_norm_backward(m or norm(), g or norm_in(), n, dh, lddh, dy, lddy, stca.norm_grads(**a), ws, ws_bytes,
                                   None, check=False)


@pytest.mark.parametrize("kw,status", [
    (dict(d=0), BAD), (dict(d=60), NO), (dict(d=4104), NO), (dict(dtype=2), BAD), (dict(kind=2), BAD), (dict(kind=-1), BAD),
    (dict(gate=3), BAD), (dict(gate=-1), BAD), (dict(scale=INF), BAD), (dict(eps=0.0), BAD), (dict(eps=NAN), BAD),
    (dict(eps=INF), BAD), (dict(eps=-1.0), BAD)])
def test_norm_is_checked(kw, status):
    assert norm_forward(norm(**kw)) == status and norm_backward(norm(**kw)) == status
    assert stca.stca_norm_workspace_size(norm(**kw), 5) == 0


def test_norm_arguments():
    for kw in (dict(x=0), dict(x=0x100008), dict(block=0), dict(gate=0), dict(block=0x200001), dict(pre_w=0x400002),
               dict(layer_scale=0x400401), dict(ldx=32), dict(ldblock=65), dict(ldgate=1 << 23)):
        assert norm_forward(g=norm_in(**kw)) == BAD and norm_backward(g=norm_in(**kw)) == BAD, kw
    # a gate, a norm's parameters and results where the form has none
    assert norm_forward(norm(gate=0)) == BAD and norm_forward(norm(post=False)) == BAD
    assert norm_forward(norm(pre=False), y=0) == BAD and norm_forward(norm(pre=False)) == BAD
    alone = dict(block=0, gate=0, post_w=0, post_b=0, layer_scale=0)
    m = norm(gate=0, post=False)
    assert norm_forward(m, norm_in(**alone)) == BAD  # h without a block
    assert norm_forward(m, norm_in(**{**alone, "layer_scale": 0x400400}), h=0) == BAD
    assert norm_forward(norm(gate=0, post=False, pre=False), norm_in(**alone, pre_w=0, pre_b=0), h=0, y=0) == BAD
    for kw in (dict(h=0), dict(y=0), dict(h=0x500004), dict(ldh=8), dict(ldy=68), dict(n=-1)):
        assert norm_forward(**kw) == BAD, kw
    assert norm_forward(n=1 << 31) == NO
    assert norm_forward(n=0, h=0, y=0, g=norm_in(x=0, block=0, gate=0)) == OK
    for kw in (dict(dy=0), dict(dy=0x800008), dict(dh=0x700001), dict(lddy=8), dict(dx=0xa00004), dict(lddx=60), dict(ws=0),
               dict(dpre_w=0xd00002), dict(dpost_b=0xd10001)):
        assert norm_backward(**kw) == BAD, kw
    assert norm_backward(ws_bytes=stca.stca_norm_workspace_size(norm(), 5) - 1) == SMALL
    assert norm_backward(norm(pre=False), norm_in(pre_w=0, pre_b=0), dy=0, dh=0, dpre_w=0) == BAD
    # gradients of what is not there
    assert norm_backward(norm(gate=0), norm_in(gate=0)) == BAD
    assert norm_backward(norm(post=False), norm_in(post_w=0, post_b=0)) == BAD
    assert norm_backward(m, norm_in(**alone), dgate=0, dpost_b=0) == BAD
    size = [stca.stca_norm_workspace_size(norm(), n) for n in (0, 1, 100, 10000, 1 << 20, 1 << 30)]
    assert size == sorted(size) and size[0] > 0


# ---- the norm of all gradients

def clip(items, max_norm=1.0, norm_out=0x100, ws=0x200000, ws_bytes=1 << 40):
    return stca.stca_clip(stca.grads(items), max_norm, norm_out, ws, ws_bytes, None, check=False)


def g(at=0x1000000, out=0x2000000, n=100, dtype=F32, out_dtype=F32, count=0, row=0):
    return at, out or 0, n, dtype, out_dtype, count, row


def test_clip_arguments():
    for kw in (dict(at=0), dict(at=0x1000002), dict(out=0x2000001), dict(n=-1), dict(n=(1 << 40) + 1), dict(dtype=2),
               dict(out_dtype=2), dict(count=0x3000000), dict(count=0x3000000, row=33), dict(count=0x3000001, row=10),
               dict(count=0x3000000, row=-10), dict(at=0x1000001, dtype=BF16)):
        assert clip([g(0x5000000, 0x6000000), g(**kw)]) == BAD, kw
    for max_norm in (0.0, -1.0, NAN):
        assert clip([g()], max_norm) == BAD
    assert clip([g()], ws=0) == BAD and clip([g()], ws=0x200008) == BAD and clip([g()], norm_out=0x102) == BAD
    for n in (0, 1, 64, 65, 1000):
        assert clip([g()] * 0 + [g(0x10000000 + 4096 * i, None) for i in range(n)],
                    ws_bytes=stca.stca_clip_workspace_size(n) - 1) == SMALL


def test_results_of_a_clip_lie_on_nothing_else():
    a, b = 0x1000000, 0x1000000 + 400
    for items in ([g(a, b), g(b, a)],                       # exchanged
                  [g(a, a), g(a, a)],                       # the same twice
                  [g(a, a), g(a, None)],                    # ... and once more to be counted
                  [g(a, a + 4)],                            # shifted by an element
                  [g(a + 4, a)],
                  [g(a, a, dtype=BF16)],                    # the same place, another type
                  [g(a, a), g(a + 200, 0x2000000)],         # a part of another
                  [g(a, None, n=1000), g(a + 400, a + 400)],
                  [g(a + 400, a + 400), g(a, 0x2000000, n=101)],
                  [g(a, 0x2000000), g(b, 0x2000000 + 396)]):  # results on each other
        for order in (items, items[::-1]):
            assert clip(order, ws_bytes=0) == BAD, items
    for items in ([g(a, a), g(b, b)], [g(a, b), g(0x2000000, a + 800)], [g(a, None), g(a, 0x2000000)],
                  [g(a, 0x2000000), g(a, 0x3000000)], [g(0, 0, n=0), g(a, a)], [g(a, a, dtype=BF16, out_dtype=BF16)]):
        for order in (items, items[::-1]):
            assert clip(order, ws_bytes=0) == SMALL, items  # (taken, as far as the workspace)


# ---- what the Python side refuses

def test_objects_refuse():
    torch = pytest.importorskip("torch")
    from paper_2511_06077_amd.layers import BlockNorm, EmbeddingGradient, EmbeddingSum, GradientNorm
    cpu = dict(device="cpu")
    with pytest.raises(ValueError):
        EmbeddingSum((3,) * 9, 64, **cpu)
    with pytest.raises(ValueError):
        EmbeddingSum((), 64, **cpu)
    e = EmbeddingSum((3, 4), 64, dtype=torch.float32, **cpu)
    t, i = [torch.zeros(3, 64), torch.zeros(4, 64)], [torch.zeros(5, dtype=torch.int32)] * 2
    for tables, ids in ((t[:1], i), (t, i[:1]), (t[::-1], i), ([t[0].bfloat16(), t[1]], i), (t, [i[0].long(), i[1]]),
                        (t, [i[0][:3], i[1]]), (t, [i[0], i[1][::2]]), ([t[0].t().contiguous().t(), t[1]], i),
                        (t, [i[0][None], i[1]])):
        with pytest.raises(ValueError):
            e.forward(tables, ids)
    for bad in (dict(rows=0, n=5, d=64), dict(rows=5, n=5, d=63), dict(rows=5, n=-1, d=64)):
        with pytest.raises(stca.StcaError):
            EmbeddingGradient(**bad, **cpu)
    eg = EmbeddingGradient(9, 5, 64, **cpu)
    d5 = torch.zeros(5, 64)
    for parts in ([], [(i[0], d5)] * 2, [(i[0], d5[:4])], [(i[0], d5.bfloat16())], [(i[0].long(), d5)], [(i[0], d5.t())]):
        with pytest.raises(ValueError):
            eg.dense(parts)
        with pytest.raises(ValueError):
            eg.sparse(parts)
    with pytest.raises(ValueError):
        eg.dense([(i[0], d5)], accumulate=True)
    with pytest.raises(ValueError):
        eg.sparse([(i[0], d5)], out=(torch.zeros(4, dtype=torch.int32), torch.zeros(4, 64), torch.zeros(1, dtype=torch.int32)))
    for bad in (dict(kind="batch"), dict(gate="tanh"), dict(dtype=torch.float16)):
        with pytest.raises(ValueError):
            BlockNorm(64, **bad, **cpu)
    with pytest.raises(stca.StcaError):
        BlockNorm(60, **cpu)
    m, w = BlockNorm(64, gate="silu", dtype=torch.float32, **cpu), torch.ones(64)
    for kw in (dict(gate=d5), dict(post=(w,)), dict(layer_scale=w), dict(pre=False), dict(block=d5), dict(block=d5, gate=d5[:4]),
               dict(block=d5, gate=d5, pre=(w[:60],)), dict(block=d5, gate=d5, pre=(w, w, w)), dict(block=d5, gate=d5, post=(w.double(),)),
               dict(pre=(w.bfloat16(),))):
        with pytest.raises(ValueError):
            m.forward(d5, **kw)
    with pytest.raises(ValueError):
        m.backward(d5, d5)  # made without backward=True
    m = BlockNorm(64, dtype=torch.float32, backward=True, **cpu)
    for kw in (dict(dy=None), dict(dy=d5[:3]), dict(dy=d5, block=d5, pre=False), dict(dy=None, block=d5, pre=False),
               dict(dy=d5, dh=d5.bfloat16())):
        with pytest.raises(ValueError):
            m.backward(kw.pop("dy"), d5, **kw)
    for bad in (0.0, -1.0, NAN):
        with pytest.raises(ValueError):
            GradientNorm(bad, **cpu)
    c = GradientNorm(1.0, most=2, **cpu)
    for kw in (dict(grads=[w] * 3), dict(grads=[w], out=[]), dict(grads=[w], counts=[None, None]), dict(grads=[d5.t()]),
               dict(grads=[w], out=[torch.ones(63)]), dict(grads=[w.half()]), dict(grads=[d5], counts=[torch.ones(1)]),
               dict(grads=[torch.tensor(1.0)], counts=[torch.ones(1, dtype=torch.int32)])):
        with pytest.raises(ValueError):
            c.clip(**kw)
    # nothing is wrong with the arguments, but the tensors are the host's
    for call in (lambda: c.clip([w]), lambda: m.forward(d5), lambda: e.forward(t, i), lambda: eg.dense([(i[0], d5)])):
        with pytest.raises(ValueError, match="GPU"):
            call()


# ---- the oracle

def test_oracle_embedding():
    rng = np.random.default_rng(0)
    t, ids = rng.standard_normal((7, 4)), np.array([3, -1, 6, 3, 9])
    out, mag = O.embed([t, t], [ids, ids[::-1]], 2.0)
    one = np.zeros((5, 7))
    one[[0, 2, 3], [3, 6, 3]] = 1
    both_hot = one + one[::-1]
    assert np.allclose(out, 2 * both_hot @ t) and np.allclose(mag, 2 * both_hot @ np.abs(t))
    g = rng.standard_normal((5, 4))
    rows, dt, _, k = O.embed_grad([(ids[:2], g[:2]), (ids[2:], g[2:])], 7, 2.0)
    assert rows.tolist() == [3, 6] and k.tolist() == [2, 1] and np.allclose(dt, 2 * (one.T @ g)[[3, 6]])


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("act", [None, "sigmoid", "silu"])
@pytest.mark.parametrize("post", [True, False])
def test_oracle_norm(kind, act, post):
    """Against automatic differentiation in float64."""
    torch = pytest.importorskip("torch")
    rng = np.random.default_rng(3)
    n, d, eps, scale = 6, 24, 1e-3, 0.7
    names = ["x", "block"] + (["gate"] if act else [])
    a = {k: rng.standard_normal((n, d)) * 3 for k in names + ["dy", "dh"]}
    p = {k: rng.standard_normal(d) for k in ("pre_w", "pre_b", "post_w", "post_b", "ls")}
    ref = O.norm(a["x"], kind, eps, scale, a["block"], a.get("gate"), act, pre=(p["pre_w"], p["pre_b"]),
                 post=(p["post_w"], p["post_b"]) if post else None, ls=p["ls"], dy=a["dy"], dh=a["dh"])
    t = {k: torch.from_numpy(v).requires_grad_() for k, v in {**a, **p}.items()}
    def unit(v):
        if kind == "layer":
            return torch.nn.functional.layer_norm(v, (d,), eps=eps)
        return v * torch.rsqrt((v * v).mean(1, keepdim=True) + eps)
    o = unit(t["block"]) * t["post_w"] + t["post_b"] if post else t["block"]
    if act:
        o = o * (torch.sigmoid(t["gate"]) if act == "sigmoid" else torch.nn.functional.silu(t["gate"]))
    h = t["x"] + scale * t["ls"] * o
    y = unit(h) * t["pre_w"] + t["pre_b"]
    ((h * t["dh"].detach()).sum() + (y * t["dy"].detach()).sum()).backward()
    assert np.allclose(ref["h"], h.detach().numpy(), rtol=1e-12) and np.allclose(ref["y"], y.detach().numpy(), rtol=1e-10)
    want = dict(dx="x", dblock="block", pre_w="pre_w", pre_b="pre_b", ls="ls")
    want.update(dict(dgate="gate") if act else {}, **(dict(post_w="post_w", post_b="post_b") if post else {}))
    for k, name in want.items():
        assert np.allclose(ref[k], t[name].grad.numpy(), rtol=1e-9, atol=1e-11), k


def test_oracle_norm_alone():
    """A row of equal values, whose layer norm is the bias, and an rms norm's length."""
    r = O.norm(np.full((2, 8), 3.0), "layer", 1e-6, 1.0, pre=(np.arange(8.0), np.arange(8.0)))
    assert np.array_equal(r["y"], np.tile(np.arange(8.0), (2, 1)))
    r = O.norm(np.array([[3.0, 4.0] * 4]), "rms", 0.0, 1.0)
    assert np.allclose(r["y"], np.array([[3.0, 4.0] * 4]) / np.sqrt(12.5))


def test_oracle_clip():
    norm, f = O.clip([np.array([3.0]), np.array([[4.0, 0.0]])], 1.0)
    assert norm == 5.0 and f == 0.2
    assert O.clip([np.array([3.0])], 3.0)[1] == 1.0 and O.clip([np.array([np.inf])], 3.0)[1] == 1.0


@pytest.mark.parametrize("n,d", [(1, 8), (700, 64), (20000, 32), (2500, 1024), (41001, 520), (200000, 4096), (1500000, 72)])
def test_oracle_bounds_the_sums_over_rows(n, d):
    """A norm's sums of [d] as they are divided: a lane's rows one after the other, a
    workgroup's lanes, then fp64; with terms that are lost beside the first one of a lane."""
    cus, lanes = 256, max(8, 1 << (d // 8 - 1).bit_length())
    teams = 256 // lanes if lanes <= 64 else 1
    groups = min(-(-n // teams), 2 * cus)
    turn = groups * teams
    terms = np.full(-(-n // turn) * turn, 2.0 ** -24, dtype=np.float32)
    terms[:turn], terms[n:] = 1.0, 0.0
    lane = np.zeros(turn, dtype=np.float32)
    for k in range(0, len(terms), turn):
        lane += terms[k:k + turn]
    group = np.zeros(groups, dtype=np.float32)
    for k in range(teams):
        group += lane.reshape(groups, teams)[:, k]
    got, want = float(np.float32(group.sum(dtype=np.float64))), float(terms.sum(dtype=np.float64))
    assert abs(got - want) <= (O.sum_depth(n, d) + 1) * O.U * want
