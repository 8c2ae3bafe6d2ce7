"""Arguments of the stand-alone attention and the cache that are refused on the
host (nothing is launched), sizes, bucket edges and the oracle's own pins; runs
without a GPU."""
import ctypes

import numpy as np
import pytest

import attn_common
from oracle import attn_oracle as O
from paper_2511_06077_amd import stca

BAD, NO, SMALL = stca.STCA_ERR_INVALID_ARG, stca.STCA_ERR_UNSUPPORTED, stca.STCA_ERR_WORKSPACE
EDGES = np.array([1, 2, 4, 8, 16, 32, 64], dtype=np.int32)


def attn(**kw):
    a = dict(n_heads=8, n_kv_heads=4, d_head=32, dtype=stca.STCA_BF16, scale=0.2, softcap=0.0, masked=True,
             n_buckets=8, edges=EDGES)
    a.update(kw)
    return stca.attn(**a)


def batch(h=(0, 40, 100), t=(0, 3, 9), host=True):
    h, t = np.asarray(h, dtype=np.int32), np.asarray(t, dtype=np.int32)
    b = stca.batch(len(h) - 1, int(h[-1]), int(t[-1]), 0x10000, 0x20000, h if host else None, t if host else None)
    b.keep = (h, t)
    return b


def given(**kw):
    a = dict(q=0x100000, k=0x200000, v=0x300000, tgt_pos=0x400000, hist_pos=None, bias=0x500000)
    a.update(kw)
    return stca.attn_in(**a)


def forward(a=None, b=None, g=None, out=0x600000, ws=0x700000, ws_bytes=1 << 40):
    return stca.stca_attn_forward(a or attn(), b or batch(), g or given(), out, None, ws, ws_bytes, None, check=False)


@pytest.mark.parametrize("kw,status", [
    (dict(n_heads=7), BAD), (dict(n_kv_heads=0), BAD), (dict(n_heads=0), BAD), (dict(dtype=3), BAD),
    (dict(scale=float("nan")), BAD), (dict(scale=float("inf")), BAD), (dict(softcap=-1.0), BAD),
    (dict(softcap=float("nan")), BAD), (dict(n_buckets=129), BAD), (dict(n_buckets=-1), BAD), (dict(edges=None), BAD),
    (dict(edges=EDGES[::-1].copy()), BAD), (dict(edges=EDGES * 0 + 1), BAD), (dict(edges=EDGES - 1), BAD), (dict(edges=np.r_[EDGES[:6], 2 ** 31 - 1].astype(np.int32)), BAD),
    (dict(d_head=48), NO), (dict(d_head=256), NO), (dict(d_head=16), NO), (dict(n_heads=65, n_kv_heads=1), NO),
    (dict(n_heads=1024, n_kv_heads=1024, d_head=128), NO)])
def test_scores_are_checked(kw, status):
    a = attn(**kw)
    assert forward(a) == status
    assert stca.stca_attn_workspace_size(a, batch()) == 0
    assert stca.stca_attn_saved_size(a, batch()) == 0


@pytest.mark.parametrize("kw", [
    dict(softcap=3e38), dict(scale=-3e38), dict(scale=1e-3, softcap=1e37), dict(scale=1e20, softcap=1e-20),
    dict(scale=1e-38, softcap=100.0)])
def test_factors_of_a_score_have_to_fit_fp32(kw):
    """Finite, but softcap log2 e is infinite, or scale / softcap is not a normal
    number: scores would be NaN, or lose their bits."""
    assert forward(attn(**kw)) == BAD and stca.stca_attn_workspace_size(attn(**kw), batch()) == 0
    for ok in (dict(softcap=1e30), dict(scale=0.0, softcap=5.0), dict(scale=-1e30), dict(scale=1e-30, softcap=1.0),
               dict(scale=2e38), dict(scale=0.1, softcap=1e-30)):
        assert stca.stca_attn_workspace_size(attn(**ok), batch()) > 0, ok


@pytest.mark.parametrize("h,t", [([0, 5, 3], [0, 1, 2]), ([1, 5, 6], [0, 1, 2]), ([0, 5, 6], [0, 3, 2])])
def test_host_offsets_are_checked(h, t):
    assert forward(b=batch(h, t)) == BAD


def test_pointers_strides_and_sizes_are_checked():
    for kw in (dict(q=0), dict(k=0), dict(v=0), dict(q=0x100008), dict(k=0x200002), dict(tgt_pos=0), dict(bias=0),
               dict(tgt_pos=0x400002), dict(bias=0x500001), dict(ldq=8), dict(ldq=260), dict(ldk=127), dict(ldv=1 << 23),
               dict(ldk=-128)):
        assert forward(g=given(**kw)) == BAD, kw
    assert forward(out=0) == BAD and forward(out=0x600008) == BAD and forward(ws=0) == BAD
    need = stca.stca_attn_workspace_size(attn(), batch())
    assert need > 0 and forward(ws_bytes=need - 1) == SMALL
    b = batch()
    b.n_requests = 0
    assert forward(b=b) == BAD
    b = batch(host=False)
    b.n_hist = 0x7fffffff
    assert forward(b=b) == NO


def test_backward_arguments_are_checked():
    def call(dout=0x800000, saved=0x900000, ws_bytes=1 << 40, **kw):
        g = dict(dq=0xa00000, dk=0xb00000, dv=0xc00000, dbias=0xd00000)
        g.update(kw)
        return stca.stca_attn_backward(attn(), batch(), given(), saved, dout, stca.attn_grads(**g), 0x700000, ws_bytes,
                                       None, check=False)
    for kw in (dict(dout=0), dict(dout=0x800008), dict(saved=0), dict(dq=0), dict(dk=0), dict(dv=0), dict(dbias=0),
               dict(dk=0xb00004), dict(lddq=16), dict(lddk=129)):
        assert call(**kw) == BAD, kw
    assert call(ws_bytes=stca.stca_attn_workspace_size(attn(), batch(), True) - 1) == SMALL


def test_saved_layout_and_workspace():
    a, b = attn(), batch()
    lay = stca.stca_attn_saved_layout(a, b)
    rows = 9 * 8
    assert lay.max >= lay.a + 4 * rows * 32 and lay.sum >= lay.max + 4 * rows and lay.total >= lay.sum + 4 * rows
    assert lay.total == stca.stca_attn_saved_size(a, b)
    # a long history is split and its parts are kept; a split that the host cannot see is bounded
    long = batch([0, 100000], [0, 9])
    assert stca.stca_attn_workspace_size(a, long) > 4 * rows * 32 * 10
    assert stca.stca_attn_workspace_size(a, batch([0, 100000], [0, 9], host=False)) <= 4 * rows * 35 * 17 + 4096


def cache(**kw):
    a = dict(n_pages=10, page_size=64, n_kv_heads=4, d_head=32, fmt=stca.STCA_CACHE_INT8, k=0x1000000, v=0x2000000,
             k_exp=0x3000000, v_exp=0x4000000, pos=None)
    a.update(kw)
    return stca.cache(**a)


def rows(**kw):
    a = dict(n_requests=2, n_rows=5, row_off=0x10000, start=0x20000, table=0x30000, table_ld=3)
    a.update(kw)
    return stca.cache_rows(**a)


@pytest.mark.parametrize("kw,status", [
    (dict(n_pages=0), BAD), (dict(fmt=2), BAD), (dict(k=0), BAD), (dict(v=0x2000008), BAD), (dict(k_exp=0), BAD),
    (dict(v_exp=0), BAD), (dict(pos=0x5000002), BAD), (dict(page_size=48), NO), (dict(page_size=8), NO),
    (dict(page_size=512), NO), (dict(d_head=40), NO)])
def test_cache_is_checked(kw, status):
    c = cache(**kw)
    for f in (stca.stca_cache_write, stca.stca_cache_read):
        assert f(c, rows(), stca.STCA_BF16, 0x6000000, 0x7000000, check=False) == status
    b = stca.cache_batch(2, 9, 0x10000, 0x20000, 100, 0x30000, 2)
    assert stca.stca_cache_attn(attn(), c, b, 0x6000000, 0, 0x400000, 0x500000, 0x8000000, 0x9000000, 1 << 40,
                                check=False) == status


def test_cache_rows_are_checked():
    for r, a in ((rows(n_requests=0), {}), (rows(row_off=0), {}), (rows(start=0), {}), (rows(table=0), {}),
                 (rows(n_rows=-1), {}), (rows(), dict(dtype=5)), (rows(), dict(k=0)), (rows(), dict(v=0x7000004)),
                 (rows(), dict(ldk=64)), (rows(), dict(ldv=130)), (rows(), dict(ws=0x8)), (rows(), dict(pos=0x2))):
        args = dict(dtype=stca.STCA_BF16, k=0x6000000, v=0x7000000)
        args.update(a)
        for f in (stca.stca_cache_write, stca.stca_cache_read):
            assert f(cache(), r, check=False, **args) == BAD, (r, a)


def test_cache_attention_arguments_are_checked():
    host = np.array([0, 3, 9], dtype=np.int32)

    def call(a=None, q=0x6000000, ldq=0, tgt_pos=0x400000, bias=0x500000, out=0x8000000, ws=0x9000000, ws_bytes=1 << 40,
             **kw):
        b = dict(n_requests=2, n_tgt=9, tgt_off=0x10000, lens=0x20000, max_len=100, table=0x30000, table_ld=2,
                 tgt_off_host=host)
        b.update(kw)
        b = stca.cache_batch(**b)
        return stca.stca_cache_attn(a or attn(), cache(), b, q, ldq, tgt_pos, bias, out, ws, ws_bytes, check=False)
    for kw in (dict(q=0), dict(q=0x6000002), dict(ldq=100), dict(tgt_pos=0), dict(bias=0), dict(out=0), dict(ws=0),
               dict(n_requests=0), dict(tgt_off=0), dict(lens=0), dict(table=0), dict(table_ld=1), dict(max_len=-1),
               dict(tgt_off_host=np.array([0, 9, 3], dtype=np.int32)), dict(a=attn(n_kv_heads=2)), dict(a=attn(d_head=64))):
        assert call(**kw) == BAD, kw
    assert call(a=attn(dtype=stca.STCA_F32)) == NO
    b = stca.cache_batch(2, 9, 0x10000, 0x20000, 100, 0x30000, 2, host)
    need = stca.stca_cache_attn_workspace_size(attn(), cache(), b)
    assert need > 0 and call(ws_bytes=need - 1) == SMALL


def test_bias_edges():
    for n, exact, top in ((2, 1, 2), (32, 8, 8192), (128, 64, 2 ** 31 - 2), (128, 1, 128), (100, 99, 100), (8, 7, 8)):
        e = stca.bias_edges(n, exact, top)
        assert len(e) == n - 1 and e[0] == 1 and (np.diff(e.astype(np.int64)) >= 1).all() and e[-1] <= top
        assert list(e[:exact]) == list(range(1, min(exact, n - 1) + 1))
        if exact < n - 1:
            assert e[-1] == top
    for n, exact, top in ((1, 1, 8), (129, 8, 8192), (8, 0, 100), (8, 8, 100), (8, 2, 7), (8, 2, 2 ** 31 - 1)):
        with pytest.raises(stca.StcaError):
            stca.bias_edges(n, exact, top)
    assert stca.lib().stca_bias_edges(8, 2, 100, ctypes.POINTER(ctypes.c_int32)()) == BAD


# ---- the oracle's own pins

def _tiny(seed=0):
    rng = np.random.default_rng(seed)
    hoff, toff = np.array([0, 5, 12]), np.array([0, 3, 4])
    q, k, v, g = (rng.standard_normal(s) for s in ((4, 4, 8), (12, 2, 8), (12, 2, 8), (4, 4, 8)))
    return dict(q=q, k=k, v=v, hoff=hoff, toff=toff, scale=0.3, cap=1.5, edges=[1, 3], bias=rng.standard_normal((4, 3)),
                masked=True, tgt_pos=np.array([2, 4, -1, 6])), g


def test_oracle_matches_autograd():
    torch = pytest.importorskip("torch")
    a, g = _tiny()
    r = O.attention(**a, dout=g)
    q, k, v, bias = (torch.tensor(a[n], requires_grad=True) for n in ("q", "k", "v", "bias"))
    out = torch.zeros(4, 4, 8, dtype=torch.float64)
    for i in range(2):
        for t in range(a["toff"][i], a["toff"][i + 1]):
            for h in range(4):
                js = [j for j in range(a["hoff"][i], a["hoff"][i + 1]) if j - a["hoff"][i] <= a["tgt_pos"][t]]
                if not js:
                    continue
                d = [a["tgt_pos"][t] - (j - a["hoff"][i]) for j in js]
                x = torch.stack([1.5 * torch.tanh(0.3 * (q[t, h] @ k[j, h // 2]) / 1.5) +
                                 bias[h, (dd >= 1) + int(dd >= 3)] for j, dd in zip(js, d)])
                out[t, h] = torch.softmax(x, 0) @ v[js, h // 2]
    (out * torch.tensor(g)).sum().backward()
    assert np.allclose(r["out"], out.detach().numpy(), rtol=1e-12, atol=1e-14)
    for n, x in (("dq", q), ("dk", k), ("dv", v), ("dbias", bias)):
        assert np.allclose(r[n], x.grad.numpy(), rtol=1e-11, atol=1e-13), n
        assert (np.abs(r[n]) <= r[n + "_abs"] + 1e-12).all(), n


@pytest.mark.parametrize("wrong", [dict(masked=False), dict(cap=0.0), dict(edges=[1, 4]), dict(scale=0.31)])
def test_oracle_sees_planted_mistakes(wrong):
    a, g = _tiny()
    x, y = O.attention(**a, dout=g), O.attention(**{**a, **wrong}, dout=g)
    assert max(np.abs(x[n] - y[n]).max() for n in ("out", "dq", "dk", "dv")) > 1e-3


def test_oracle_quantises_to_the_nearest():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((50, 32)) * 2.0 ** rng.integers(-100, 100, size=(50, 1))
    n, e = O.quantise(x)
    step = 2.0 ** (e - 127.0)
    top = np.abs(x).max(axis=1)
    assert (np.abs(n) <= 127).all() and (step * 64 <= top).all() and (top < step * 128).all()
    err = np.abs(O.held(n, e) - x)
    assert (err <= step[:, None] * np.where(np.abs(x) > 127.5 * step[:, None], 1.0, 0.5)).all()
    assert O.quantise(np.zeros((1, 32)))[1][0] == 1 and O.quantise(np.full((1, 32), np.nan))[1][0] == 255


@pytest.mark.parametrize("d_head", [32, 64, 128])
@pytest.mark.parametrize("dtype", [stca.STCA_F32, stca.STCA_BF16])
def test_every_accepted_table_has_its_lds(d_head, dtype):
    """Query heads a kv head and buckets up to their limits, of one kv head and
    of several to a workgroup, packed and paged, few targets, many and none:
    every plan fits a CU's LDS (one that does not has no size)."""
    for buckets in (0, 1, 34, 35, 70, 71, 100, 127, 128):
        edges = np.arange(1, max(buckets, 1), dtype=np.int32)
        for G in (1, 2, 3, 16, 31, 32, 33, 48, 61, 62, 63, 64):
            for Hk in (1, 2, 4):
                if Hk * G * d_head > 65536:
                    continue
                a = attn(n_heads=Hk * G, n_kv_heads=Hk, d_head=d_head, dtype=dtype, n_buckets=buckets, edges=edges)
                for m in (0, 1, 16, 40, 70):
                    b = batch([0, 300000, 300001], [0, m, m])
                    assert stca.stca_attn_workspace_size(a, b, False) and stca.stca_attn_workspace_size(a, b, True)
                if dtype == stca.STCA_BF16:
                    c = cache(n_kv_heads=Hk, d_head=d_head, page_size=16)
                    assert stca.stca_cache_attn_workspace_size(
                        a, c, stca.cache_batch(1, 3, 0x10000, 0x20000, 1000000, 0x30000, 1 << 20))


@pytest.mark.parametrize("L,m,fwd,bwd", [
    ([256] * 255 + [10240], [16] * 256, 16, 64),
    ([256] * 2047 + [32768], [16] * 2048, 128, 512),
    ([1] * 1000 + [100000], [1] * 1001, 16, 128),
    # both ends at once: longer chunks, dk and dv of the passes wait in fp32 (543 MiB)
    ([256] * 2047 + [32768], [16] * 2047 + [512], 256, 2048), ([256] * 2047 + [32768], [512] + [16] * 2047, 256, 2048)])
def test_one_long_history_among_short_ones(L, m, fwd, bwd):
    """Workspaces (MiB) of the order of the batch's own rows, not of the longest
    history times all targets (4 and 33 GB for the second batch)."""
    def off(n):
        return np.concatenate([[0], np.cumsum(n)])
    a, b = attn(n_heads=8, n_kv_heads=2, d_head=64), batch(off(L), off(m))
    assert 0 < stca.stca_attn_workspace_size(a, b, False) <= fwd << 20
    assert 0 < stca.stca_attn_workspace_size(a, b, True) <= bwd << 20


def test_edges_and_offsets_keep_their_values():
    """Numbers that int32 cannot hold are refused, not wrapped or cut."""
    pytest.importorskip("torch")
    from paper_2511_06077_amd import attention
    for bad in ([0, 2 ** 32 + 5], [0, -2 ** 31 - 1], [0, 1.5], [0, float("nan")], ["a"], np.array([0, 2 ** 31], dtype=np.uint32)):
        with pytest.raises(ValueError):
            attention._int32("edges", bad)
        with pytest.raises(ValueError):
            attention._offsets(bad, "cpu")
    for good in ([0, 3], (0, 3), [0.0, 3.0], np.array([0, 3]), np.array([0, 3], dtype=np.uint8), np.array([0, 9, 3])[::2]):
        host, dev = attention._offsets(good, "cpu")
        assert host.dtype == np.int32 and host.flags.c_contiguous and list(host) == [0, 3] and dev.tolist() == [0, 3]
    assert attention._int32("edges", []).shape == (0,)


@pytest.mark.parametrize("G", [1, 4])
@pytest.mark.parametrize("first", [1 << 20, 0x7fff0000 - 60, 0x5fff0001])
def test_the_longest_history_beside_targets_without_one(G, first):
    """Chunks of the longest history there may be stay below 2^31 rows."""
    a = attn(n_heads=4 * G, n_kv_heads=4, d_head=128)
    b = batch([0, first, first, first + 50], [0, 1, 1000001, 1000002])
    for back in (False, True):
        own = 8 * 1000002 * a.n_heads * (a.d_head + 2) * 4 + (8 * (first + 50) * 4 * 128 if back else 0) + (first << 4)
        assert 0 < stca.stca_attn_workspace_size(a, b, back) < own


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hk,dh,L,m", [s for i, s in enumerate(attn_common.SPREAD) if i != 1])
def test_a_lost_block_is_seen(Hk, dh, L, m, dtype):
    """The bounds of the long histories' test against the oracle without one block
    of 32 rows: out, dq and dbias each show it."""
    torch = pytest.importorskip("torch")
    rng = np.random.default_rng(7)
    m = [min(x, 3) for x in m]
    f, opts = attn_common.spread(rng, L, m, Hk, Hk, dh)
    f = {n: attn_common.rounded(torch, x, dtype)[1] for n, x in f.items()}
    hoff, toff = attn_common.offsets(L), attn_common.offsets(m)
    pos = np.arange(hoff[-1]) - np.repeat(hoff[:-1], L)
    r = int(np.argmax(L))
    for block in (0, L[r] // 64, L[r] // 32 - 1):
        keep = np.ones(hoff[-1], dtype=bool)
        keep[hoff[r] + 32 * block:hoff[r] + 32 * block + 32] = False
        less = np.array([keep[a:b].sum() for a, b in zip(hoff[:-1], hoff[1:])])
        kw = dict(scale=1.0, masked=True, **{n: x.astype(np.float64) if n == "bias" else x for n, x in opts.items()})
        if block == 0:
            ref = O.attention(f["q"], f["k"], f["v"], hoff, toff, dout=f["dout"], hist_pos=pos, **kw)
        bad = O.attention(f["q"], f["k"][keep], f["v"][keep], attn_common.offsets(less), toff, dout=f["dout"],
                          hist_pos=pos[keep], **kw)
        c = attn_common.deep(dtype, dh, L, ref)
        for n in ("out", "dq", "dbias"):
            e = attn_common.worst(bad[n], ref[n], ref[n + "_abs"], "f32" if n == "dbias" else dtype, c)
            assert e > 1.5, (n, block, e)  # (a result may be off by the bound itself)
