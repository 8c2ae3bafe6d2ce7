"""The paged history cache and the attention over it on the GPU: written bytes
against the definition to the bit, reads, attention against the float64 oracle
on the values held, and train, fill and serve run together."""
import numpy as np
import pytest

from attn_common import offsets, rel, rounded, worst
from oracle import attn_oracle as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available(), "GPU tests need a GPU"
    return t


class Users:
    """Requests with `start` rows before the packed rows, pages in any order."""

    def __init__(self, torch, n, start, page, *, Hk=2, dh=32, dtype="bf16", fmt="int8", seed=0, positions=False,
                 spare=2, gain=None):
        from paper_2511_06077_amd.attention import HistoryCache
        rng = np.random.default_rng([seed, page, dh])
        self.torch, self.page, self.dtype, self.fmt = torch, page, dtype, fmt
        self.n, self.start, self.off = np.asarray(n), np.asarray(start, dtype=np.int32), offsets(n)
        pages = -(-(self.start + self.n) // page)
        total = int(pages.sum()) + spare
        order = rng.permutation(total).astype(np.int32)
        self.table = np.full((len(n), max(1, int(pages.max(initial=1)))), -1, dtype=np.int32)
        at = 0
        for r, c in enumerate(pages):
            self.table[r, :c] = order[at:at + c]
            at += c
        rows = int(self.off[-1])
        self.t, self.f = {}, {}
        for name in ("k", "v"):
            x = rng.standard_normal((rows, Hk, dh)) * (2.0 ** rng.integers(-30, 30, size=(rows, Hk, 1)) if gain is None else gain)
            self.t[name], self.f[name] = rounded(torch, x, dtype)
        self.pos = rng.integers(-1000, 1000, size=rows).astype(np.int32) if positions else None
        self.cache = HistoryCache(total, page, Hk, dh, fmt=fmt, positions=positions)

    def dev(self, a):
        return None if a is None else self.torch.from_numpy(np.ascontiguousarray(a)).cuda()

    def where(self):
        return self.dev(self.off), self.dev(self.start), self.dev(self.table)

    def write(self):
        self.cache.write(self.t["k"].cuda(), self.t["v"].cuda(), *self.where(), pos=self.dev(self.pos))
        assert self.cache.device_status() == 0

    def slots(self):
        req = np.repeat(np.arange(len(self.n)), self.n)
        row = np.arange(self.off[-1]) - self.off[req] + self.start[req]
        return self.table[req, row // self.page], row % self.page

    def expect(self):
        """Page arrays by the definition (zero elsewhere), and the values held."""
        c, page, slot, torch = self.cache, *self.slots(), self.torch
        out, vals = {}, {}
        for name in ("k", "v"):
            x = self.f[name]
            buf = np.zeros(tuple(getattr(c, name).shape))
            if self.fmt == "int8":
                n, e = O.quantise(x)
                vals[name] = O.held(n, e)
                exps = np.zeros(tuple(c.k_exp.shape))
                exps[page, :, slot] = e
                out[name + "_exp"] = exps
            else:
                n = vals[name] = torch.from_numpy(x).to(torch.bfloat16).double().numpy()
            if name == "k":
                buf[page, :, slot, :] = n
            else:
                buf[page, :, :, slot] = n
            out[name] = buf
        return out, vals

    def check(self):
        want, vals = self.expect()
        for name, w in want.items():
            got = getattr(self.cache, name).double().cpu().numpy()
            assert np.array_equal(got, w), (name, np.argwhere(got != w)[:4])
        return vals


WRITES = [([1], [0]), ([1, 3, 0, 2], [5, 63, 9, 0]), ([64, 128, 17], [0, 64, 0]), ([200, 1, 90], [13, 700, 47]),
          ([0, 0], [3, 0])]


@pytest.mark.parametrize("fmt", ["int8", "bf16"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page,dh", [(16, 32), (64, 64), (256, 128), (32, 128), (128, 32)])
@pytest.mark.parametrize("n,start", WRITES)
def test_write_and_read(torch, fmt, dtype, page, dh, n, start):
    u = Users(torch, n, start, page, dh=dh, dtype=dtype, fmt=fmt, positions=page == 64)
    u.write()
    vals = u.check()
    if u.pos is not None:
        p, s = u.slots()
        assert np.array_equal(u.cache.pos.cpu().numpy()[p, s], u.pos)
    for out in (torch.bfloat16, torch.float32):
        got = u.cache.read(*u.where(), int(u.off[-1]), dtype=out)
        assert u.cache.device_status() == 0
        for name, y in zip(("k", "v"), got):
            assert torch.equal(y.double().cpu(), torch.from_numpy(vals[name]).to(out).double()), name
        if u.pos is not None:
            assert np.array_equal(got[2].cpu().numpy(), u.pos)


def test_rows_one_after_the_other(torch):
    """Appends of single rows give the bytes of one write, and leave the other
    slots of a page as they were."""
    u = Users(torch, [70, 20], [0, 0], 32, seed=4)
    u.cache.k.fill_(77), u.cache.v.fill_(77), u.cache.k_exp.fill_(77), u.cache.v_exp.fill_(77)
    table = u.dev(u.table)
    for i in range(70):
        n = [1, 1 if i < 20 else 0]
        rows = [i] + ([70 + i] if i < 20 else [])
        u.cache.write(u.t["k"][rows].cuda(), u.t["v"][rows].cuda(), u.dev(offsets(n)),
                      u.dev(np.array([i, min(i, 20)], dtype=np.int32)), table)
    want, _ = u.expect()
    page, slot = u.slots()
    used = np.zeros((u.cache.n_pages, 32), dtype=bool)
    used[page, slot] = True
    for name, w in want.items():
        got = getattr(u.cache, name).double().cpu().numpy()
        m = used[:, None, None, :] if name == "v" else used[:, None, :, None] if name == "k" else used[:, None, :]
        assert np.array_equal(got, np.where(np.broadcast_to(m, w.shape), w, 77)), name


def test_rounding_borders_and_odd_rows(torch):
    """Ties, powers of two and their neighbours, zeros, the smallest and largest
    values, and rows that are not finite (read as NaN)."""
    dh, big = 32, float(torch.finfo(torch.float32).max)
    rows = [np.linspace(-1, 1, dh), np.full(dh, 0.0), np.r_[1.0, np.arange(31) / 128 + 1 / 128 / 2],
            np.r_[np.nextafter(np.float32(2), np.float32(0)), np.full(31, 1.9999)], np.full(dh, 2.0),
            np.r_[big, -big, np.zeros(30)], np.full(dh, 2.0 ** -149), np.full(dh, 2.0 ** -126) * np.arange(dh),
            np.r_[np.inf, np.zeros(31)], np.r_[np.ones(31), np.nan], np.r_[-1.0, np.full(31, 127.5 / 128)]]
    u = Users(torch, [len(rows)], [3], 16, dtype="f32", Hk=1, gain=1.0)
    for name in ("k", "v"):
        x = np.stack(rows).astype(np.float32)[:, None, :]
        u.t[name], u.f[name] = torch.from_numpy(x), x.astype(np.float64)
    u.write()
    vals = u.check()
    for name, y in zip(("k", "v"), u.cache.read(*u.where(), len(rows), dtype=torch.float32)):
        assert np.array_equal(y.cpu().numpy().astype(np.float64), vals[name].astype(np.float32), equal_nan=True)


def test_strided_rows_and_missing_pages(torch):
    """K and V as slices of fused rows; rows whose page is missing are left out,
    the others written, and the status says so."""
    from paper_2511_06077_amd import stca
    u = Users(torch, [40, 50], [0, 10], 16, Hk=2, seed=9)
    fused = torch.full((90, 3, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    fused[:, 0], fused[:, 2] = u.t["k"].flatten(1).cuda(), u.t["v"].flatten(1).cuda()
    off, start, table = u.where()
    u.cache.write(fused[:, 0], fused[:, 2], off, start, table)
    u.check()
    before = u.cache.k.clone()
    for bad in (-1, u.cache.n_pages, 2 ** 31 - 1):
        holes = table.clone()
        holes[0, 1] = bad
        u.cache.write(-fused[:, 0], fused[:, 2], off, start, holes)
        assert u.cache.device_status() == stca.STCA_ERR_INVALID_ARG
        assert torch.equal(u.cache.k[u.table[0, 1]], before[u.table[0, 1]])
        assert torch.equal(u.cache.k[u.table[0, 0]], -before[u.table[0, 0]])
        u.cache.write(fused[:, 0], fused[:, 2], off, start, table)
    u.cache.write(fused[:, 0], fused[:, 2], off, start, table[:, :1].contiguous())  # a table that is too short
    assert u.cache.device_status() == stca.STCA_ERR_INVALID_ARG
    u.check()


# ---- attention over the cache

def serve(u, torch, m, H, lens=None, *, cap=0.0, nb=0, masked=False, seed=0, max_len=None, q_gain=1.0):
    """Attention of m[r] targets over user r's first lens[r] rows (start 0), and the oracle's."""
    from paper_2511_06077_amd.attention import CacheAttention, bias_edges
    rng = np.random.default_rng([seed, 5])
    dh, Hk = u.cache.d_head, u.cache.n_kv_heads
    lens = u.n if lens is None else np.asarray(lens)
    toff = offsets(m)
    nt = int(toff[-1])
    qt, qf = rounded(torch, q_gain * rng.standard_normal((nt, H, dh)), "bf16")
    edges = bias_edges(nb, max(1, nb // 3), 700) if nb else None
    bias = rng.standard_normal((H, nb)).astype(np.float32) if nb else None
    tgt_pos = None
    if nb or masked:
        tgt_pos = np.concatenate([rng.integers(-1, max(l, 1) + 3, size=c) if u.pos is None else
                                  rng.integers(-1100, 1100, size=c) for l, c in zip(lens, m)]).astype(np.int32)
    scale = float(np.float32(dh ** -0.5))
    plan = CacheAttention(u.cache, toff, H, int(max(lens) if max_len is None else max_len), scale=scale, softcap=cap,
                          edges=edges, masked=masked)
    out = plan.forward(qt.cuda(), u.dev(lens.astype(np.int32)), u.dev(u.table), tgt_pos=u.dev(tgt_pos), bias=u.dev(bias))
    _, vals = u.expect()
    keep = np.concatenate([np.arange(o, o + l) for o, l in zip(u.off, lens)] + [np.zeros(0, int)]).astype(int)
    ref = O.attention(qf, vals["k"][keep], vals["v"][keep], offsets(lens), toff, scale=scale, cap=cap, edges=edges,
                      bias=None if bias is None else bias.astype(np.float64), masked=masked, tgt_pos=tgt_pos,
                      hist_pos=None if u.pos is None else u.pos[keep])
    e = worst(out.double().cpu().numpy(), ref["out"], ref["out_abs"], "bf16",
              rel("bf16", dh, int(max(lens.max(initial=1), 1)), ref, cap))
    print(f"[cache attention] {e:.3f} of the bound", flush=True)
    return plan, out, e


SERVES = {
    "one_row": dict(n=[1], m=[1], H=2),
    "decode": dict(n=[1000, 17, 333], m=[1, 1, 1], H=4, nb=16),
    "chunks": dict(n=[70, 300, 1, 64, 0, 15], m=[5, 20, 3, 0, 2, 40], H=2, nb=32, masked=True),
    "shared": dict(n=[257, 40], m=[9, 30], H=8, cap=3.0, masked=True),
    "many": dict(n=[90], m=[150], H=2, nb=8),
    "positions": dict(n=[129, 31], m=[6, 17], H=4, nb=64, masked=True, positions=True),
    "long": dict(n=[5000], m=[2], H=2, nb=32, masked=True),
}


@pytest.mark.parametrize("fmt", ["int8", "bf16"])
@pytest.mark.parametrize("page,dh", [(16, 32), (64, 64), (128, 128), (256, 32)])
@pytest.mark.parametrize("name", list(SERVES))
def test_cache_attention(torch, name, page, dh, fmt):
    s = dict(SERVES[name])
    n, m, H = s.pop("n"), s.pop("m"), s.pop("H")
    u = Users(torch, n, [0] * len(n), page, dh=dh, fmt=fmt, positions=s.pop("positions", False), gain=1.0)
    u.write()
    plan, _, e = serve(u, torch, m, H, **s)
    assert plan.device_status() == 0
    assert e <= 1.0


@pytest.mark.parametrize("fmt", ["int8", "bf16"])
def test_shorter_lens_and_stale_pages(torch, fmt):
    """Fewer rows than the pages hold, under a larger max_len; what lies behind
    the last row (NaN here) is not looked at."""
    u = Users(torch, [200, 100, 64], [0, 0, 0], 64, fmt=fmt, gain=1.0, seed=6)
    lens = [77, 0, 33]
    for r, l in enumerate(lens):
        for name in ("k", "v"):
            u.t[name][u.off[r] + l:u.off[r + 1]] = float("nan")
            u.f[name][u.off[r] + l:u.off[r + 1]] = np.nan
    u.write()
    plan, out, e = serve(u, torch, [4, 2, 17], 4, lens, nb=8, max_len=201)
    assert plan.device_status() == 0 and e <= 1.0
    assert not out[4:6].any()


def test_rows_that_are_not_finite(torch):
    """A row stored as NaN reaches the targets that see it and no other."""
    for fmt in ("int8", "bf16"):
        u = Users(torch, [100], [0], 32, fmt=fmt, gain=1.0, seed=2)
        for name in ("k", "v"):
            u.t[name][60] = float("nan")
            u.f[name][60] = np.nan
        u.write()
        plan, out, e = serve(u, torch, [30], 2, masked=True)
        assert e <= 1.0 and bool(out.isnan().any()) and not bool(out.isnan().all())


def test_missing_pages_and_long_lens(torch):
    """A page outside the cache hides its rows; a length beyond max_len is cut;
    both are reported."""
    from paper_2511_06077_amd import stca
    u = Users(torch, [100, 50], [0, 0], 16, gain=1.0, seed=8)
    u.write()
    plan, out, e = serve(u, torch, [3, 3], 2)
    q = torch.ones((6, 2, 32), dtype=torch.bfloat16, device="cuda")
    lens, table = u.dev(np.array([100, 50], dtype=np.int32)), u.dev(u.table)
    want = plan.forward(q, lens, table)
    holes = table.clone()
    holes[0, 6] = 10 ** 9  # rows 96..99 of the first request
    got = plan.forward(q, lens, holes)
    assert plan.device_status() == stca.STCA_ERR_INVALID_ARG
    short = plan.forward(q, u.dev(np.array([96, 50], dtype=np.int32)), table)
    assert plan.device_status() == 0
    assert torch.equal(got, short) and not torch.equal(got, want)
    plan.forward(q, u.dev(np.array([100, 2 ** 30], dtype=np.int32)), table)
    assert plan.device_status() == stca.STCA_ERR_INVALID_ARG


def test_shared_pages_and_captured_decode(torch):
    """Two requests over the same pages agree; a decode step (append, attend)
    captured once follows lens and rows as they grow."""
    u = Users(torch, [150], [0], 64, gain=1.0, seed=11)
    u.write()
    from paper_2511_06077_amd.attention import CacheAttention
    q = torch.randn((2, 2, 32), device="cuda").to(torch.bfloat16)
    q[1] = q[0]
    table = u.dev(np.repeat(u.table, 2, axis=0))
    plan = CacheAttention(u.cache, [0, 1, 2], 2, 192)
    lens = torch.tensor([100, 100], dtype=torch.int32, device="cuda")
    out = plan.forward(q, lens, table)
    assert torch.equal(out[0], out[1])
    one = CacheAttention(u.cache, [0, 1], 2, 192)
    row_off = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    start, n = (torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(2))
    k, v = (torch.zeros((1, 2, 32), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    t1, q1 = table[:1].contiguous(), q[:1].contiguous()
    kd, vd = u.t["k"].cuda(), u.t["v"].cuda()

    def step():
        u.cache.write(k, v, row_off, start, t1)
        return one.forward(q1, n, t1)

    start.fill_(100), n.fill_(101), k.copy_(kd[100:101]), v.copy_(vd[100:101])
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = step()
    for i in (100, 101, 127, 128, 140):
        start.fill_(i), n.fill_(i + 1), k.copy_(kd[i:i + 1]), v.copy_(vd[i:i + 1])
        g.replay()
        torch.cuda.synchronize()
        want = one.forward(q1, n, t1)
        assert torch.equal(y, want), i
    u.check()


def test_cache_past_4_gib(torch):
    """Pages whose bytes lie past 2^32: written, read and attended to."""
    from paper_2511_06077_amd.attention import CacheAttention, HistoryCache
    Hk, dh, page = 8, 128, 256
    n_pages = 2 ** 32 // (Hk * dh * page) + 6
    c = HistoryCache(n_pages, page, Hk, dh)
    gen = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn((600, Hk, dh), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    small = HistoryCache(3, page, Hk, dh)
    off, start = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 600], [0]))
    far = torch.tensor([[n_pages - 1, n_pages - 3, n_pages - 2]], dtype=torch.int32, device="cuda")
    near = torch.tensor([[0, 1, 2]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([600], dtype=torch.int32, device="cuda")
    q = torch.randn((5, Hk, dh), generator=gen, device="cuda").to(torch.bfloat16)
    res = []
    for cache, table in ((c, far), (small, near)):
        cache.write(k, v, off, start, table)
        res.append((*cache.read(off, start, table, 600), CacheAttention(cache, [0, 5], Hk, 600).forward(q, lens, table)))
    for a, b in zip(*res):
        assert torch.equal(a, b)


def test_train_fill_and_serve(torch):
    """The three together: a step's attention over packed rows, the same rows in
    a bf16 cache (the same values, so both within their bounds of each other)
    and in an 8-bit one (within what half a step of K and V can move it)."""
    from paper_2511_06077_amd.attention import CacheAttention, CrossAttention, bias_edges
    n, m, H, Hk, dh = [300, 65, 900], [16, 3, 20], 4, 2, 32
    edges = bias_edges(16, 4, 500)
    gen = torch.Generator(device="cuda").manual_seed(3)
    hoff, toff = offsets(n), offsets(m)
    q, k, v = (torch.randn((r, h, dh), generator=gen, device="cuda").to(torch.bfloat16)
               for r, h in ((int(toff[-1]), H), (int(hoff[-1]), Hk), (int(hoff[-1]), Hk)))
    bias = torch.randn((H, 16), generator=gen, device="cuda")
    tgt_pos = torch.cat([torch.randint(l // 2, l, (c,), generator=gen, device="cuda") for l, c in zip(n, m)]).int()
    plan = CrossAttention(hoff, toff, H, dh, n_kv_heads=Hk, edges=edges, masked=True, backward=True)
    for _ in range(2):  # a step of the table and of the queries
        out = plan.forward(q, k, v, tgt_pos=tgt_pos, bias=bias)
        dq, dk, dv, dbias = plan.backward(out, q, k, v, tgt_pos=tgt_pos, bias=bias)
        bias = bias - 0.01 * dbias
        q = (q.float() - 0.01 * dq.float()).to(torch.bfloat16)
    out = plan.forward(q, k, v, tgt_pos=tgt_pos, bias=bias)
    for fmt in ("bf16", "int8"):
        u = Users(torch, n, [0, 0, 0], 64, Hk=Hk, fmt=fmt, gain=1.0)
        u.t = {"k": k.cpu(), "v": v.cpu()}
        u.f = {x: y.double().numpy() for x, y in u.t.items()}
        u.write()
        u.check()
        serve_plan = CacheAttention(u.cache, toff, H, max(n), edges=edges, masked=True)
        got = serve_plan.forward(q, u.dev(np.asarray(n, dtype=np.int32)), u.dev(u.table), tgt_pos=tgt_pos, bias=bias)
        assert serve_plan.device_status() == 0
        d = (got.float() - out.float()).abs()
        if fmt == "bf16":
            assert float((d / (out.float().abs() + 1e-3)).max()) <= 2.0 ** -7  # neighbouring bf16 values at most
        else:
            # half a step: max|x| 2^-7 of each row's largest value, about 4 here.  Values: 4 2^-7; scores: sum |q|
            # 4 2^-7 / sqrt(dh) each way, which moves weights by twice that and the output by that times max |v|
            vmax, qsum = float(v.float().abs().max()), float(q.float().abs().sum(-1).max())
            top = max(vmax, float(k.float().abs().max()))
            move = 2 * qsum * top * 2.0 ** -7 / dh ** 0.5
            assert float(d.max()) <= top * 2.0 ** -7 + 2 * vmax * float(np.expm1(move))
