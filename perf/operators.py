"""The operators around the target-to-history attention, as cases to be timed.

Three operators beside the layer stack's own kernels:

  attention  ragged target-to-history cross attention with capped scores, a
             learned bias by buckets of distance and a mask to the prefix a
             target may see: forward ("forward") and training step ("train":
             forward, then the gradients of q, k, v and the bias table)
  cache      a paged K/V cache, in 8 bits or bf16: rows written and read back
             ("cache_write"), stored rows read ("cache_read")
  serving    attention of each request's new tokens over its cached rows
             ("cache_attend"), with the same cap, bias and mask

For target t at position p_t, history row j at p_j, head h of kv head g:

  z = scale q.k;  y = c tanh(z / c) if c else z;  x = y + bias[h][b(p_t - p_j)]
  b(D) = number of edges <= max(D, 0);  a row with p_t < p_j is hidden if masked
  out = softmax over the visible rows times v, and 0 where there is none

Cache of 8 bits, per row and kv head: step = 2^max(floor(log2 max|x|) - 6, -126),
n = x / step rounded to nearest even, within -127..127.  K pages are
[page][kv head][slot][d], V pages [page][kv head][d][slot].

A case is a dict of plain values; "L" and "m" are (lowest, highest) history
length and target count as "lo-hi", drawn uniform by "shape", which belongs to
the case; the seed given to prepare() draws the values.
"""
import math

import numpy as np
import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_ES = {"bf16": 2, "f32": 4}


def _case(name, op, requests, L, m="0-0", *, dtype="bf16", heads=8, kv_heads=None, d_head=32, cap=0.0, buckets=0,
          masked=False, pos="index", fmt="int8", page=64, shape=0):
    return {"name": name, "op": op, "requests": requests, "L": L, "m": m, "dtype": dtype, "heads": heads,
            "kv_heads": kv_heads or heads, "d_head": d_head, "cap": cap, "buckets": buckets, "masked": masked,
            "pos": pos, "fmt": fmt, "page": page, "shape": shape}


def listed():
    return [
        # a parity or debugging run in fp32, a few small requests
        _case("forward_small_f32", "forward", 4, "256-256", "4-4", dtype="f32", heads=2, buckets=16),
        # evaluation over the training window, 16 targets a request, time buckets
        _case("forward_window", "forward", 256, "2048-2048", "16-16", buckets=32, masked=True, pos="time"),
        # the small model's training step: d = 128, 1k histories
        _case("train_uniform", "train", 64, "1024-1024", "16-16", heads=4, buckets=32, masked=True),
        # the training window: 2k histories, each target sees what came before it
        _case("train_window", "train", 256, "2048-2048", "16-16", buckets=32, masked=True, pos="time"),
        # ragged histories and targets, wider heads that share K and V, capped scores
        _case("train_ragged_shared", "train", 48, "1-2048", "1-64", heads=8, kv_heads=2, d_head=64, cap=30.0,
              buckets=64, masked=True, shape=5),
        # a gradient check in fp32 storage, odd lengths
        _case("train_small_f32", "train", 6, "7-300", "1-19", dtype="f32", heads=2, cap=20.0, buckets=16,
              masked=True, shape=3),
        # a serving step's new events: a row or a few per user at any slot
        _case("cache_append", "cache_write", 256, "1-4", shape=7),
        # users' histories projected for the first time
        _case("cache_fill", "cache_write", 24, "512-10240", shape=8),
        # cached histories read back to be trained on or moved
        _case("cache_read", "cache_read", 64, "512-4096", shape=9),
        # one candidate of one user: latency
        _case("attend_one", "cache_attend", 1, "10240-10240", "1-1", buckets=32),
        # a full serving batch: 10k histories, 32 candidates per request
        _case("attend_batch", "cache_attend", 128, "10240-10240", "32-32", buckets=32),
        # chunks of new tokens that see each other's past, wide shared heads, bf16 pages
        _case("attend_chunk", "cache_attend", 24, "1-10240", "1-16", heads=16, kv_heads=4, d_head=128, cap=50.0,
              masked=True, fmt="bf16", page=16, shape=11),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ranges (rng: random.Random)."""
    op = rng.choice(["forward", "train", "train", "cache_write", "cache_read", "cache_attend", "cache_attend"])
    dh = rng.choice([32, 32, 64, 128])
    hk = rng.choice([1, 2, 4, 8])
    h = hk * rng.choice([1, 1, 2, 4])
    hi = _log_int(rng, 1, 10240)
    lo = rng.choice([1, hi, max(1, hi // 2), max(1, hi - 3)])
    mhi = _log_int(rng, 1, 64)
    mlo = rng.choice([1, mhi])
    f32 = op in ("forward", "train") and rng.random() < 0.25
    # no dearer than the dearest listed cases: history elements and scores
    rows = {"forward": 4e7, "train": 4e7, "cache_write": 2.5e7, "cache_read": 2.5e7, "cache_attend": 2e8}[op]
    scores = 3e7 if f32 or op == "train" else 6e7
    top = min(rows / (hi * hk * dh), scores / (hi * mhi * h), 256)
    R = _log_int(rng, 1, max(1, int(top)))
    buckets = rng.choice([0, 8, 16, 32, 64, 100])
    return {"op": op, "requests": R, "L": f"{lo}-{hi}",
            "m": "0-0" if op in ("cache_write", "cache_read") else f"{mlo}-{mhi}",
            "dtype": "f32" if f32 else "bf16", "heads": h, "kv_heads": hk, "d_head": dh,
            "cap": rng.choice([0.0, 0.0, 10.0, 50.0]), "buckets": buckets,
            "masked": rng.random() < 0.6, "pos": rng.choice(["index", "time"]),
            "fmt": rng.choice(["int8", "int8", "bf16"]), "page": rng.choice([16, 32, 64, 128, 256]),
            "shape": rng.randrange(1 << 20)}


# ---- inputs

def _edges(buckets, pos):
    """Single distances first, then a geometric series (strictly ascending)."""
    top = 8192 if pos == "index" else 1 << 22
    n, exact = buckets - 1, min(8, (buckets - 1) // 2 + 1)
    out = []
    for i in range(n):
        e = i + 1 if i < exact else exact * (top / exact) ** ((i - exact + 1) / (n - exact))
        out.append(max(int(e), out[-1] + 1 if out else 1))
    return out


def _shape(case):
    rng = np.random.default_rng([case["shape"], case["requests"]])
    def pick(s):
        lo, hi = (int(x) for x in s.split("-"))
        return rng.integers(lo, hi + 1, size=case["requests"])
    return pick(case["L"]), pick(case["m"])


def _off(n):
    return np.concatenate([[0], np.cumsum(n)]).astype(np.int32)


def _positions(case, L, m, rng):
    """Positions of the history rows and of the targets: indices, or event
    times with gaps of seconds to hours; masked targets lie in the second half
    of their history, now and then before all of it."""
    hp, tp = [], []
    for l, n in zip(L, m):
        if case["pos"] == "time":
            p = np.cumsum(np.exp(rng.uniform(0, 8, size=l)).astype(np.int64))
        else:
            p = np.arange(l, dtype=np.int64)
        if case["masked"]:
            t = p[rng.integers(l // 2, l, size=n)]
            t[rng.random(n) < 0.02] = -1
        else:
            t = p[-1] + rng.integers(1, 9, size=n)
        hp.append(p)
        tp.append(np.sort(t))
    return np.concatenate(hp).astype(np.int32), np.concatenate(tp).astype(np.int32)


def _normal(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)


def _inputs(case, seed):
    """Everything the call is given, on the GPU, and the shapes on the host."""
    rng = np.random.default_rng([seed, case["shape"]])
    gen = torch.Generator(device="cuda").manual_seed(seed * 1000003 + case["shape"])
    L, m = _shape(case)
    H, Hk, dh, dt = case["heads"], case["kv_heads"], case["d_head"], _DT[case["dtype"]]
    s = {"case": case, "L": L, "m": m, "hoff": _off(L), "toff": _off(m)}
    nh, nt = int(L.sum()), int(m.sum())
    s["edges"] = _edges(case["buckets"], case["pos"]) if case["buckets"] else None
    s["bias"] = _normal(gen, (H, case["buckets"]), torch.float32) if case["buckets"] else None
    s["scale"] = 1.0 / math.sqrt(dh)
    if case["op"] in ("forward", "train"):
        hp, tp = _positions(case, L, m, rng)
        placed = case["buckets"] > 0 or case["masked"]
        s["hist_pos"] = torch.from_numpy(hp).cuda() if placed and case["pos"] == "time" else None
        s["tgt_pos"] = torch.from_numpy(tp).cuda() if placed else None
        s["q"], s["k"], s["v"] = (_normal(gen, (n, h, dh), dt) for n, h in ((nt, H), (nh, Hk), (nh, Hk)))
        if case["op"] == "train":
            s["dout"] = _normal(gen, (nt, H, dh), dt)
        return s
    # the cache: pages handed out in any order, rows at any slot
    page = case["page"]
    s["start"] = rng.integers(0, 3 * page, size=len(L)).astype(np.int32) if case["op"] != "cache_attend" \
        else np.zeros(len(L), dtype=np.int32)
    pages = -(-(s["start"] + L) // page)
    s["n_pages"] = int(pages.sum()) + 3
    order = rng.permutation(s["n_pages"]).astype(np.int32)
    table = np.zeros((len(L), int(pages.max())), dtype=np.int32)
    at = 0
    for r, n in enumerate(pages):
        table[r, :n] = order[at:at + n]
        at += n
    req = np.repeat(np.arange(len(L)), L)
    row = np.arange(nh) - s["hoff"][:-1][req] + s["start"][req]
    s["page_of"] = torch.from_numpy(table[req, row // page].astype(np.int64)).cuda()
    s["slot_of"] = torch.from_numpy((row % page).astype(np.int64)).cuda()
    s["table"], s["row_off"] = torch.from_numpy(table).cuda(), torch.from_numpy(s["hoff"]).cuda()
    s["start_dev"], s["lens"] = torch.from_numpy(s["start"]).cuda(), torch.from_numpy(L.astype(np.int32)).cuda()
    s["k"], s["v"] = (_normal(gen, (nh, Hk, dh), dt) for _ in range(2))
    s["pos"] = None
    if case["op"] == "cache_attend":
        hp, tp = _positions(case, L, m, rng)
        placed = case["buckets"] > 0 or case["masked"]
        s["tgt_pos"] = torch.from_numpy(tp).cuda() if placed else None
        s["pos"] = torch.from_numpy(hp).cuda() if placed and case["pos"] == "time" else None
        s["q"] = _normal(gen, (nt, H, dh), dt)
    return s


def _pages(s):
    """Empty page buffers of the cache's layout."""
    c = s["case"]
    n, hk, p, dh = s["n_pages"], c["kv_heads"], c["page"], c["d_head"]
    t = torch.int8 if c["fmt"] == "int8" else torch.bfloat16
    b = {"k": torch.zeros((n, hk, p, dh), dtype=t, device="cuda"),
         "v": torch.zeros((n, hk, dh, p), dtype=t, device="cuda")}
    if c["fmt"] == "int8":
        b["k_exp"] = torch.zeros((n, hk, p), dtype=torch.uint8, device="cuda")
        b["v_exp"] = torch.zeros((n, hk, p), dtype=torch.uint8, device="cuda")
    if s["pos"] is not None:
        b["pos"] = torch.zeros((n, p), dtype=torch.int32, device="cuda")
    return b


def prepare(case, seed):
    s = _inputs(case, seed)
    cached = case["op"].startswith("cache")
    if cached:
        b = s["pages"] = _pages(s)
        if case["op"] != "cache_write":
            _plain_write(s)
    if own:
        from paper_2511_06077_amd.attention import CacheAttention, CrossAttention, HistoryCache
        opts = dict(scale=s["scale"], softcap=case["cap"], edges=s["edges"], masked=case["masked"])
        if cached:
            s["cache"] = HistoryCache(s["n_pages"], case["page"], case["kv_heads"], case["d_head"], fmt=case["fmt"],
                                      positions=s["pos"] is not None)
            for name, t in b.items():
                getattr(s["cache"], name).copy_(t)
            if case["op"] == "cache_attend":
                s["plan"] = CacheAttention(s["cache"], s["toff"], case["heads"], int(s["L"].max()), **opts)
        else:
            s["plan"] = CrossAttention(s["hoff"], s["toff"], case["heads"], case["d_head"],
                                       n_kv_heads=case["kv_heads"], dtype=_DT[case["dtype"]],
                                       backward=case["op"] == "train", **opts)
    return s


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    op = s["case"]["op"]
    if op == "cache_attend":
        return s["plan"].forward(s["q"], s["lens"], s["table"], tgt_pos=s["tgt_pos"], bias=s["bias"])
    if op in ("cache_write", "cache_read"):
        if op == "cache_write":
            s["cache"].write(s["k"], s["v"], s["row_off"], s["start_dev"], s["table"])
        return s["cache"].read(s["row_off"], s["start_dev"], s["table"], s["k"].shape[0], dtype=s["k"].dtype)
    given = dict(tgt_pos=s["tgt_pos"], hist_pos=s["hist_pos"], bias=s["bias"])
    out = s["plan"].forward(s["q"], s["k"], s["v"], **given)
    if op == "forward":
        return out
    g = s["plan"].backward(s["dout"], s["q"], s["k"], s["v"], **given)
    return [out] + [x for x in g if x is not None]


# ---- plain form

def _run_plain(s):
    op = s["case"]["op"]
    if op in ("cache_write", "cache_read"):
        if op == "cache_write":
            _plain_write(s)
        return tuple(x.to(s["k"].dtype) for x in _plain_read(s))
    if op == "cache_attend":
        k, v = _plain_read(s)
        pos = s["pos"]
        if pos is not None:
            pos = s["pages"]["pos"][s["page_of"], s["slot_of"]]
        return _plain_forward(s, k, v, pos)[0]
    if op == "forward":
        return _plain_forward(s, s["k"].float(), s["v"].float(), s["hist_pos"])[0]
    return _plain_train(s)


def _plain_write(s):
    c, b = s["case"], s["pages"]
    if s["pos"] is not None:
        b["pos"][s["page_of"], s["slot_of"]] = s["pos"]
    for name in ("k", "v"):
        x = s[name]
        if c["fmt"] == "int8":
            x = x.float()
            top = x.abs().amax(dim=-1)
            e = torch.where(top > 0, torch.frexp(top).exponent - 1 - 6, -126).clamp(min=-126)
            x = torch.round(torch.ldexp(x, -e[..., None])).clamp(-127, 127).to(torch.int8)
            b[name + "_exp"][s["page_of"], :, s["slot_of"]] = (e + 127).to(torch.uint8)
        else:
            x = x.to(torch.bfloat16)
        if name == "k":
            b["k"][s["page_of"], :, s["slot_of"], :] = x
        else:
            b["v"][s["page_of"], :, :, s["slot_of"]] = x


def _plain_read(s):
    b, at = s["pages"], (s["page_of"], slice(None), s["slot_of"])
    k, v = b["k"][at].float(), b["v"][s["page_of"], :, :, s["slot_of"]].float()
    if s["case"]["fmt"] == "int8":
        k = torch.ldexp(k, b["k_exp"][at].int()[..., None] - 127)
        v = torch.ldexp(v, b["v_exp"][at].int()[..., None] - 127)
    return k, v


def _plain_scores(s, r, q, k, pos):
    """Scores [H][m][L] of request r before and after the bias, the bucket of
    each pair and which pairs are visible."""
    c = s["case"]
    H, Hk = c["heads"], c["kv_heads"]
    m, l = q.shape[0], k.shape[0]
    y = torch.matmul(q.transpose(0, 1).reshape(Hk, H // Hk * m, -1), k.permute(1, 2, 0).contiguous())
    y = (y * s["scale"]).reshape(H, m, l)
    if c["cap"]:
        y = c["cap"] * torch.tanh(y / c["cap"])
    b, vis, x = None, torch.ones((m, l), dtype=torch.bool, device=q.device), y
    if s["tgt_pos"] is not None:
        p = pos if pos is not None else torch.arange(l, device=q.device)
        d = s["tgt_pos"][s["toff"][r]:s["toff"][r + 1], None].long() - p[None, :].long()
        if c["buckets"]:
            e = torch.tensor(s["edges"], device=q.device)
            b = (d.clamp(min=0)[..., None] >= e).sum(-1)
            x = y + s["bias"][:, b]
        if c["masked"]:
            vis = d >= 0
    return y, x, b, vis


def _plain_softmax(x, vis):
    x = torch.where(vis, x, -math.inf)
    top = x.amax(dim=-1, keepdim=True)
    w = torch.where(vis, torch.exp(x - torch.where(top == -math.inf, 0.0, top)), 0.0)
    return w / w.sum(dim=-1, keepdim=True).clamp(min=1e-38)


def _plain_forward(s, k, v, pos, keep=None):
    c = s["case"]
    H, Hk = c["heads"], c["kv_heads"]
    out = torch.zeros_like(s["q"])
    for r in range(c["requests"]):
        t, j = slice(*s["toff"][r:r + 2]), slice(*s["hoff"][r:r + 2])
        m, l = int(s["m"][r]), int(s["L"][r])
        q = s["q"][t].float()
        y, x, b, vis = _plain_scores(s, r, q, k[j], None if pos is None else pos[j])
        w = _plain_softmax(x, vis)
        o = torch.matmul(w.reshape(Hk, H // Hk * m, l), v[j].transpose(0, 1).contiguous())
        o = o.reshape(H, m, -1).transpose(0, 1)
        out[t] = o.to(out.dtype)
        if keep is not None:
            keep(r, t, j, q, y, b, w, o)
    return out, None


def _plain_train(s):
    c = s["case"]
    H, Hk, cap = c["heads"], c["kv_heads"], c["cap"]
    k, v = s["k"].float(), s["v"].float()
    dq, dk, dv = (torch.zeros_like(s[n]) for n in ("q", "k", "v"))
    dbias = torch.zeros((H, c["buckets"]), dtype=torch.float64, device=dq.device)

    def reverse(r, t, j, q, y, b, w, o):
        m, l = y.shape[1:]
        do = s["dout"][t].float()
        g = do.transpose(0, 1).reshape(Hk, H // Hk * m, -1)
        dp = torch.matmul(g, v[j].permute(1, 2, 0).contiguous()).reshape(H, m, l)
        dx = w * (dp - (do * o).sum(-1).transpose(0, 1)[..., None])
        if c["buckets"]:
            one = (b.reshape(-1, 1) == torch.arange(c["buckets"], device=b.device)).double()
            dbias.add_(torch.matmul(dx.reshape(H, m * l).double(), one))
        dz = (dx * (1 - (y / cap) ** 2) if cap else dx) * s["scale"]
        dz, p = dz.reshape(Hk, H // Hk * m, l), w.reshape(Hk, H // Hk * m, l)
        qg = q.transpose(0, 1).reshape(Hk, H // Hk * m, -1)
        dq[t] = torch.matmul(dz, k[j].transpose(0, 1).contiguous()).reshape(H, m, -1).transpose(0, 1).to(dq.dtype)
        dk[j] = torch.matmul(dz.transpose(1, 2).contiguous(), qg).transpose(0, 1).to(dk.dtype)
        dv[j] = torch.matmul(p.transpose(1, 2).contiguous(), g).transpose(0, 1).to(dv.dtype)

    out, _ = _plain_forward(s, k, v, s["hist_pos"], reverse)
    return [out, dq, dk, dv] + ([dbias.float()] if c["buckets"] else [])


# ---- 64 bits, from the definition

def exact(case, seed):
    s = _inputs(case, seed)
    op, k, v = case["op"], s["k"].double(), s["v"].double()
    if op.startswith("cache"):
        k, v = (_exact_held(x, case["fmt"]) for x in (k, v))
        if op != "cache_attend":
            return k, v
    H, Hk, nb, dev = case["heads"], case["kv_heads"], case["buckets"], k.device
    hist_pos = s["pos"] if op == "cache_attend" else s["hist_pos"]
    q = s["q"].double()
    out, dq, dk, dv = (torch.zeros_like(x) for x in (q, q, k, v))
    dbias = torch.zeros((H, nb), dtype=torch.float64, device=dev)
    edges = torch.tensor(s["edges"], device=dev) if nb else None
    for r in range(case["requests"]):
        t0, t1, j0, j1 = s["toff"][r], s["toff"][r + 1], s["hoff"][r], s["hoff"][r + 1]
        hidden = torch.zeros((t1 - t0, j1 - j0), dtype=torch.bool, device=dev)
        bucket = None
        if s["tgt_pos"] is not None:
            p = torch.arange(j1 - j0, device=dev) if hist_pos is None else hist_pos[j0:j1].long()
            dist = s["tgt_pos"][t0:t1].long()[:, None] - p
            if nb:
                bucket = torch.searchsorted(edges, dist.clamp(min=0), right=True)
            if case["masked"]:
                hidden = dist < 0
        for h in range(H):
            g = h // (H // Hk)
            kg, vg, qh = k[j0:j1, g], v[j0:j1, g], q[t0:t1, h]
            z = qh @ kg.T * s["scale"]
            th = torch.tanh(z / case["cap"]) if case["cap"] else None
            x = case["cap"] * th if case["cap"] else z
            if nb:
                x = x + s["bias"][h].double()[bucket]
            x = x.masked_fill(hidden, -math.inf)
            seen = (~hidden).any(dim=1, keepdim=True)
            w = torch.softmax(torch.where(seen, x, 0.0), dim=1) * seen
            out[t0:t1, h] = w @ vg
            if op != "train":
                continue
            go = s["dout"][t0:t1, h].double()
            dx = w * (go @ vg.T - (go * out[t0:t1, h]).sum(1, keepdim=True))
            if nb:
                dbias[h].index_add_(0, bucket.reshape(-1), dx.reshape(-1))
            dz = (dx * (1 - th * th) if case["cap"] else dx) * s["scale"]
            dq[t0:t1, h] = dz @ kg
            dk[j0:j1, g] += dz.T @ qh
            dv[j0:j1, g] += w.T @ go
    if op != "train":
        return out
    return [out, dq, dk, dv] + ([dbias] if nb else [])


def _exact_held(x, fmt):
    if fmt == "bf16":
        return x.to(torch.bfloat16).double()
    top = x.abs().amax(dim=-1, keepdim=True)
    step = torch.exp2(torch.floor(torch.log2(top.clamp(min=1e-300))).clamp(min=-120) - 6)
    return (x / step).round().clamp(-127, 127) * step


# ---- what a pass cannot do without

def work(case):
    L, m = (int(x.sum()) for x in _shape(case))
    Ls, ms = _shape(case)
    pairs = int((Ls * ms).sum())
    H, Hk, dh, es = case["heads"], case["kv_heads"], case["d_head"], _ES[case["dtype"]]
    row = 2 * Hk * dh  # K and V elements of one history row
    held = 2 * Hk * (dh + 1) if case["fmt"] == "int8" else 2 * row
    op = case["op"]
    if op == "cache_write":
        return {"bytes": L * (2 * row * es + 2 * held), "flops": 4 * L * row}
    if op == "cache_read":
        return {"bytes": L * (row * es + held), "flops": L * row}
    places = 4 * (m + (L if case["pos"] == "time" else 0)) if case["buckets"] or case["masked"] else 0
    table = 4 * H * case["buckets"]
    if op == "cache_attend":
        return {"bytes": L * held + 2 * m * H * dh * es + places + table, "flops": 4 * pairs * H * dh}
    if op == "forward":
        return {"bytes": (L * row + 2 * m * H * dh) * es + places + table, "flops": 4 * pairs * H * dh}
    return {"bytes": (2 * L * row + 4 * m * H * dh) * es + places + 2 * table, "flops": 14 * pairs * H * dh}
