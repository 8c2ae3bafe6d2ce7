"""The operators between ids, rows and gradients, as cases to be timed.

What a training or serving program has around the target-to-history attention:

  embed      rows from ids: out_i = scale sum_f T_f[id_f(i)], no row for a
             negative id
  grad       the gradient of one table, over one or several parts (the history's
             and the targets' ids) that share it: dT[v] = scale sum_{id(i) = v} dout_i,
             dense, or sparse as the distinct ids in ascending order, their rows
             and their number
  norm       the norms around a block with its gate and residual scale, forward
             ("norm") or forward and backward ("norm_train"):
               t = post(o) act(g);  h = x + scale ls t;  y = pre(h)
             post, pre: rms or layer norms with weights (and biases), act: sigmoid
             or silu; everything but x and pre may be absent
  clip       the norm of all gradients together, and every one times
             min(1, max_norm / norm), into other buffers; a sparse gradient counts
             as far as its number of rows says

A case is a dict of plain values, every size among them; the seed given to
prepare() draws the values.
"""
import math

import numpy as np
import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_ES = {"bf16": 2, "f32": 4}


def _embed(name, n, d, tables, *, dtype="bf16", out="bf16", ids="zipf", pad=0.0):
    return {"name": name, "op": "embed", "n": n, "d": d, "tables": tables, "dtype": dtype, "out": out, "ids": ids,
            "pad": pad}


def _grad(name, n, d, rows, *, dtype="f32", ids="zipf", form="sparse", pad=0.0):
    return {"name": name, "op": "grad", "n": n, "d": d, "rows": rows, "dtype": dtype, "ids": ids, "form": form,
            "pad": pad}


def _norm(name, n, d, *, train=True, dtype="bf16", kind="rms", block=True, gate="sigmoid", post=True, vector=True,
          biases=False):
    return {"name": name, "op": "norm_train" if train else "norm", "n": n, "d": d, "dtype": dtype, "kind": kind,
            "block": block, "gate": gate, "post": post, "vector": vector, "biases": biases}


def _clip(name, sizes, *, rows=0, d=256, used=0.0, out="f32", sigma=0.01, max_norm=1.0):
    return {"name": name, "op": "clip", "sizes": sizes, "rows": rows, "d": d, "used": used, "out": out, "sigma": sigma,
            "max_norm": max_norm}


# the gradients of four layers of 256 features, stacked: wq, wk, wv, wo, w1, w2
_STACK = "262144,262144,262144,262144,1048576,1048576"


def listed():
    return [
        # one page of candidates of one user looked up as they arrive: latency
        _embed("embed_page", 40, 256, "200000"),
        # the training window's history rows, 256 x 2048: item, action and
        # position summed, fp32 tables to the bf16 rows that the layers take
        _embed("embed_window", 524288, 256, "1000000,16,2048", dtype="f32"),
        # a parity or debugging run's gradient: 4 requests of 256 rows, 4 targets
        _grad("grad_small", "1024,16", 64, 5000),
        # the item table's gradient at the training window: history rows and targets
        # share it, ids as traffic has them (few are frequent, most are rare)
        _grad("grad_items", "524288,4096", 256, 1000000),
        # the action table's: every row of it is looked up tens of thousands of times
        _grad("grad_actions", "524288", 256, 16, dtype="bf16", ids="uniform", form="dense"),
        # the norm in front of a layer for a few targets in fp32: latency
        _norm("norm_small", 16, 64, train=False, dtype="f32", kind="layer", block=False, gate="", post=False,
              vector=False, biases=True),
        # the training window's rows normalised for the projections of K and V
        _norm("norm_window", 524288, 256, train=False, block=False, gate="", post=False, vector=False),
        # a training step of a block over them: post norm, gate, scaled residual, next norm
        _norm("norm_train_window", 524288, 256),
        # wide rows of an odd number, layer norms with biases, a SiLU gate
        _norm("norm_train_wide", 8191, 2000, kind="layer", gate="silu", biases=True),
        # a small model's gradients: many tensors, small and odd
        _clip("clip_small", "64,64,4096,4096,1,4097,333,16384,16384,999,64,64,4096,4096,7,4097,333,16384,16384,5"),
        # the four-layer stack's
        _clip("clip_stack", _STACK),
        # a whole step's: the stack, a position table, norms' weights, and the item
        # table's sparse rows, of which some are used; attention's in bf16
        _clip("clip_step", _STACK + ",524288,256,256,256,256,4096,b1048576,b1048576,b524288", rows=528384, used=0.4),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the listed ranges (rng: random.Random)."""
    op = rng.choice(["embed", "grad", "grad", "norm", "norm_train", "norm_train", "clip"])
    if op == "clip":
        n = _log_int(rng, 1, 48)
        top = _log_int(rng, 64, 4000000)
        sizes = ",".join(rng.choice(["", "", "b"]) + str(_log_int(rng, 1, top)) for _ in range(n))
        rows = rng.choice([0, 0, _log_int(rng, 1, 200000)])
        return {"op": "clip", "sizes": sizes, "rows": rows, "d": 8 * rng.randrange(1, 33), "used": rng.random(),
                "out": rng.choice(["f32", "same"]), "sigma": 0.01, "max_norm": rng.choice([0.05, 1.0, 1e6])}
    d = 8 * rng.choice([rng.randrange(1, 65), 8, 16, 32, _log_int(rng, 1, 256)])
    n = _log_int(rng, 1, max(1, min(2000000, 100000000 // d)))
    if op == "embed":
        tables = ",".join(str(_log_int(rng, 1, min(2000000, 250000000 // d))) for _ in range(rng.randrange(1, 5)))
        return {"op": "embed", "n": n, "d": d, "tables": tables, "dtype": rng.choice(["bf16", "f32"]),
                "out": rng.choice(["bf16", "f32"]), "ids": rng.choice(["zipf", "uniform"]),
                "pad": rng.choice([0.0, 0.0, 0.1])}
    if op == "grad":
        parts = [n] if n == 1 or rng.random() < 0.5 else [n - n // 8 - 1, n // 8 + 1]
        form = rng.choice(["sparse", "dense"])
        rows = _log_int(rng, 1, 20000000 if form == "sparse" else min(1000000, 100000000 // d))
        return {"op": "grad", "n": ",".join(str(p) for p in parts if p), "d": d, "rows": rows,
                "dtype": rng.choice(["bf16", "f32"]), "ids": rng.choice(["zipf", "uniform"]), "form": form,
                "pad": rng.choice([0.0, 0.0, 0.1])}
    block = rng.random() < 0.75
    return {"op": op, "n": n, "d": d, "dtype": rng.choice(["bf16", "bf16", "f32"]),
            "kind": rng.choice(["rms", "layer"]), "block": block,
            "gate": rng.choice(["", "sigmoid", "silu"]) if block else "", "post": block and rng.random() < 0.7,
            "vector": block and rng.random() < 0.5, "biases": rng.random() < 0.4}


# ---- inputs

def _gen(seed, salt):
    return torch.Generator(device="cuda").manual_seed(seed * 1000003 + salt)


def _normal(gen, shape, dtype, sigma=1.0):
    return (sigma * torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)).to(dtype)


def _some_ids(gen, n, rows, how, pad):
    """int32 ids: uniform, or p(rank) falling as 1 / rank over a shuffled table;
    a part of them -1 (no row)."""
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    if how == "zipf":
        rank = (torch.exp(u * math.log(rows + 1.0)) - 1.0).long().clamp(0, rows - 1)
        ids = torch.randperm(rows, generator=gen, device="cuda")[rank]
    else:
        ids = (u * rows).long().clamp(0, rows - 1)
    if pad:
        ids = torch.where(torch.rand(n, generator=gen, device="cuda") < pad, -1, ids)
    return ids.to(torch.int32)


def _numbers(text):
    return [int(x) for x in text.split(",")]


def _inputs(case, seed):
    """Everything the call is given, on the GPU."""
    gen, s, op = _gen(seed, 17), {"case": case}, case["op"]
    if op == "embed":
        rows, d = _numbers(case["tables"]), case["d"]
        s["scale"] = math.sqrt(d)
        s["tables"] = [_normal(gen, (v, d), _DT[case["dtype"]], 1.0 / math.sqrt(d)) for v in rows]
        s["ids"] = [_some_ids(gen, case["n"], v, case["ids"], case["pad"]) for v in rows]
    elif op == "grad":
        s["scale"] = math.sqrt(case["d"])
        s["parts"] = [(_some_ids(gen, n, case["rows"], case["ids"], case["pad"]),
                       _normal(gen, (n, case["d"]), _DT[case["dtype"]])) for n in _numbers(case["n"])]
    elif op == "clip":
        s["grads"] = [_normal(gen, (int(x.lstrip("b")),), _DT["bf16" if x[0] == "b" else "f32"], case["sigma"])
                      for x in case["sizes"].split(",")]
        s["counts"] = [None] * len(s["grads"])
        if case["rows"]:
            s["grads"].append(_normal(gen, (case["rows"], case["d"]), torch.float32, case["sigma"]))
            s["counts"].append(torch.tensor([_used(case)], dtype=torch.int32, device="cuda"))
    else:
        n, d, dt = case["n"], case["d"], _DT[case["dtype"]]
        rows = ["x"] + (["block"] if case["block"] else []) + (["gate"] if case["gate"] else [])
        rows += ["dh", "dy"] if op == "norm_train" else []
        for name in ("x", "block", "gate", "dh", "dy"):
            s[name] = _normal(gen, (n, d), dt) if name in rows else None
        def vec(there, middle, sigma):
            return middle + _normal(gen, (d,), torch.float32, sigma) if there else None
        s["pre"] = (vec(True, 1.0, 0.1), vec(case["biases"], 0.0, 0.1))
        s["post"] = (vec(case["post"], 1.0, 0.1), vec(case["post"] and case["biases"], 0.0, 0.1))
        s["ls"] = vec(case["vector"], 0.5, 0.1)
        s["scale"], s["eps"] = 0.7, 1e-6
    return s


def _used(case):
    return int(case["rows"] * case["used"])


def prepare(case, seed):
    s, op = _inputs(case, seed), case["op"]
    if op == "grad" and case["form"] == "sparse":
        n = sum(_numbers(case["n"]))
        cap = min(n, case["rows"])
        # the program's own buffers, kept from step to step: rows behind the last
        # distinct id stay as they are
        s["out"] = (torch.zeros(cap, dtype=torch.int32, device="cuda"),
                    torch.zeros((cap, case["d"]), dtype=torch.float32, device="cuda"),
                    torch.zeros(1, dtype=torch.int32, device="cuda"))
    if op == "clip":
        s["out"] = [torch.zeros_like(g, dtype=torch.float32 if case["out"] == "f32" else g.dtype) for g in s["grads"]]
    if own:
        from paper_2511_06077_amd.layers import BlockNorm, EmbeddingGradient, EmbeddingSum, GradientNorm
        if op == "embed":
            s["plan"] = EmbeddingSum(_numbers(case["tables"]), case["d"], scale=s["scale"], dtype=_DT[case["dtype"]],
                                     out_dtype=_DT[case["out"]])
        elif op == "grad":
            s["plan"] = EmbeddingGradient(case["rows"], sum(_numbers(case["n"])), case["d"], scale=s["scale"],
                                          dtype=_DT[case["dtype"]])
        elif op == "clip":
            s["plan"] = GradientNorm(case["max_norm"])
        else:
            s["plan"] = BlockNorm(case["d"], kind=case["kind"], gate=case["gate"] or None, scale=s["scale"],
                                  eps=s["eps"], dtype=_DT[case["dtype"]], backward=op == "norm_train")
    return s


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    op, plan = s["case"]["op"], s["plan"]
    if op == "embed":
        return plan.forward(s["tables"], s["ids"])
    if op == "grad":
        return plan.dense(s["parts"]) if s["case"]["form"] == "dense" else plan.sparse(s["parts"], out=s["out"])
    if op == "clip":
        return [plan.clip(s["grads"], out=s["out"], counts=s["counts"])] + s["out"]
    given = dict(block=s["block"], gate=s["gate"], pre=s["pre"], post=s["post"] if s["case"]["post"] else None,
                 layer_scale=s["ls"])
    h, y = plan.forward(s["x"], **given)
    if op == "norm":
        return [h, y] if s["case"]["block"] else [y]
    g = plan.backward(s["dy"], s["x"], dh=s["dh"], **given)
    out = [h, y] if s["case"]["block"] else [y]
    return out + [t for t in (g.x, g.block, g.gate, *g.pre, *g.post, g.layer_scale) if t is not None]


# ---- plain form

def _run_plain(s):
    op = s["case"]["op"]
    if op == "embed":
        return _plain_embed(s)
    if op == "grad":
        return _plain_grad(s)
    if op == "clip":
        return _plain_clip(s)
    return _plain_norm(s)


def _plain_embed(s):
    out = 0.0
    for table, ids in zip(s["tables"], s["ids"]):
        rows = table[ids.clamp(min=0).long()].float()
        out = out + rows * (ids >= 0)[:, None]
    return (out * s["scale"]).to(_DT[s["case"]["out"]])


def _plain_grad(s):
    c = s["case"]
    ids = torch.cat([p[0] for p in s["parts"]]).long()
    dout = torch.cat([p[1] for p in s["parts"]]).float()
    there = ids >= 0
    ids, dout = ids[there], dout[there]
    if c["form"] == "dense":
        # (a row of a small table is a long sum)
        total = torch.zeros((c["rows"], c["d"]), dtype=torch.float64, device="cuda")
        return (total.index_add_(0, ids, dout.double()) * s["scale"]).float()
    which, at = torch.unique(ids, sorted=True, return_inverse=True)
    total = torch.zeros((which.shape[0], c["d"]), dtype=torch.float64, device="cuda")
    total.index_add_(0, at, dout.double())
    rows, grads, count = (torch.zeros_like(t) for t in s["out"])
    rows[:which.shape[0]] = which.int()
    grads[:which.shape[0]] = (total * s["scale"]).float()
    count += which.shape[0]
    return rows, grads, count


def _plain_clip(s):
    c, total, seen = s["case"], 0.0, []
    for g, count in zip(s["grads"], s["counts"]):
        x = g.float()
        if count is not None:
            live = torch.arange(g.shape[0], device="cuda") < count
            x = x * live[:, None]
        seen.append(x)
        total = total + x.double().square().sum()
    norm = total.sqrt()
    factor = torch.where(torch.isfinite(norm), (c["max_norm"] / norm).clamp(max=1.0), 1.0).float()
    return [norm.float()] + [(x * factor).to(o.dtype) for x, o in zip(seen, s["out"])]


def _plain_unit(x, kind, eps):
    if kind == "layer":
        x = x - x.mean(dim=-1, keepdim=True)
    r = torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + eps)
    return x * r, r


def _plain_affine(unit, weight, bias):
    out = unit * weight
    return out if bias is None else out + bias


def _plain_unit_grad(a, unit, r, kind):
    g = a - unit * (a * unit).mean(dim=-1, keepdim=True)
    if kind == "layer":
        g = g - a.mean(dim=-1, keepdim=True)
    return g * r


def _plain_norm(s):
    c = s["case"]
    kind, eps, dt, scale = c["kind"], s["eps"], _DT[c["dtype"]], s["scale"]
    x = h = s["x"].float()
    ls = scale if s["ls"] is None else scale * s["ls"]
    if c["block"]:
        t = n = s["block"].float()
        if c["post"]:
            ou, orr = _plain_unit(t, kind, eps)
            t = n = _plain_affine(ou, *s["post"])
        if c["gate"]:
            g = s["gate"].float()
            sig = 1.0 / (1.0 + torch.exp(-g))
            act = sig * g if c["gate"] == "silu" else sig
            t = n * act
        h = x + ls * t
    hu, hr = _plain_unit(h, kind, eps)
    y = _plain_affine(hu, *s["pre"])
    out = [h.to(dt), y.to(dt)] if c["block"] else [y.to(dt)]
    if c["op"] == "norm":
        return out
    dy = s["dy"].float()
    dh = s["dh"].float() + _plain_unit_grad(dy * s["pre"][0], hu, hr, kind)
    out.append(dh.to(dt))
    tail = [_plain_sum(dy * hu)] + ([_plain_sum(dy)] if c["biases"] else [])
    if c["block"]:
        dt_ = dn = dh * ls
        if c["gate"]:
            slope = sig * (1.0 - sig)
            dg = dt_ * n * (sig + g * slope if c["gate"] == "silu" else slope)
            dn = dt_ * act
        do = dn
        if c["post"]:
            do = _plain_unit_grad(dn * s["post"][0], ou, orr, kind)
            tail += [_plain_sum(dn * ou)] + ([_plain_sum(dn)] if c["biases"] else [])
        out.append(do.to(dt))
        if c["gate"]:
            out.append(dg.to(dt))
        if c["vector"]:
            tail.append(_plain_sum(dh * t * scale))
    return out + tail


def _plain_sum(x):
    """Sums over rows, in 64 bits: there may be millions of them."""
    return x.sum(dim=0, dtype=torch.float64).float()


# ---- 64 bits, from the definitions

def exact(case, seed):
    s, op = _inputs(case, seed), case["op"]
    if op == "embed":
        out = torch.zeros((case["n"], case["d"]), dtype=torch.float64, device="cuda")
        for table, ids in zip(s["tables"], s["ids"]):
            at = torch.nonzero(ids >= 0)[:, 0]
            for a in at.split(1 << 18):
                out[a] += table.index_select(0, ids[a].long()).double()
        return out * s["scale"]
    if op == "grad":
        return _exact_grad(case, s)
    if op == "clip":
        live = [g if n is None else g[:int(n)] for g, n in zip(s["grads"], s["counts"])]
        norm = math.sqrt(sum(float((g.double() ** 2).sum()) for g in live))
        factor = 1.0 if norm <= case["max_norm"] else case["max_norm"] / norm
        out = [torch.zeros(g.shape, dtype=torch.float64, device="cuda") for g in s["grads"]]
        for o, g in zip(out, live):
            o[:g.shape[0]] = g.double() * factor
        return [torch.tensor(norm, dtype=torch.float64)] + out
    return _exact_norm(case, s)


def _exact_grad(case, s):
    """By the order of the ids: every run of one id is a group, its rows are added in 64 bits."""
    ids = torch.cat([i for i, _ in s["parts"]]).long()
    order = torch.argsort(ids, stable=True)
    order = order[int((ids < 0).sum()):]
    held = ids[order]
    first = torch.ones_like(held, dtype=torch.bool)
    first[1:] = held[1:] != held[:-1]
    group = torch.cumsum(first, 0) - 1
    k = int(first.sum())
    sums = torch.zeros((k, case["d"]), dtype=torch.float64, device="cuda")
    rows = torch.cat([g for _, g in s["parts"]])
    for a in torch.arange(order.shape[0], device="cuda").split(1 << 18):
        sums.scatter_add_(0, group[a][:, None].expand(-1, case["d"]), rows[order[a]].double())
    sums *= s["scale"]
    if case["form"] == "dense":
        out = torch.zeros((case["rows"], case["d"]), dtype=torch.float64, device="cuda")
        out[held[first]] = sums
        return out
    cap = min(ids.shape[0], case["rows"])
    which = torch.zeros(cap, dtype=torch.int32, device="cuda")
    out = torch.zeros((cap, case["d"]), dtype=torch.float64, device="cuda")
    which[:k], out[:k] = held[first].int(), sums
    return which, out, torch.tensor([k], dtype=torch.int32)


def _exact_norm(case, s):
    """By automatic differentiation in 64 bits, a slice of the rows at a time."""
    names = ["x", "block", "gate"]
    params = [s["pre"][0], s["pre"][1], s["post"][0], s["post"][1], s["ls"]]
    train = case["op"] == "norm_train"
    p = [None if t is None else t.double().requires_grad_(train) for t in params]
    done = []
    for at in torch.arange(case["n"], device="cuda").split(max(1, (1 << 25) // case["d"])):
        rows = slice(int(at[0]), int(at[-1]) + 1)
        x, o, g = (None if s[k] is None else s[k][rows].double().requires_grad_(train) for k in names)
        h = x
        if o is not None:
            t = o if p[2] is None else _exact_unit(o, case, s["eps"]) * p[2]
            t = t if p[3] is None else t + p[3]
            if g is not None:
                t = t * torch.sigmoid(g) * (g if case["gate"] == "silu" else 1.0)
            t = t * s["scale"]
            h = x + (t if p[4] is None else t * p[4])
        y = _exact_unit(h, case, s["eps"]) * p[0]
        y = y if p[1] is None else y + p[1]
        got = [h.detach(), y.detach()] if o is not None else [y.detach()]
        if train:
            ((h * s["dh"][rows].double()).sum() + (y * s["dy"][rows].double()).sum()).backward()
            got += [t.grad for t in (x, o, g) if t is not None]
        done.append(got)
    return [torch.cat(c) for c in zip(*done)] + ([t.grad for t in p if t is not None] if train else [])


def _exact_unit(v, case, eps):
    if case["kind"] == "layer":
        var, mean = torch.var_mean(v, dim=1, correction=0, keepdim=True)
        return (v - mean) / torch.sqrt(var + eps)
    return v / torch.sqrt((v * v).mean(1, keepdim=True) + eps)


# ---- what a pass cannot do without

def _distinct(n, rows, how):
    """Expected number of different ids among n."""
    if how == "uniform":
        return rows * -math.expm1(n * math.log1p(-1.0 / rows)) if rows > 1 else min(n, 1)
    k = np.arange(1, rows + 1, dtype=np.float64)
    p = np.log1p(1.0 / k) / math.log(rows + 1.0)
    with np.errstate(divide="ignore"):
        return float(-np.expm1(n * np.log1p(-np.minimum(p, 1.0))).sum())


def work(case):
    op = case["op"]
    if op == "clip":
        sizes = [(int(x.lstrip("b")), 2 if x[0] == "b" else 4) for x in case["sizes"].split(",")]
        if case["rows"]:
            sizes.append((_used(case) * case["d"], 4))
        moved = sum(n * (es + (4 if case["out"] == "f32" else es)) for n, es in sizes)
        return {"bytes": moved + 4, "flops": 3 * sum(n for n, _ in sizes)}
    d = case["d"]
    if op == "embed":
        n, rows = case["n"], _numbers(case["tables"])
        read = sum(_distinct(n * (1 - case["pad"]), v, case["ids"]) for v in rows)
        return {"bytes": int(4 * n * len(rows) + read * d * _ES[case["dtype"]] + n * d * _ES[case["out"]]),
                "flops": n * d * (len(rows) + 1)}
    if op == "grad":
        n = sum(_numbers(case["n"]))
        kept = n * (1 - case["pad"])
        out = case["rows"] * d * 4 if case["form"] == "dense" else \
            _distinct(kept, case["rows"], case["ids"]) * (4 * d + 4)
        return {"bytes": int(4 * n + kept * d * _ES[case["dtype"]] + out), "flops": int(kept * d)}
    rows = 1 + bool(case["block"]) + bool(case["gate"])  # x, block, gate
    given, made = rows, 1 + bool(case["block"])
    if op == "norm_train":
        given, made = given + 2, made + rows
    return {"bytes": case["n"] * d * _ES[case["dtype"]] * (given + made) + 4 * d * 5,
            "flops": case["n"] * d * (40 if op == "norm_train" else 10)}
