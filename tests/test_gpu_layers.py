"""The operators between ids, rows and gradients run together, as a training step
does: with the attention between them, captured into a graph, on another stream."""
import numpy as np
import pytest

from layers_common import strided

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available(), "GPU tests need a GPU"
    return t


def test_training_step(torch):
    """ids -> rows -> norm -> attention of targets over histories -> gate, residual and
    next norm, and back to the item table and the weights, clipped; fp32 storage,
    against automatic differentiation in float64."""
    from paper_2511_06077_amd.attention import CrossAttention
    from paper_2511_06077_amd.layers import BlockNorm, EmbeddingGradient, EmbeddingSum, GradientNorm
    L, m, d, H, items = [70, 1, 0, 45], [3, 2, 1, 4], 64, 2, 40
    hoff, toff = (np.concatenate([[0], np.cumsum(n)]).astype(np.int32) for n in (L, m))
    nh, nt = int(hoff[-1]), int(toff[-1])
    gen = torch.Generator().manual_seed(3)
    def normal(*shape, gain=1.0):
        return gain * torch.randn(*shape, generator=gen, dtype=torch.float32)
    table, actions = normal(items, d), normal(4, d)
    hid, aid = torch.randint(-1, items, (nh,), generator=gen), torch.randint(0, 4, (nh,), generator=gen)
    tid = torch.randint(0, items, (nt,), generator=gen)
    w = {k: normal(d, d, gain=d ** -0.5) for k in ("q", "k", "v", "g")}
    vec = {k: 1 + normal(d, gain=0.2) for k in ("in_w", "post_w", "pre_w", "ls")}
    dh, dy = normal(nt, d), normal(nt, d)

    # float64
    P = {k: v.double().requires_grad_() for k, v in {"table": table, "actions": actions, **w, **vec}.items()}
    def unit(v):
        return v / torch.sqrt((v * v).mean(1, keepdim=True) + float(np.float32(1e-6)))
    rows = (P["table"][hid.clamp(min=0)] * (hid >= 0)[:, None] + P["actions"][aid]) * 0.5
    x = P["table"][tid] * 0.5
    hn, xn = unit(rows) * P["in_w"], unit(x) * P["in_w"]
    q, k, v, gate = xn @ P["q"], hn @ P["k"], hn @ P["v"], xn @ P["g"]
    o = []
    for r in range(len(L)):
        for t in range(toff[r], toff[r + 1]):
            j = slice(hoff[r], hoff[r + 1])
            heads = []
            for h in range(H):
                c = slice(h * 32, h * 32 + 32)
                s = torch.softmax(k[j, c] @ q[t, c] * 32 ** -0.5, 0)
                heads.append(s @ v[j, c])
            o.append(torch.cat(heads))
    o = torch.stack(o)
    h_ = x + 0.7 * P["ls"] * (unit(o) * P["post_w"] * torch.sigmoid(gate))
    y_ = unit(h_) * P["pre_w"]
    ((h_ * dh).sum() + (y_ * dy).sum()).backward()

    # the GPU
    f32 = dict(dtype=torch.float32)
    G = {k: t.cuda() for k, t in {"table": table, "actions": actions, **w, **vec, "dh": dh, "dy": dy}.items()}
    hist_ids, act_ids, tgt_ids = (t.int().cuda() for t in (hid, aid, tid))
    first = BlockNorm(d, backward=True, **f32)
    block = BlockNorm(d, gate="sigmoid", scale=0.7, backward=True, **f32)
    attn = CrossAttention(hoff, toff, H, 32, backward=True, **f32)
    hist = EmbeddingSum((items, 4), d, scale=0.5, out_dtype=torch.float32, **f32).forward((G["table"], G["actions"]), (hist_ids, act_ids))
    tgt = EmbeddingSum(items, d, scale=0.5, out_dtype=torch.float32, **f32).forward(G["table"], tgt_ids)
    _, hy = first.forward(hist, pre=(G["in_w"],))
    _, ty = first.forward(tgt, pre=(G["in_w"],))
    qkv = [a @ G[n] for a, n in ((ty, "q"), (hy, "k"), (hy, "v"))]
    gate = ty @ G["g"]
    out = attn.forward(*(t.view(-1, H, 32) for t in qkv)).view(nt, d)
    given = dict(block=out, gate=gate, post=(G["post_w"],), pre=(G["pre_w"],), layer_scale=G["ls"])
    h, y = block.forward(tgt, **given)
    b = block.backward(G["dy"], tgt, dh=G["dh"], **given)
    dq, dk, dv, _ = (None if t is None else t.reshape(-1, d) for t in
                     attn.backward(b.block.view(nt, H, 32), *(t.view(-1, H, 32) for t in qkv)))
    dw = {n: a.t() @ g for n, a, g in (("q", ty, dq), ("k", hy, dk), ("v", hy, dv), ("g", ty, b.gate))}
    back_t = first.backward(dq @ G["q"].t() + b.gate @ G["g"].t(), tgt, dh=b.x, pre=(G["in_w"],))
    back_h = first.backward(dk @ G["k"].t() + dv @ G["v"].t(), hist, pre=(G["in_w"],))
    rows_, values, count = EmbeddingGradient(items, nh + nt, d, scale=0.5).sparse([(hist_ids, back_h.x), (tgt_ids, back_t.x)])
    dact = EmbeddingGradient(4, nh, d, scale=0.5).dense([(act_ids, back_h.x)])
    n = int(count)
    dtable = torch.zeros_like(G["table"])
    dtable[rows_[:n].long()] = values[:n]
    got = {**dw, "table": dtable, "actions": dact, "in_w": back_t.pre[0] + back_h.pre[0], "post_w": b.post[0],
           "pre_w": b.pre[0], "ls": b.layer_scale}
    # fp32 storage between a dozen operators whose sums have up to 200 terms: each is off by at
    # most some 200 U of its largest value, 12 * 200 * 2^-24 = 1.4e-4 together
    for name, g in list(got.items()) + [("h", h), ("y", y)]:
        want = P[name].grad if name in P else h_ if name == "h" else y_
        e = float((g.double().cpu() - want.detach()).abs().max() / want.detach().abs().max())
        print(f"[training step] {name} {e:.2e}", flush=True)
        assert e <= 1.5e-4, (name, e)
    names = [k for k in got if k not in ("table",)]
    total = np.sqrt(sum(float((P[k].grad ** 2).sum()) for k in names + ["table"]))
    norm = GradientNorm(0.5 * total).clip([got[k] for k in names] + [values], counts=[None] * len(names) + [count])
    assert abs(float(norm) / total - 1) <= 1.5e-4
    for k in names:
        e = float((got[k].double().cpu() - 0.5 * P[k].grad).abs().max() / P[k].grad.abs().max())
        assert e <= 1.5e-4, (k, e)


class Step:
    """All operators one after the other on buffers of their own."""

    def __init__(self, torch, n, d, rows):
        from paper_2511_06077_amd.layers import BlockNorm, EmbeddingGradient, EmbeddingSum, GradientNorm
        self.torch, self.n, self.d, self.rows = torch, n, d, rows
        self.embed = EmbeddingSum(rows, d, dtype=torch.float32, out_dtype=torch.bfloat16)
        self.norm = BlockNorm(d, kind="layer", gate="silu", backward=True)
        self.grad = EmbeddingGradient(rows, n, d, dtype=torch.bfloat16)
        self.dense = EmbeddingGradient(rows, n, d, dtype=torch.bfloat16)
        self.clip = GradientNorm(0.1)
        self.s = {k: torch.zeros((n, d), dtype=torch.bfloat16, device="cuda") for k in ("block", "gate", "dh", "dy")}
        self.s.update(table=torch.zeros((rows, d), device="cuda"), w=torch.zeros(d, device="cuda"),
                      ids=torch.zeros(n, dtype=torch.int32, device="cuda"))
        cap = min(n, rows)
        self.sparse = (torch.zeros(cap, dtype=torch.int32, device="cuda"), torch.zeros((cap, d), device="cuda"),
                       torch.zeros(1, dtype=torch.int32, device="cuda"))

    def fill(self, seed):
        gen = self.torch.Generator(device="cuda").manual_seed(seed)
        for k, t in self.s.items():
            if k == "ids":
                t.copy_(self.torch.randint(-1, self.rows, t.shape, generator=gen, device="cuda"))
            else:
                t.copy_(self.torch.randn(t.shape, generator=gen, device="cuda"))
        for t in self.sparse:
            t.zero_()

    def run(self, stream=None):
        s, at = self.s, dict(stream=stream)
        x = self.embed.forward(s["table"], s["ids"], **at)
        given = dict(block=s["block"], gate=s["gate"], post=(s["w"], s["w"]), pre=(s["w"], s["w"]), layer_scale=s["w"])
        h, y = self.norm.forward(x, **given, **at)
        g = self.norm.backward(s["dy"], x, dh=s["dh"], **given, **at)
        parts = [(s["ids"], g.x)]
        self.grad.sparse(parts, out=self.sparse, **at)
        dense = self.dense.dense(parts, **at)
        norm = self.clip.clip([self.sparse[1], dense, g.pre[0], g.layer_scale, g.block], counts=[self.sparse[2]] + [None] * 4, **at)
        return [x, h, y, g.x, g.block, g.gate, *g.pre, *g.post, g.layer_scale, *self.sparse, dense, norm]


@pytest.mark.parametrize("n,d,rows", [(300, 64, 50), (9000, 256, 3000), (9000, 72, 4)])
def test_graph(torch, n, d, rows):
    """Captured and replayed on new inputs, with eager work between the replays."""
    step, eager = Step(torch, n, d, rows), Step(torch, n, d, rows)
    step.fill(1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step.run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step.run()
    for seed in (2, 3, 4, 5):
        step.fill(seed), eager.fill(seed)
        want = [t.clone() for t in eager.run()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(out, want)):
            assert torch.equal(a, b), (seed, i)


def test_streams(torch):
    """Two objects' steps at the same time on streams of their own, named by their handle,
    give what they give alone."""
    a, b = Step(torch, 9000, 256, 500), Step(torch, 7001, 64, 9000)
    want = []
    for k, s in enumerate((a, b)):
        s.fill(k)
        want.append([t.clone() for t in s.run()])
        s.fill(k)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [s.run(st.cuda_stream) for s, st in zip((a, b), streams)]
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(x, y) for x, y in zip(g, w))


def test_rows_for_the_layers(torch):
    """Looked-up rows as the history and targets of the layer stack, and its gradients
    of rows (fp32) back to the table both share."""
    from paper_2511_06077_amd import workload as W
    from paper_2511_06077_amd.device import DeviceBatch, to_device
    from paper_2511_06077_amd.layers import EmbeddingGradient, EmbeddingSum, GradientNorm
    b = W.make_custom_batch("looked_up", [300, 45, 1], [5, 33, 2], d_model=256, n_heads=8, n_layers=2, dtype="bf16", seed=7,
                            with_grad=True)
    nh, nt, items = b.n_hist, b.n_tgt_total, 200
    gen = torch.Generator(device="cuda").manual_seed(0)
    table = torch.randn((items, 256), generator=gen, device="cuda")
    hid, tid = (torch.randint(0, items, (n,), generator=gen, device="cuda").int() for n in (nh, nt))
    embed = EmbeddingSum(items, 256, dtype=torch.float32)
    hist, tgt = embed.forward(table, hid), embed.forward(table, tid)
    assert torch.equal(hist, table[hid.long()].bfloat16()) and torch.equal(tgt, table[tid.long()].bfloat16())
    db = DeviceBatch.from_tensors(b, hist, tgt, {k: to_device(b.weights[k], "cuda") for k in W.WEIGHT_NAMES}, backward=True)
    db.forward()
    g = db.backward(to_device(b.grad_out, "cuda"))
    rows, values, count = EmbeddingGradient(items, nh + nt, 256).sparse([(hid, g["dhist"]), (tid, g["dtgt"])])
    want = torch.zeros((items, 256), dtype=torch.float64, device="cuda")
    mag = torch.zeros_like(want)
    for i, x in ((hid, g["dhist"]), (tid, g["dtgt"])):
        want.index_add_(0, i.long(), x.double())
        mag.index_add_(0, i.long(), x.double().abs())
    n = int(count)
    at = rows[:n].long()
    assert bool(((values[:n].double() - want[at]).abs() <= 64 * 2.0 ** -24 * mag[at]).all())  # (at most 20 rows each)
    weights = [g[k] for k in sorted(g) if k.startswith("dw")]
    total = sum(float((x.double() ** 2).sum()) for x in weights + [values[:n]]) ** 0.5
    assert abs(float(GradientNorm(1.0).clip(weights + [values], counts=[None] * len(weights) + [count])) / total - 1) <= 1e-7
