"""The stand-alone attention at the ends of what its calls allow: device offsets
that are not the host's."""
import numpy as np
import pytest

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
