"""Rows from ids and a table's gradient on the GPU against the float64 oracle: runs
that end at and cross every border of the division, ids without a row, dense and
sparse results, rows that are not to be touched."""
import numpy as np
import pytest

from layers_common import rounded, strided, worst
from oracle import layers_oracle as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available(), "GPU tests need a GPU"
    return t


def ids_of(torch, a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


# ---- rows from ids

@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("n,d,rows", [
    (1, 8, (1,)), (1, 256, (200,)), (40, 256, (1000,)), (3, 24, (5, 7)), (257, 200, (30, 1, 9)), (1000, 64, (64,) * 8),
    (33, 520, (100, 4)), (5, 1032, (11, 3)), (19, 4096, (6,)), (7, 8192, (4, 2)), (4099, 40, (50, 2000))])
def test_rows(torch, n, d, rows, dtype, out):
    from paper_2511_06077_amd.layers import EmbeddingSum
    rng = np.random.default_rng([n, d, len(rows)])
    t, f = zip(*(rounded(torch, rng.standard_normal((r, d)), dtype) for r in rows))
    ids = [rng.integers(-1, r, size=n) for r in rows]
    ids[0][n // 2] = -2 ** 31
    scale = float(np.float32(d ** 0.5))
    e = EmbeddingSum(rows, d, scale=scale, dtype=t[0].dtype, out_dtype=torch.bfloat16 if out == "bf16" else torch.float32)
    got = e.forward(t, [ids_of(torch, i) for i in ids])
    ref, mag = O.embed(f, ids, scale)
    assert e.device_status() == 0
    assert worst(got, ref, (len(rows) + 1) * O.U * mag, out) <= 1.0
    wide = torch.full((n, d + 16), 7.0, dtype=got.dtype, device="cuda")
    e.forward([strided(torch, x) for x in t], [ids_of(torch, i) for i in ids], out=wide[:, 8:8 + d])
    assert torch.equal(wide[:, 8:8 + d], got) and bool((wide[:, :8] == 7).all()) and bool((wide[:, 8 + d:] == 7).all())


def test_ids_behind_the_table(torch):
    """They are no rows, and the status says so until it is cleared."""
    from paper_2511_06077_amd import stca
    from paper_2511_06077_amd.layers import EmbeddingSum
    t = torch.randn((10, 64), device="cuda")
    e = EmbeddingSum(10, 64, dtype=torch.float32, out_dtype=torch.float32)
    good = e.forward(t, ids_of(torch, [3, -1, 9]))
    assert e.device_status() == 0 and torch.equal(good, torch.stack([t[3], 0 * t[0], t[9]]))
    assert torch.equal(e.forward(t, ids_of(torch, [3, 10, 2 ** 31 - 1])), torch.stack([t[3], 0 * t[0], 0 * t[0]]))
    assert e.device_status() == stca.STCA_ERR_INVALID_ARG
    e.forward(t, ids_of(torch, [1]))
    assert e.device_status() == stca.STCA_ERR_INVALID_ARG
    e.clear_status()
    assert e.device_status() == 0
    assert e.forward(t, ids_of(torch, [])).shape == (0, 64)


def test_odd_values_stay_in_their_rows(torch):
    from paper_2511_06077_amd.layers import EmbeddingSum
    t = torch.randn((4, 32), device="cuda")
    t[0], t[2, 5], t[3, 1] = float("nan"), float("inf"), 3e38
    got = EmbeddingSum((4, 4), 32, dtype=torch.float32, out_dtype=torch.float32).forward(
        (t, t), (ids_of(torch, [1, -1, 2, 0, 3]), ids_of(torch, [-1, 1, 1, 1, -1])))
    assert torch.equal(got[0], t[1]) and torch.equal(got[1], t[1]) and torch.equal(got[4], t[3])
    assert torch.isinf(got[2, 5]) and torch.isfinite(got[2, :5]).all() and torch.isnan(got[3]).all()


# ---- the gradient

def runs(*lengths):
    """Ids of runs of these lengths, in an order that is not theirs."""
    ids = np.repeat(np.arange(len(lengths)) * 3 + 1, lengths)
    return np.random.default_rng(len(ids)).permutation(ids)


GRADS = {
    "one": ([5], 6, 64),
    "one_of_one_row": ([0], 1, 8),
    "none_has_a_row": ([-1, -7, -1], 10, 64),
    "all_the_same": ([3] * 1000, 5, 64),
    "all_different": (np.random.default_rng(1).permutation(1000), 1000, 32),
    "team_borders": (runs(31, 1, 32, 33, 64, 63, 65, 1, 1, 95), 100, 256),
    "workgroup_borders": (runs(255, 1, 256, 257, 512, 1, 1023, 2, 30), 40, 256),
    "through_workgroups": (runs(10, 1500, 300, 1, 700), 40, 256),
    "small_limit": (np.random.default_rng(2).integers(0, 50, 4096), 50, 16),
    "above_small": (np.random.default_rng(3).integers(-1, 300, 4097), 300, 24),
    "long_runs": (np.random.default_rng(4).integers(0, 3, 70001), 3, 256),
    "long_and_short": (np.where(np.arange(40000) % 3 == 0, 17, np.random.default_rng(5).integers(-2, 30000, 40000)), 30000, 64),
    "narrow": (np.random.default_rng(6).integers(0, 700, 30000), 700, 8),
    "wide": (np.random.default_rng(7).integers(0, 40, 900), 40, 1000),
    "widest": (np.random.default_rng(8).integers(0, 9, 300), 9, 8192),
    # more workgroups than the card holds at once, of fewer tokens than threads
    "many_workgroups": (np.random.default_rng(10).zipf(1.2, 300000) % 100000, 100000, 136),
    "many_workgroups_256": (np.random.default_rng(11).integers(-1, 30000, 270000), 30000, 256),
    # several tiles a sorting workgroup
    "several_tiles": (np.random.default_rng(12).integers(-1, 70000, 1300001), 70000, 8),
    "several_tiles_one_id": (np.full(1100000, 2), 3, 16),
    "digits_255": (np.random.default_rng(9).integers(0, 255, 5000), 255, 16),
    "digits_256": (np.random.default_rng(9).integers(0, 256, 5000), 256, 16),
    "digits_65536": (np.random.default_rng(9).integers(0, 65536, 9000), 65536, 16),
}


def depth(k):
    """Additions in a row behind one another: 32 tokens of a team, 64 teams, and that
    again in at most three levels; a sum of fewer has no more."""
    return (np.minimum(k, 3 * (32 + 64)) + 2)[:, None] * O.U


def sparse_check(torch, got, want, dtype_rows=None):
    rows, values, count = got
    ids, ref, mag, k = want
    assert int(count) == len(ids)
    assert np.array_equal(rows.cpu().numpy()[:len(ids)], ids)
    assert worst(values[:len(ids)], ref, depth(k) * mag, "f32") <= 1.0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", list(GRADS))
def test_gradient(torch, name, dtype):
    from paper_2511_06077_amd.layers import EmbeddingGradient
    ids, rows, d = GRADS[name]
    ids = np.asarray(ids)
    rng = np.random.default_rng(len(ids))
    t, f = rounded(torch, rng.standard_normal((len(ids), d)), dtype)
    scale = float(np.float32(0.3))
    want = O.embed_grad([(ids, f)], rows, scale)
    g = EmbeddingGradient(rows, len(ids), d, scale=scale, dtype=t.dtype)
    parts = [(ids_of(torch, ids), t)]
    got = g.sparse(parts)
    assert g.device_status() == 0
    sparse_check(torch, got, want)
    n = len(want[0])
    dense = g.dense(parts)
    assert torch.equal(dense[torch.from_numpy(want[0]).cuda()], got[1][:n])
    rest = torch.ones(rows, dtype=torch.bool)
    rest[torch.from_numpy(want[0])] = False
    assert bool((dense[rest.cuda()] == 0).all())
    again = g.sparse(parts)
    assert torch.equal(again[1][:n], got[1][:n])
    if len(ids) > 2:  # in three parts, one of them empty, strided rows
        a = len(ids) // 3
        three = [(parts[0][0][:a], strided(torch, t[:a])), (parts[0][0][:0], t[:0]), (parts[0][0][a:].contiguous(), t[a:])]
        split = g.sparse(three)
        assert torch.equal(split[1][:n], got[1][:n]) and int(split[2]) == n


def test_ids_of_the_largest_tables(torch):
    from paper_2511_06077_amd.layers import EmbeddingGradient
    rows = 2 ** 31 - 2 ** 16
    for n in (77, 6000):
        rng = np.random.default_rng(n)
        ids = np.concatenate([rng.integers(0, rows, n - 4), [rows - 1, rows - 1, 0, 1 << 24]])
        t, f = rounded(torch, rng.standard_normal((n, 16)), "f32")
        g = EmbeddingGradient(rows, n, 16)
        sparse_check(torch, g.sparse([(ids_of(torch, ids), t)]), O.embed_grad([(ids, f)], rows, 1.0))
        assert g.device_status() == 0


def test_what_lies_behind_is_left(torch):
    """Rows behind the count, a dense table's other columns, and, added to, its other
    rows; ids behind the table are reported and left out."""
    from paper_2511_06077_amd import stca
    from paper_2511_06077_amd.layers import EmbeddingGradient
    for n in (700, 9000):
        rng = np.random.default_rng(n)
        ids = rng.integers(0, 50, n)
        t, f = rounded(torch, rng.standard_normal((n, 72)), "bf16")
        want = O.embed_grad([(ids, f)], 1000, 1.0)
        g = EmbeddingGradient(1000, 10000, 72, dtype=torch.bfloat16)
        out = (torch.full((1001,), 77, dtype=torch.int32, device="cuda"), torch.full((1001, 72), 7.0, device="cuda"),
               torch.full((1,), 77, dtype=torch.int32, device="cuda"))
        sparse_check(torch, g.sparse([(ids_of(torch, ids), t)], out=out), want)
        assert bool((out[0][50:] == 77).all()) and bool((out[1][50:] == 7).all())
        wide = torch.full((1000, 80), 7.0, device="cuda")
        g.dense([(ids_of(torch, ids), t)], out=wide[:, 4:76])
        assert torch.equal(wide[:50, 4:76], out[1][:50]) and bool((wide[50:, 4:76] == 0).all())
        assert bool((wide[:, :4] == 7).all()) and bool((wide[:, 76:] == 7).all())
        wide.fill_(7.0)
        g.dense([(ids_of(torch, ids), t)], out=wide[:, 4:76], accumulate=True)
        # one addition, rounded
        assert worst(wide[:50, 4:76], 7.0 + want[1], depth(want[3]) * want[2], "f32") <= 1.0
        assert bool((wide[50:] == 7).all())
        bad = ids.copy()
        bad[5] = 1000
        t2, bad_ref = g.sparse([(ids_of(torch, bad), t)]), O.embed_grad([(bad, f)], 1000, 1.0)
        assert g.device_status() == stca.STCA_ERR_INVALID_ARG
        sparse_check(torch, t2, bad_ref)
        g.sparse([(ids_of(torch, ids), t)])
        assert g.device_status() == 0


def test_no_ids(torch):
    from paper_2511_06077_amd.layers import EmbeddingGradient
    g = EmbeddingGradient(9, 0, 16)
    none = [(ids_of(torch, []), torch.empty((0, 16), device="cuda"))]
    rows, values, count = g.sparse(none)
    assert rows.shape == (0,) and values.shape == (0, 16) and int(count) == 0
    assert torch.equal(g.dense(none, out=torch.full((9, 16), 3.0, device="cuda")), torch.zeros((9, 16), device="cuda"))
    kept = torch.full((9, 16), 3.0, device="cuda")
    assert bool((g.dense(none, out=kept, accumulate=True) == 3).all())


def test_odd_values_stay_in_their_gradients(torch):
    from paper_2511_06077_amd.layers import EmbeddingGradient
    for n in (600, 20000):
        ids = np.arange(n) % 6 - 1
        t = torch.ones((n, 32), device="cuda")
        t[torch.from_numpy(ids == 2).cuda()] = float("nan")
        t[torch.from_numpy(ids == -1).cuda()] = float("nan")
        t[4, 3] = float("inf")  # id 3
        rows, values, count = EmbeddingGradient(5, n, 32).sparse([(ids_of(torch, ids), t)])
        assert int(count) == 5 and torch.isnan(values[2]).all() and torch.isinf(values[3, 3])
        k = torch.from_numpy(np.bincount(ids[ids >= 0], minlength=5)).float().cuda()
        for r in (0, 1, 4):
            assert bool((values[r] == k[r]).all())


@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("fields", [4, 5, 6, 7])
@pytest.mark.parametrize("n,d", [(1, 64), (333, 264)])
def test_fields_of_several_groups(torch, n, d, fields, dtype, out):
    """Four fields are looked up together; of more, what is left after them."""
    from paper_2511_06077_amd.layers import EmbeddingSum
    rng = np.random.default_rng([n, d, fields])
    rows = tuple(int(r) for r in rng.integers(1, 40, size=fields))
    t, f = zip(*(rounded(torch, rng.standard_normal((r, d)), dtype) for r in rows))
    ids = [rng.integers(-1, r, size=n) for r in rows]
    e = EmbeddingSum(rows, d, scale=0.5, dtype=t[0].dtype, out_dtype=torch.bfloat16 if out == "bf16" else torch.float32)
    ref, mag = O.embed(f, ids, 0.5)
    assert worst(e.forward(t, [ids_of(torch, i) for i in ids]), ref, (fields + 1) * O.U * mag, out) <= 1.0
    assert e.device_status() == 0
    ids[-1][n - 1] = rows[-1]  # (an id behind the last table)
    ref, mag = O.embed(f, ids, 0.5)
    assert worst(e.forward(t, [ids_of(torch, i) for i in ids]), ref, (fields + 1) * O.U * mag, out) <= 1.0
    assert e.device_status() != 0


@pytest.mark.parametrize("d,dtype", [(256, "f32"), (520, "bf16"), (8, "bf16"), (64, "f32")])
def test_rows_of_later_turns(torch, d, dtype):
    """More rows than 32 workgroups a CU take at once, of four rows a team: exact, with one
    field; with five, what a call of those rows alone gives."""
    from paper_2511_06077_amd.layers import EmbeddingSum
    pieces = d // (4 if dtype == "f32" else 8)
    lanes = min(64, max(8, 1 << (pieces - 1).bit_length()))
    first = 32 * torch.cuda.get_device_properties(0).multi_processor_count * (256 // lanes) * 4
    n = first + 9001
    gen = torch.Generator(device="cuda").manual_seed(d)
    rows = (1000, 3, 77, 1, 500)
    kind = torch.bfloat16 if dtype == "bf16" else torch.float32
    tables = [torch.randn((r, d), generator=gen, device="cuda").to(kind) for r in rows]
    ids = [torch.randint(-1, r, (n,), generator=gen, device="cuda").int() for r in rows]
    got = EmbeddingSum(rows[0], d, dtype=kind, out_dtype=kind).forward(tables[0], ids[0])
    want = torch.where((ids[0] >= 0)[:, None], tables[0][ids[0].clamp(min=0).long()], 0)
    assert torch.equal(got, want)
    del want
    e = EmbeddingSum(rows, d, scale=0.3, dtype=kind, out_dtype=kind)
    got = e.forward(tables, ids)
    for at in (slice(0, first // 2), slice(first // 2, first), slice(first, n)):
        assert torch.equal(got[at], e.forward(tables, [i[at] for i in ids]))
    assert e.device_status() == 0
