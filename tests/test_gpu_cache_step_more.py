"""More of the whole-number calls of a step: trees of odd word counts, plans over several workgroups' shares with empty sequences,
missing blocks and too little room, and the outputs that a step allocates itself."""
import numpy as np
import pytest

import test_gpu_cache_step as base
from test_gpu_cache_step import dn, host, ints  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seed,rows,words,extra", [(21, [70, 96, 5], 3, 1), (22, [160, 33], 5, 0), (23, [1, 224, 2], 7, 4), (24, [993, 20], 31, 2)])
@pytest.mark.parametrize("shape", ["random", "chain", "bad"])
def test_tree_mask_of_odd_words(dn, seed, rows, words, extra, shape):
    base.test_tree_mask(dn, seed, rows, words, extra, shape)


def walk(seed, counts, breaks):
    """A block table whose walk has runs of about `breaks` blocks, its ids, and the pool's size."""
    rng = np.random.default_rng(seed)
    total = int(np.sum(counts))
    cuts = np.flatnonzero(rng.random(total) < 1.0 / breaks)
    pieces = np.split(np.arange(total), cuts)
    ids = np.concatenate([pieces[i] for i in rng.permutation(len(pieces))]) if total else np.zeros(0, dtype=int)
    table = np.full((len(counts), max(counts) + 1), -1)
    at = 0
    for s, n in enumerate(counts):
        table[s, :n] = ids[at:at + n]
        at += n
    return table, total + 3


@pytest.mark.parametrize("seed,counts,breaks", [
    (1, [0, 0, 2047, 0, 1, 0, 2048, 3], 5), (2, [700, 0, 1, 650, 700, 699, 1500, 2, 0], 40), (3, [1] * 3000 + [0] * 50 + [2] * 700, 3),
    (4, [511, 1, 512, 513, 1023, 1, 1025, 2049], 1e9), (5, [9000], 1.01)])
def test_plan_over_many_shares(dn, seed, counts, breaks):
    table, n_pool = walk(seed, counts, breaks)
    bt, total = 4, sum(counts)
    want = dn.deinfer_kv_compact_plan(table, np.array(counts), n_pool, total + 2, bt)
    tokens = ints(np.array(counts) * bt)
    got = dn.deinfer_kv_compact_plan_device(ints(table), tokens, n_pool, total + 2, bt)
    for g, w in zip(got, want):
        assert np.array_equal(host(g), w)
    runs = int(host(got[0])[0])
    if runs > 1:
        short = dn.deinfer_kv_compact_plan_device(ints(table), tokens, n_pool, total + 2, bt, capacity_runs=runs - 1)
        assert host(short[0])[:4].tolist() == [0, 0, 8, 0] and np.array_equal(host(short[1]), want[1])
    exact = dn.deinfer_kv_compact_plan_device(ints(table), tokens, n_pool, total, bt, capacity_runs=runs)
    assert host(exact[0])[:4].tolist() == [runs, total, 0, 0]


@pytest.mark.parametrize("at", [0, 1, 2047, 2048, 2049, 4500, 5999])
@pytest.mark.parametrize("bad", [-1, 1 << 30])
def test_plan_with_a_missing_block(dn, at, bad):
    counts = [1500, 0, 2500, 2000]
    table, n_pool = walk(7, counts, 30)
    remap = dn.deinfer_kv_compact_plan(table, np.array(counts), n_pool, 6000, 2)[1].reshape(table.shape).copy()
    s = int(np.searchsorted(np.cumsum(counts), at, side="right"))
    page = at - int(np.sum(counts[:s]))
    table[s, page], remap[s, page] = bad, -1
    got = dn.deinfer_kv_compact_plan_device(ints(table), ints(np.array(counts) * 2), n_pool, 6000, 2)
    assert host(got[0])[:4].tolist() == [0, 0, 1, 0]
    assert np.array_equal(host(got[1]).reshape(table.shape), remap)


@pytest.mark.parametrize("n,rows", [(0, 1), (1, 1), (2, 5), (3, 8), (4, 7), (5, 13), (8, 16)])
def test_outputs_that_a_step_allocates(dn, n, rows):
    import torch
    cached, new = ints(np.arange(n) * 5), ints(np.ones(n))
    free = ints(np.arange(40))
    tables = [torch.full((n, 12), 2, dtype=torch.int32, device="cuda") for _ in range(2)]
    got = dn.deinfer_kv_step(cached, new, tables[0], free, 4, 40, rows)
    z = lambda k: torch.zeros(k, dtype=torch.int32, device="cuda")
    want = dn.deinfer_kv_step(cached, new, tables[1], free, 4, 40, rows, out=dn.KvStep(z(n + 1), z(rows), z(rows), z(4)))
    assert [tuple(t.shape) for t in got] == [(n + 1,), (rows,), (rows,), (4,)]
    assert all(torch.equal(g, w) for g, w in zip(got, want)) and torch.equal(*tables)
    assert got.slots.data_ptr() % 16 == 0 and got.positions.data_ptr() % 16 == 0


@pytest.mark.parametrize("shift", [0, 1, 2, 3])
@pytest.mark.parametrize("spare", [0, 1, 2, 5])
def test_plan_at_any_word(dn, shift, spare):
    """The plan may begin at any word: every word of it is written, none beside it."""
    import torch
    counts = [30, 0, 11]
    table, n_pool = walk(9, counts, 4)
    want = dn.deinfer_kv_compact_plan(table, np.array(counts), n_pool, 41 + spare, 2)
    n = len(want[0])
    room = torch.full((n + 8,), 55, dtype=torch.int32, device="cuda")
    out = (room[shift:shift + n], torch.zeros(table.shape, dtype=torch.int32, device="cuda"), torch.zeros((41 + spare) * 2, dtype=torch.int32, device="cuda"))
    got = dn.deinfer_kv_compact_plan_device(ints(table), ints(np.array(counts) * 2), n_pool, 41 + spare, 2, out=out)
    for g, w in zip(got, want):
        assert np.array_equal(host(g), w)
    assert bool((room[:shift] == 55).all()) and bool((room[shift + n:] == 55).all())
