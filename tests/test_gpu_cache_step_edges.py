"""The calls of a step over the paged cache at the ends of their ranges."""
import numpy as np
import pytest

from oracle import cache_step as cs
from test_gpu_cache_step import cache_case, check_attention, dn, host, ints, normal, random_mask  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("first", [0, 3])
@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("cached,new", [([], []), ([5, 0, 40], [0, 0, 0]), ([5, 0, 40], [2, 30, 1])])
def test_a_step_without_rows(dn, cached, new, first, given):
    """row_start and counts are written: a program may carry counts[3] on as the next step's free_first."""
    import torch
    bt, n_pool, free, n = 16, 20, list(range(10, 20)), len(cached)
    table = np.arange(n * 4).reshape(n, 4) % 9
    tab = ints(table)
    z = lambda k: torch.full((k,), 77, dtype=torch.int32, device="cuda")
    junk = [z(m) for m in (4096, 64, 16)]                            # (what the next allocations are likely to hold)
    del junk
    out = dn.KvStep(z(n + 1), z(0), z(0), z(4)) if given else None
    got = dn.deinfer_kv_step(ints(cached), ints(new), tab, ints(free), bt, n_pool, 0, free_first=ints([first]) if first else None, out=out)
    want = cs.kv_step(cached, new, table, free, first, n_pool, bt, 0)
    assert host(got.row_start).tolist() == [0] * (n + 1) == want[0].tolist()
    assert host(got.counts).tolist() == want[4].tolist() == [sum(new), 0, 0, first]
    assert got.slots.numel() == 0 and got.positions.numel() == 0 and np.array_equal(host(tab), table)


@pytest.mark.parametrize("in_place", [False, True])
def test_queries_alone_with_slots(dn, in_place):
    """Without a pool beside them every slot that is not negative is one in use; a row without one is left as it is."""
    import torch
    rows, heads, D = 5, 2, 32
    q = torch.randn(rows, heads * D, device="cuda").bfloat16()
    f = torch.tensor(cs.frequencies(D, 10000.0)[0], device="cuda")
    pos, slots = ints([3, 1000, 7, 0, 99]), ints([4, 0, -1, 2 ** 31 - 1, 123456])
    want = q.clone()
    dn.deinfer_rope_store(want, None, None, pos, f, heads, 0, D)
    mine, out = q.clone(), torch.full_like(q, 3.0)
    got, k_out, v_out = dn.deinfer_rope_store(mine, None, None, pos, f, heads, 0, D, slots=slots, q_out=None if in_place else out)
    assert got is (mine if in_place else out) and k_out is None and v_out is None
    used = torch.tensor([0, 1, 3, 4], device="cuda")
    assert torch.equal(got[used], want[used]) and torch.equal(got[2], q[2] if in_place else torch.full_like(q[2], 3.0))


def test_the_calls_of_a_step_without_rows(dn):
    """Every call of a step takes a step without rows; the cache stays as it is."""
    import torch
    bt, n_pool, hq, hk, D = 16, 8, 4, 2, 64
    cached, new, table = ints([5, 20]), ints([0, 0]), ints([[0, 1, 2], [3, 4, 5]])
    step = dn.deinfer_kv_step(cached, new, table, ints([6, 7]), bt, n_pool, 0)
    pools = [torch.full((n_pool * bt, hk * D), 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    qkv = torch.zeros((0, (hq + 2 * hk) * D), dtype=torch.bfloat16, device="cuda")
    q, k, v = qkv[:, :hq * D], qkv[:, hq * D:(hq + hk) * D], qkv[:, (hq + hk) * D:]
    f = torch.tensor(cs.frequencies(D, 10000.0)[0], device="cuda")
    mask = torch.zeros((0, 1), dtype=torch.int32, device="cuda")
    dn.deinfer_tree_mask(step.slots, step.row_start, cached, mask, step.positions)
    dn.deinfer_rope_store(q, k, v, step.positions, f, hq, hk, D, slots=step.slots, k_out=pools[0], v_out=pools[1])
    dn.deinfer_rope_store(q, k, v, step.positions, f, hq, hk, D, slots=step.slots, q_out=torch.zeros((4, hq * D), dtype=torch.bfloat16, device="cuda"), k_out=pools[0], v_out=pools[1])
    ws = dn.Workspace(dn.deinfer_tree_attention_workspace_bytes(0, 2, hq, hk, D))
    out = dn.deinfer_tree_attention(q, pools[0], pools[1], table, step.row_start, cached, ws, hq, hk, bt, mask=mask)
    assert out.shape == (0, hq * D) and all(bool((p == 3.0).all()) for p in pools)


def test_rotary_store_of_more_rows_than_a_grid_has_threads_for(dn):
    """2^24 + 3 rows, a workgroup each: more threads than 32 bits count.  Against the same call on a few of the rows."""
    import torch
    rows, D = (1 << 24) + 3, 2
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn(rows, D, device="cuda", generator=g).bfloat16() for _ in range(3))
    pos = torch.arange(rows, device="cuda", dtype=torch.int32)
    slots = (rows - 1 - pos).contiguous()
    f = torch.tensor([0.37], dtype=torch.float64, device="cuda")
    pools = [torch.full((rows, D), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    some = torch.cat([torch.tensor([0, 1, (1 << 20) - 1, 1 << 20, (1 << 24) - 1, 1 << 24, rows - 1], device="cuda"), torch.randint(0, rows, (3000,), device="cuda", generator=g)])
    want = [t[some].contiguous() for t in (q, k)]
    dn.deinfer_rope_store(want[0], want[1], None, pos[some].contiguous(), f, 1, 1, D)
    out = torch.full_like(q, 9.0)
    dn.deinfer_rope_store(q, k, v, pos, f, 1, 1, D, slots=slots, q_out=out, k_out=pools[0], v_out=pools[1])
    assert torch.equal(out[some], want[0]) and torch.equal(pools[0][slots[some].long()], want[1])
    assert torch.equal(pools[1].flip(0), v)
    assert bool((out != 9.0).all()) and bool((pools[0] != 9.0).all())


def test_rows_of_a_tree_behind_its_mask(dn):
    """A chain of 70 tokens with one word of bits: rows 32 .. 69 see nothing drafted and count as tokens without ancestors; the row
    before is whole, and so is every row with three words."""
    import torch
    n, c = 70, 11
    parents, start, cached = ints(np.arange(n) - 1), ints([0, n]), ints([c])
    for words in (1, 3):
        mask, pos = torch.full((n, words), 5, dtype=torch.int32, device="cuda"), torch.full((n,), 5, dtype=torch.int32, device="cuda")
        dn.deinfer_tree_mask(parents, start, cached, mask, pos)
        j = np.arange(n)
        inside = j < 32 * words
        assert np.array_equal(host(pos), np.where(inside, c + j, c))
        bits = (host(mask).view(np.uint32)[:, :, None] >> np.arange(32, dtype=np.uint32)) & 1
        assert np.array_equal(bits.reshape(n, -1), np.tril(np.ones((n, 32 * words))) * inside[:, None])


def test_attention_refuses_blocks_of_no_tokens_and_heads_of_no_features(dn):
    """As an error of the library, like every other size, and before a launch."""
    import torch
    x = torch.zeros((2, 64), dtype=torch.bfloat16, device="cuda")
    ws = dn.Workspace(dn.deinfer_tree_attention_workspace_bytes(2, 1, 1, 1, 64))
    for bt in (0, -16):
        with pytest.raises(dn.DeinferError) as e:
            dn.deinfer_tree_attention(x, x, x, ints([[0]]), ints([0, 2]), ints([0]), ws, 1, 1, bt)
        assert e.value.code == dn.ERR_INVALID_ARG
    with pytest.raises(dn.DeinferError) as e:
        dn.deinfer_tree_attention(x[:, :0], x, x, ints([[0]]), ints([0, 2]), ints([0]), ws, 1, 1, 2)
    assert e.value.code == dn.ERR_UNSUPPORTED


@pytest.mark.parametrize("spare", [0, 1500])
@pytest.mark.parametrize("dtype,hq,hk,D,words", [("bf16", 2, 2, 64, 0), ("f16", 8, 1, 128, 0), ("bf16", 4, 1, 128, 10)])
def test_attention_of_a_batch_that_mixes_chunks_and_single_tokens(dn, dtype, hq, hk, D, words, spare):
    """Forty single tokens and a chunk of 300: the rows of a tile go by the average, 16 here, and 128 or 256 where the buffer has
    1500 rows to spare.  The result is the same."""
    import torch
    rng = np.random.default_rng(D)
    cached, new = rng.integers(0, 200, 42), np.ones(42, dtype=int)
    new[7], new[20] = 300, 0
    table, k, v = cache_case(61, cached, new, hk, D, 16, dtype)
    start = np.concatenate([[0], np.cumsum(new)])
    T = int(start[-1]) + spare
    q = torch.tensor(normal(62, T, hq * D), device="cuda").to(k.dtype)
    check_attention(dn, q, k, v, table, start, cached, hq, hk, 16, dtype, random_mask(rng, new, words, T) if words else None)
