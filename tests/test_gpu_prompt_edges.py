"""The calls between the projections of a prompt where they can go wrong.  Tolerances: as in test_gpu_prompt.py."""
import numpy as np
import pytest

from oracle import prompt as op
from test_gpu_cache_step import HALF, dn, host, ints, kind_of, normal, wide  # noqa: F401
from test_gpu_prompt import angles_of, check_norm, norm_case, packed

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ values that are no numbers
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("right", [0, -1])
@pytest.mark.parametrize("n,hq,D", [(6, 2, 128), (40, 4, 128), (150, 2, 64), (300, 2, 128), (60, 2, 256), (90, 2, 80)])
def test_seen_infinities_whose_probability_is_nothing(dn, dtype, right, n, hq, D):
    """0 x infinity is no number, whether some other row does not see the key or all do.  The key's score is 400 and more under the
    others, which are all 0: exp(-400) is 0 in every type, also as the factor of a sum."""
    import torch
    bad = n // 2
    q = torch.ones(n, hq * D, dtype=kind_of(dtype), device="cuda")
    k = torch.zeros(n, D, dtype=q.dtype, device="cuda")
    k[bad] = -50.0
    v = packed(43, [n], 1, D, dtype)
    v[bad] = 0.0
    ref, size = (op.attention(wide(q), wide(k), f(wide(v)), [0, n], None, hq, 1, -1, right, D ** -0.5, np.zeros((n, hq * D))) for f in (np.asarray, np.abs))
    v[bad, 5], v[bad, 7] = float("inf"), -float("inf")
    ws = dn.Workspace(dn.deinfer_prompt_attention_workspace_bytes(n, 1, hq, 1, D))
    got = wide(dn.deinfer_prompt_attention(q, k, v, ints([0, n]), ws, hq, 1, right=right)).reshape(n, hq, D)
    hit = np.zeros((n, hq, D), dtype=bool)
    hit[bad if right == 0 else 0:, :, [5, 7]] = True
    assert np.array_equal(np.isnan(got), hit), np.argwhere(np.isnan(got) != hit)[:5]
    tol = HALF[dtype] * (np.abs(ref) + size) * 1.01 + 4e-4 * size + (n * 2.0 ** -25 * np.max(size) if dtype == "f16" else 0.0)
    assert np.all((np.abs(got - ref.reshape(hit.shape)) <= tol.reshape(hit.shape))[~hit])


# ------------------------------------------------------------------ norms: eps of any size
@pytest.mark.parametrize("size,eps", [(0.0, 1e-50), (1e-28, 1e-50), (1e-30, 1e-46), (3e-23, 1e-46), (3e18, 3.4e38), (0.0, 3.4e38), (1e-12, 1e-40), (1.0, 1e-60)])
@pytest.mark.parametrize("D", [8, 64])
def test_norms_with_an_eps_beyond_fp32(dn, size, eps, D):
    """eps is a 64-bit number: one that fp32 has no bits for is not nothing, and one near its end does not make the sum infinite."""
    import torch
    T, H = 5, 3
    x = torch.tensor(np.clip(normal(9, T, H * D), -1.0, 1.0) * size, device="cuda").float()
    w, f, pos = torch.ones(D, device="cuda"), torch.tensor(10000.0 ** (-2.0 * np.arange(D // 2) / D), device="cuda"), np.arange(T)
    y = dn.deinfer_norm_rope_store(x.clone(), None, None, ints(pos), f, H, 0, D, q_weight=w, eps=eps)[0]
    check_norm(wide(y), wide(x), H, wide(w), eps, angles_of(pos[None], np.zeros(D // 2), host(f)), 1.0, False, "f32")


# ------------------------------------------------------------------ rows behind the last sequence
def test_norms_of_a_captured_step_leave_rows_without_a_slot(dn):
    """A graph replayed for steps of fewer and fewer tokens, slots from the step: what lies behind the last sequence's rows stays as it is in the
    queries too.  Without slots every row of the buffers is written."""
    import torch
    rows, hq, hk, D, bt, n_pool = 40, 4, 2, 64, 8, 16
    q, k, v, (qw, kw) = norm_case("bf16", rows, hq, hk, D, 0, seed=8)
    f = torch.tensor(10000.0 ** (-2.0 * np.arange(D // 2) / D), device="cuda")
    cached, new, table = ints([0, 0]), ints([0, 0]), torch.full((2, 8), -1, dtype=torch.int32, device="cuda")
    free = ints(np.arange(n_pool))
    step = dn.deinfer_kv_step(cached, new, table, free, bt, n_pool, rows)
    pools = [torch.zeros(n_pool * bt, hk * D, dtype=q.dtype, device="cuda") for _ in range(2)]
    to, straight = torch.zeros_like(q), torch.zeros_like(q)

    def call():
        dn.deinfer_kv_step(cached, new, table, free, bt, n_pool, rows, out=step)
        dn.deinfer_norm_rope_store(q, k, v, step.positions, f, hq, hk, D, q_weight=qw, k_weight=kw, slots=step.slots, q_out=to, k_out=pools[0], v_out=pools[1])
        dn.deinfer_norm_rope_store(q, None, None, step.positions, f, hq, 0, D, q_weight=qw, q_out=straight)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for lengths in ([20, 20], [9, 14], [1, 1], [0, 0], [30, 1]):
        new.copy_(ints(lengths))
        to.fill_(float("nan")), straight.fill_(float("nan"))
        for p in pools:
            p.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        n = sum(lengths)
        pos = np.r_[np.concatenate([np.arange(m) for m in lengths]), np.zeros(rows - n)]
        angles = angles_of(pos[None], np.zeros(D // 2), host(f))
        check_norm(wide(straight), wide(q), hq, wide(qw), 1e-6, angles, 1.0, False, "bf16")
        assert torch.equal(to[:n], straight[:n]) and bool(torch.isnan(to[n:]).all())
        slots = host(step.slots)
        assert np.all(slots[:n] >= 0) and np.all(slots[n:] == -1)
        unused = np.setdiff1d(np.arange(n_pool * bt), slots[:n])
        assert bool(torch.isnan(pools[0][unused]).all()) and bool(torch.isnan(pools[1][unused]).all())
        assert torch.equal(pools[1][slots[:n]], v[:n])


# ------------------------------------------------------------------ keys with gaps between sequences
@pytest.mark.parametrize("cached,new", [([37, 5, 90], [2, 1, 3]), ([0, 15, 33, 1], [1, 1, 1, 1]), ([40, 0, 7], [60, 33, 20]), ([16, 30], [16, 2])])
@pytest.mark.parametrize("hq,hk,D", [(4, 2, 128), (8, 1, 64)])
def test_keys_rebuilt_from_the_low_rank_cache(dn, cached, new, hq, hk, D):
    """Plan, compacting copies, keys rebuilt and rotated, values rebuilt: every sequence begins at a block, so that there is a gap behind most,
    a sequence without rows.  Against the attention through the remapped table, and in 64 bits."""
    import torch
    bt, r, d_in, n_pool, buf_blocks, n = 16, 40, 64, 32, 20, len(cached)
    total, T = [c + m for c, m in zip(cached, new)], sum(new) + 3
    pair = lambda s: dn.deinfer_pack_factors(dn.raw_pair(torch.tensor(normal(s, d_in, r) / 8, device="cuda").to(torch.bfloat16),
                                                        torch.tensor(normal(s + 1, r, hk * D) / 6, device="cuda").to(torch.bfloat16)))
    fk, fv = pair(30), pair(32)
    pools = [torch.tensor(normal(34 + i, n_pool * bt, r), device="cuda").to(torch.bfloat16) for i in range(2)]
    blocks = [-(-c // bt) for c in total]
    table = np.full((n, 9), -1)
    ids = np.random.default_rng(2).permutation(n_pool)
    for s in range(n):
        table[s, :blocks[s]] = ids[sum(blocks[:s]):sum(blocks[:s + 1])]
    lengths = ints(total)
    plan, remap, pos = dn.deinfer_kv_compact_plan_device(ints(table), lengths, n_pool, buf_blocks, bt)
    bufs = [torch.full((buf_blocks * bt, r), 50.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for p, b in zip(pools, bufs):
        dn.deinfer_kv_compact_copy(p, bt * r * 2, plan, b)
    ws = dn.Workspace(max(dn.deinfer_workspace_bytes(buf_blocks * bt, [fk, fv]), dn.deinfer_tree_attention_workspace_bytes(T, n, hq, hk, D),
                          dn.deinfer_prompt_attention_workspace_bytes(T, 2 * n, hq, hk, D)))
    keys = dn.deinfer_lowrank_up_rope(bufs[0], fk, dn.deinfer_rope_table(pos, D), ws)
    values = dn.deinfer_lowrank_up(bufs[1], fv, ws)
    q = packed(50, new, hq, D, "bf16", 3)
    row_start = ints(starts(new))
    paged = dn.deinfer_tree_attention(q, keys, values, remap, row_start, ints(cached), ws, hq, hk, bt)
    # sequence 2 s: the rows and keys of s; sequence 2 s + 1: no rows, and the rest of its last block
    q_start = row_start[torch.tensor([0] + [s for s in range(1, n + 1) for _ in range(2)], device="cuda")].contiguous()
    block_end = torch.cumsum((lengths + bt - 1) // bt * bt, 0).int()
    first = torch.cat([torch.zeros_like(block_end[:1]), block_end[:-1]])
    k_start = torch.cat([torch.stack([first, first + lengths], 1).flatten(), block_end[-1:]]).contiguous()
    out = torch.full((T, hq * D), 3.0, dtype=torch.bfloat16, device="cuda")
    dn.deinfer_prompt_attention(q, keys, values, q_start, ws, hq, hk, k_start=k_start, out=out)
    got, qh, vh = wide(out), np.nan_to_num(wide(q)), wide(values)
    args = (host(q_start), host(k_start), hq, hk, -1, 0, D ** -0.5, np.full((T, hq * D), 3.0))
    ref, size = op.attention(qh, wide(keys), vh, *args), op.attention(qh, wide(keys), np.abs(vh), *args)
    rows = sum(new)
    assert np.all((np.abs(got - ref) <= HALF["bf16"] * (np.abs(ref) + size) * 1.01 + 4e-4 * size)[:rows])
    assert np.all(np.abs(got - wide(paged))[:rows] <= 2 * (HALF["bf16"] * (np.abs(ref) + size) * 1.01 + 4e-4 * size)[:rows])
    assert np.all(got[rows:] == 3.0)
    # (what stands in the gaps is not seen)
    for b, t in ((values, float("inf")), (keys, float("nan"))):
        for s in range(n):
            b[int(host(first)[s]) + total[s]:int(host(block_end)[s])] = t
    again = dn.deinfer_prompt_attention(q, keys, values, q_start, ws, hq, hk, k_start=k_start)
    assert np.all((np.abs(wide(again) - ref) <= HALF["bf16"] * (np.abs(ref) + size) * 1.01 + 4e-4 * size)[:rows])
