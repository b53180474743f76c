"""The calls between the projections of a prompt where they can go wrong: values that are no numbers beside windows and splits, the
workspace's end, more sequences and rows than one pass takes, rows behind the last sequence, keys with gaps between sequences.
Tolerances: as in test_gpu_prompt.py."""
import numpy as np
import pytest

from oracle import prompt as op
from test_gpu_cache_step import HALF, dn, host, ints, kind_of, normal, wide  # noqa: F401
from test_gpu_prompt import angles_of, check_norm, check_prompt, norm_case, packed, starts

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


BAD = [
    # rows, keys (None: the rows'), q heads, kv heads, head dim, left, right
    ([5], [200], 2, 1, 128, 40, 3),
    ([2, 3], [1500, 800], 8, 1, 128, 90, 1),                         # over many workgroups
    ([9, 4], [70, 300], 3, 3, 80, 64, 0),
    ([40, 30], [700, 200], 4, 1, 64, 100, 20),
    ([60, 60], [500, 130], 2, 1, 256, 64, 64),
    ([300], [900], 2, 1, 128, 70, 30),
    ([300, 200], [900, 210], 2, 2, 80, 130, 40),
    ([700, 600, 650], None, 8, 8, 64, 90, 20),                       # tiles after one another in a workgroup
    ([700, 600], None, 4, 4, 256, 33, 0),
    ([400], [2000], 4, 1, 96, -1, 0),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows,keys,hq,hk,D,left,right", BAD)
def test_values_of_several_kinds_that_are_no_numbers(dn, dtype, rows, keys, hq, hk, D, left, right):
    """Infinities of both signs and NaN in one column, at the first and the last key and on both sides of stages: each row has what the keys
    that it sees make of it.  Random scores of a few units: every probability is a number of the type."""
    import torch
    of = rows if keys is None else keys
    q, k, v = packed(1, rows, hq, D, dtype, 2), packed(2, of, hk, D, dtype, 2), packed(3, of, hk, D, dtype, 2)
    q_start, k_start = starts(rows), starts(of)
    T = q.shape[0]
    call_ws = dn.Workspace(dn.deinfer_prompt_attention_workspace_bytes(T, len(rows), hq, hk, D))
    kinds = {1: float("inf"), 2: -float("inf"), 3: float("nan")}
    found = {c: [[(0, 1), (31, 2), (32, 1), (63, 3), (64, 1), (65, 2), (127, 2), (n // 2, 1), (n // 2 + 70, 2), (n - 1, 3)] for n in of] for c in (5,)}
    found[D - 1] = [[(0, 1), (64, 1), (95, 1), (n - 1, 1)] for n in of]
    found[2] = [[(33, 2), (127, 2), (n - 33, 2)] for n in of]
    found[8] = [[(0, 3), (n - 1, 2)] for n in of]
    vc = wide(v).copy()
    kind = np.zeros(vc.shape, dtype=int)
    for c, lists in found.items():
        for s, one in enumerate(lists):
            for at, what in one:
                if 0 <= at < of[s]:
                    kind[k_start[s] + at, [h * D + c for h in range(hk)]] = what
    bad = torch.tensor(kind, device="cuda")
    for what, value in kinds.items():
        v[bad == what] = value
    vc[kind > 0] = 0.0
    got = wide(dn.deinfer_prompt_attention(q, k, v, ints(q_start), call_ws, hq, hk, k_start=None if keys is None else ints(k_start), left=left, right=right))
    qh, kh, vc = np.nan_to_num(wide(q)), np.nan_to_num(wide(k)), np.nan_to_num(vc)
    ref, size = (op.attention(qh, kh, x, q_start, None if keys is None else k_start, hq, hk, left, right, D ** -0.5, np.zeros((T, hq * D))) for x in (vc, np.abs(vc)))
    # how many of each kind a row sees: the attention's own mask, with whole numbers
    group = hq // hk
    want = ref.copy()
    for s in range(len(rows)):
        place = of[s] - rows[s] + np.arange(rows[s])[:, None]
        j = np.arange(of[s])[None, :]
        sees = np.ones((rows[s], of[s]), dtype=bool)
        if left >= 0:
            sees &= j >= place - left
        if right >= 0:
            sees &= j <= place + right
        mine = kind[k_start[s]:k_start[s + 1]]
        up, down, nan = ((sees.astype(int) @ (mine == what).astype(int)) > 0 for what in (1, 2, 3))
        for h in range(hq):
            to, cols = slice(h * D, (h + 1) * D), slice(h // group * D, (h // group + 1) * D)
            w = want[q_start[s]:q_start[s + 1], to]
            w[up[:, cols]] = np.inf
            w[down[:, cols]] = -np.inf
            w[nan[:, cols] | (up & down)[:, cols]] = np.nan
    n = int(q_start[-1])
    got, want, ref, size = got[:n], want[:n], ref[:n], size[:n]
    fine = np.isfinite(want)
    assert np.any(~fine) and np.any(fine)
    assert np.array_equal(np.isnan(got), np.isnan(want)), np.argwhere(np.isnan(got) != np.isnan(want))[:5]
    odd = ~fine & ~np.isnan(want)
    assert np.array_equal(got[odd], want[odd])
    tol = HALF[dtype] * (np.abs(ref) + size) * 1.01 + 4e-4 * size + (max(of) * 2.0 ** -25 * np.max(np.abs(vc)) if dtype == "f16" else 0.0)
    assert np.all((np.abs(got - ref) <= tol)[fine])


# ------------------------------------------------------------------ the workspace
HEIGHTS = {16: ([1, 2, 1], [900, 700, 20], 8), 128: ([40, 25], [300, 200], 2), 256: ([150, 130], [1000, 300], 2)}


@pytest.mark.parametrize("D", [40, 64, 72, 80, 96, 128, 200, 256])
@pytest.mark.parametrize("height", HEIGHTS)
def test_the_attention_keeps_to_its_workspace_whatever_it_holds(dn, height, D):
    """All bits set in it beforehand, and a guard behind the bytes that the host call gave."""
    import torch
    rows, keys, hq = HEIGHTS[height]
    hk = 1
    need, guard = dn.deinfer_prompt_attention_workspace_bytes(sum(rows), len(rows), hq, hk, D), 1 << 20
    ws = dn.Workspace(need, buf=torch.empty(need + guard, dtype=torch.uint8, device="cuda"))
    ws.buf.fill_(255)
    q, k, v = packed(D, rows, hq, D, "bf16"), packed(D + 1, keys, hk, D, "bf16"), packed(D + 2, keys, hk, D, "bf16")
    check_prompt(dn, q, k, v, starts(rows), starts(keys), hq, hk, -1, 0, "bf16", ws=ws)
    assert bool((ws.buf[need:] == 255).all())
    ws.buf.fill_(255)
    check_prompt(dn, q, k, v, starts(rows), starts(keys), hq, hk, 50, -1, "bf16", ws=ws)
    assert bool((ws.buf[need:] == 255).all())


# ------------------------------------------------------------------ more than one pass takes
@pytest.mark.parametrize("n_seqs", [511, 513, 1100])
def test_more_sequences_than_threads_of_a_tall_tile(dn, n_seqs):
    """Tiles of 256 rows: the run is found 512 sequences at a time."""
    rng = np.random.default_rng(n_seqs)
    rows, keys = rng.integers(8, 33, n_seqs), rng.integers(0, 90, n_seqs)
    rows[[0, 5, n_seqs - 1]] = [0, 300, 0]
    hq, D = 8, 64
    assert sum(rows) * hq > 128 * n_seqs
    q, k, v = packed(1, rows, hq, D, "bf16", 3), packed(2, keys, 1, D, "bf16", 1), packed(3, keys, 1, D, "bf16", 1)
    check_prompt(dn, q, k, v, starts(rows), starts(keys), hq, 1, -1, 0, "bf16")


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("f16", 128)])
def test_a_chunk_beside_single_tokens(dn, dtype, D):
    """A head for every query head: on average nine rows of a sequence, and one of 512."""
    rng = np.random.default_rng(D)
    rows = np.array([1] * 30 + [512] + [1] * 33)
    keys = rows + rng.integers(0, 700, 64)
    q, k, v = packed(4, rows, 8, D, dtype, 1), packed(5, keys, 8, D, dtype, 1), packed(6, keys, 8, D, dtype, 1)
    check_prompt(dn, q, k, v, starts(rows), starts(keys), 8, 8, -1, 0, dtype)


def test_norms_of_more_rows_than_a_grid_is_wide(dn):
    import torch
    T, D = (1 << 20) + 300, 8
    gen = torch.Generator(device="cuda").manual_seed(3)
    q = torch.randn(T, D, generator=gen, device="cuda").to(torch.bfloat16)
    w = torch.tensor(1.0 + 0.3 * normal(5, D), device="cuda").to(torch.bfloat16)
    f, pos = torch.tensor(10000.0 ** (-2.0 * np.arange(4) / D), device="cuda"), torch.arange(T, dtype=torch.int32, device="cuda") % 4099
    got = torch.full((T + 1, D), 7.0, dtype=q.dtype, device="cuda")
    dn.deinfer_norm_rope_store(q, None, None, pos, f, 1, 0, D, q_weight=w, q_out=got[:T])
    at = np.r_[0:300, (1 << 20) - 300:T]
    check_norm(wide(got[:T])[at], wide(q)[at], 1, wide(w), 1e-6, angles_of(host(pos)[None, at], np.zeros(4), host(f)), 1.0, False, "bf16")
    half = T // 2
    for rows in (slice(0, half), slice(half, T)):
        part = dn.deinfer_norm_rope_store(q[rows].contiguous(), None, None, pos[rows].contiguous(), f, 1, 0, D, q_weight=w)[0]
        assert torch.equal(part, got[rows])
    assert bool((got[T] == 7.0).all())


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


# ------------------------------------------------------------------ nothing to see, and everything
@pytest.mark.parametrize("rows,hq", [([1, 2], 2), ([40, 30], 4), ([150, 200], 2)])
def test_no_keys_at_all_and_no_rows_at_all(dn, rows, hq):
    import torch
    D, T = 64, sum(rows) + 2
    q, none = packed(1, rows, hq, D, "bf16", 2), torch.empty(0, D, dtype=torch.bfloat16, device="cuda")
    ws = dn.Workspace(dn.deinfer_prompt_attention_workspace_bytes(T, 2, hq, 1, D))
    out = torch.full((T, hq * D), 3.0, dtype=torch.bfloat16, device="cuda")
    for left, right in ((-1, 0), (-1, -1), (5, 7)):
        out.fill_(3.0)
        dn.deinfer_prompt_attention(q, none, none, ints(starts(rows)), ws, hq, 1, k_start=ints([0, 0, 0]), left=left, right=right, out=out)
        assert bool((out[:T - 2] == 0).all()) and bool((out[T - 2:] == 3.0).all())
        out.fill_(3.0)
        dn.deinfer_prompt_attention(q, q[:, :D], q[:, :D], ints([0, 0, 0]), ws, hq, 1, k_start=ints([0, 5, T]), left=left, right=right, out=out)
        assert bool((out == 3.0).all())


@pytest.mark.parametrize("rows,hq", [([5, 2], 2), ([40, 30], 4), ([150, 200], 2)])
def test_sides_of_a_window_beyond_every_length(dn, rows, hq):
    """Bit for bit those without a bound."""
    import torch
    q, k, v = packed(1, rows, hq, 64, "f16"), packed(2, rows, 1, 64, "f16"), packed(3, rows, 1, 64, "f16")
    ws = dn.Workspace(dn.deinfer_prompt_attention_workspace_bytes(sum(rows), 2, hq, 1, 64))
    call = lambda left, right: dn.deinfer_prompt_attention(q, k, v, ints(starts(rows)), ws, hq, 1, left=left, right=right)
    for far in (max(rows), 1 << 28, (1 << 31) - 1, 1 << 31, (1 << 32) + 1, (1 << 63) - 1):
        assert torch.equal(call(far, 0), call(-1, 0)) and torch.equal(call(0, far), call(0, -1)) and torch.equal(call(far, far), call(-1, -1))
