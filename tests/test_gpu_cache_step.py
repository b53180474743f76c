"""One step over a paged cache on the GPU through the C ABI, each call against the oracle: whole numbers exactly, rotations and
attention within what their roundings can make.  Every pool starts out full of NaN, so anything read where nothing was
written shows.

Tolerances.  h = half a step of the output type relative to the value (bf16 2^-8, fp16 2^-11, fp32 2^-24).
  rotation   y = a cos - b sin: angles as a fraction of a turn in fp32 (2^-26 turns, 1e-7 radians off), cos and sin within
             two units of 2^-24, two products and a sum in fp32: 5e-7 (|a| + |b|), and h |y| for the output's rounding.
  attention  with A = sum_j p_j |v_j|: the probabilities' rounding to the type, h A; the output's, h |o|; scores of D products summed
             in fp32, D 2^-24 sum |q_i k_i| scale, under 2e-4 for the sizes here, which is the relative error of p: 2 x 2e-4 A
             (numerator and sum).  fp16 probabilities under 2^-14 are off by up to 2^-25 each: n 2^-25 max |v|."""
import numpy as np
import pytest

from oracle import cache_step as cs
from oracle import paged_cache as pc
import synth_inputs as si

pytestmark = pytest.mark.gpu

HALF = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}


@pytest.fixture(scope="module")
def dn():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2604_17709_amd as dn
    dn.lib()
    return dn


def kind_of(name):
    import torch
    return {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[name]


def ints(x):
    import torch
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def host(t):
    return t.detach().cpu().numpy()


def wide(t):
    import torch
    return t.detach().to(torch.float64).cpu().numpy()


def normal(seed, *shape):
    return np.random.default_rng(seed).standard_normal(shape)


# ------------------------------------------------------------------ block tables, slots, positions
STEPS = {
    # cached, new, block tokens, pool blocks, free ids, first, table pitch, T
    "one_token": ([5], [1], 16, 8, [3, 4], 0, 4, 1),
    "block_border": ([16, 15, 0, 32, 17], [1, 2, 0, 16, 15], 16, 40, list(range(20, 40)), 0, 6, 40),
    "no_tokens": ([3, 0, 64], [0, 0, 0], 16, 16, [9], 0, 5, 8),
    "prompts": ([0, 0, 7], [100, 1, 250], 8, 200, list(range(199, 100, -1)), 3, 40, 400),
    "tokens_of_one": ([0, 2], [3, 2], 1, 12, [11, 10, 9, 8, 7, 6], 0, 9, 7),
    "odd_blocks": ([6, 20], [9, 40], 7, 32, list(range(10, 30)), 0, 12, 64),
    "too_few_rows": ([0, 5, 3], [10, 20, 30], 4, 64, list(range(30, 64)), 0, 12, 24),
    "too_few_blocks": ([4, 5, 3], [10, 20, 30], 4, 64, list(range(30, 38)), 2, 12, 64),
    "free_list_passed": ([4, 5], [10, 20], 4, 64, list(range(30, 38)), 9, 12, 64),
    "table_too_narrow": ([4, 5], [10, 20], 4, 64, list(range(30, 60)), 0, 3, 64),
    "bad_free_ids": ([4, 0], [10, 9], 4, 16, [9, 16, -3, 10, 11, 12, 1000000], 0, 8, 32),
    "negative_lengths": ([-4, 3], [5, -2], 4, 16, [9, 10, 11], 0, 8, 8),
}


def held_table(cached, bt, pitch, seed):
    n = [min(pitch, max(0, -(-c // bt))) for c in cached]
    t = np.full((len(cached), pitch), -7, dtype=np.int64)
    ids = np.random.default_rng(seed).permutation(sum(n) or 1)
    at = 0
    for s, k in enumerate(n):
        t[s, :k] = ids[at:at + k]
        at += k
    return t


def check_step(dn, cached, new, bt, pool, free, first, pitch, T, table, shift=0):
    import torch
    tab, fr = ints(table), ints(free)
    out = None
    if shift:
        new_out = lambda n: torch.full((n + 8,), 77, dtype=torch.int32, device="cuda")[shift:]
        out = dn.KvStep(new_out(len(cached) + 1), new_out(T), new_out(T), new_out(4))
    ff = None if first == 0 else ints([first])
    got = None
    for _ in range(2):                                             # a second time: the same
        got = dn.deinfer_kv_step(ints(cached), ints(new), tab, fr, bt, pool, T, free_first=ff, out=out)
    want = cs.kv_step(cached, new, table, free, first, pool, bt, T)
    n = len(cached) + 1
    assert np.array_equal(host(got.row_start)[:n], want[0])
    assert np.array_equal(host(got.slots)[:T], want[1])
    assert np.array_equal(host(got.positions)[:T], want[2])
    assert np.array_equal(host(tab), want[3])
    assert np.array_equal(host(got.counts)[:4], want[4])
    if shift:
        assert np.all(host(got.slots)[T:] == 77) and np.all(host(got.positions)[T:] == 77) and np.all(host(got.row_start)[n:] == 77)


@pytest.mark.parametrize("name", STEPS)
@pytest.mark.parametrize("shift", [0, 1])
def test_step(dn, name, shift):
    cached, new, bt, pool, free, first, pitch, T = STEPS[name]
    check_step(dn, cached, new, bt, pool, free, first, pitch, T, held_table(cached, bt, pitch, 1), shift)


@pytest.mark.parametrize("seqs,longest,most,bt,T", [(1, 5000, 9000, 16, 9001), (1024, 300, 9, 16, 9000), (1025, 40, 3, 8, 4099), (8192, 20, 2, 16, 12288), (300, 100, 200, 32, 40000)])
def test_step_of_many(dn, seqs, longest, most, bt, T):
    rng = np.random.default_rng(seqs)
    cached, new = rng.integers(0, longest, seqs), rng.integers(0, most + 1, seqs)
    pitch = -(-(longest + most) // bt) + 1
    table = held_table(cached, bt, pitch, 2)
    used = int(sum(-(-c // bt) for c in cached))
    need = int(sum(-(-(c + m) // bt) for c, m in zip(cached, new))) - used
    check_step(dn, cached, new, bt, used + need + 5, rng.permutation(need + 5) + used, 0, pitch, T, table)


def test_step_without_sequences(dn):
    import torch
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    got = dn.deinfer_kv_step(none, none, torch.zeros((0, 4), dtype=torch.int32, device="cuda"), none, 16, 8, 5)
    assert host(got.row_start).tolist() == [0] and host(got.slots).tolist() == [-1] * 5 and host(got.positions).tolist() == [0] * 5
    assert host(got.counts).tolist() == [0, 0, 0, 0]


# ------------------------------------------------------------------ the plan of the compacting copy
@pytest.mark.parametrize("seed,prompt,decode,n_pool,recycled,bt,extra", [
    (1, [9, 1, 17, 4, 0, 30], [5, 0, 2, 7, 3, 1], 256, 0, 16, 5),
    (2, [9, 1, 17, 4, 0, 30], [5, 0, 2, 7, 3, 1], 256, 40, 16, 0),
    (3, [32] * 16, [1] * 16, 1024, 0, 16, 3),
    (4, [3, 3, 3], [40, 40, 40], 200, 200, 1, 4),
    (5, [0], [0], 4, 0, 16, 6),
    (6, [8192, 3], [2, 1], 9000, 0, 16, 9),                # a run that ends behind a workgroup's share of the walk
    (7, [20000], [0], 20000, 0, 4, 1),                     # one run over three shares
    (8, [12] * 1500, [3] * 1500, 24000, 100, 8, 50),
])
def test_plan_is_the_host_call(dn, seed, prompt, decode, n_pool, recycled, bt, extra):
    import torch
    table, n_blocks = si.paged_block_tables(seed, prompt, decode, n_pool, recycled)
    table = np.pad(table, ((0, 0), (0, 2)), constant_values=-1)
    cap = int(n_blocks.sum()) + extra
    plan, remap, pos = dn.deinfer_kv_compact_plan(table, n_blocks, n_pool, cap, bt)
    rng = np.random.default_rng(seed)
    tokens = np.maximum(0, n_blocks * bt - rng.integers(0, bt, len(n_blocks)) * (n_blocks > 0))     # a last block that is not full
    new = np.minimum(tokens, rng.integers(0, 5, len(n_blocks)))
    for split in (False, True):
        got = dn.deinfer_kv_compact_plan_device(ints(table), ints(tokens - new if split else tokens), n_pool, cap, bt, n_new=ints(new) if split else None)
        for g, w in zip(got, (plan, remap, pos)):
            assert np.array_equal(host(g), w)


def test_plan_flags(dn):
    import torch
    table = [[5, 6, 7, 2], [3, 4, 9, -1], [10, 11, -1, -1]]
    tokens = [4, 3, 2]

    def call(table=table, tokens=tokens, pool=12, buf=9, cap=9, rpitch=4):
        out = tuple(torch.full(s, 55, dtype=torch.int32, device="cuda") for s in ((4 + 3 * cap,), (3, rpitch), (buf * 1,)))
        plan, remap, pos = dn.deinfer_kv_compact_plan_device(ints(table), ints(tokens), pool, buf, 1, out=out)
        return host(plan).tolist(), host(remap).tolist(), host(pos).tolist()

    plan, remap, pos = call()
    assert plan == [3, 9, 0, 0, 5, 0, 3, 2, 3, 3, 9, 6, 3] + [0] * 18
    assert remap == [[0, 1, 2, 3], [4, 5, 6, -1], [7, 8, -1, -1]] and pos == [0, 1, 2, 3, 0, 1, 2, 0, 1]
    plan, remap, _ = call(pool=11)                                   # block 11 is outside
    assert plan[:4] == [0, 0, 1, 0] and remap == [[0, 1, 2, 3], [4, 5, 6, -1], [7, -1, -1, -1]]
    plan, remap, _ = call(table=[[5, -6, 7, 2], table[1], table[2]])
    assert plan[:4] == [0, 0, 1, 0] and remap[0] == [0, -1, 2, 3]
    plan, remap, _ = call(buf=7)
    assert plan[:4] == [0, 0, 2, 0] and remap == [[0, 1, 2, 3], [4, 5, 6, -1], [-1, -1, -1, -1]]
    plan, remap, _ = call(tokens=[4, 6, 2], buf=20)                  # six blocks in a row of four
    assert plan[2] & 4 and plan[0] == 0
    plan, remap, _ = call(rpitch=3)
    assert plan[2] == 4 and plan[0] == 0
    assert call(cap=2)[0][:4] == [0, 0, 8, 0]
    assert call(pool=11, cap=2, buf=8)[0][:4] == [0, 0, 2 | 8, 0]
    # the copy moves nothing for such a plan
    pool = torch.zeros((12, 16), dtype=torch.uint8, device="cuda")
    buf = torch.full((9, 16), 3, dtype=torch.uint8, device="cuda")
    out = dn.deinfer_kv_compact_plan_device(ints(table), ints(tokens), 11, 9, 1)
    dn.deinfer_kv_compact_copy(pool, 16, out[0], buf)
    assert int((buf != 3).sum()) == 0


# ------------------------------------------------------------------ drafted trees
@pytest.mark.parametrize("seed,rows,words,extra", [
    (1, [1], 1, 0), (2, [8, 1, 0, 32, 5], 1, 3), (3, [33, 64, 2], 2, 1), (4, [40, 70, 3], 2, 0), (5, [256, 250], 8, 2), (6, [1024, 7], 32, 0),
    (7, [1000, 1100], 32, 0), (8, [3] * 1500, 1, 5)])
@pytest.mark.parametrize("shape", ["random", "chain", "star", "bad"])
def test_tree_mask(dn, seed, rows, words, extra, shape):
    import torch
    rng = np.random.default_rng(seed)
    start = np.concatenate([[0], np.cumsum(rows)])
    T = int(start[-1]) + extra
    j = np.concatenate([np.arange(n) for n in rows] + [np.zeros(extra, dtype=np.int64)])
    parents = {"chain": j - 1, "star": np.full(T, -1), "random": np.maximum(-1, j - rng.integers(1, 7, T)),
               "bad": rng.integers(-3, 40, T)}[shape]
    cached = rng.integers(-2, 5000, len(rows))
    mask = torch.full((T, words), 0x5a5a5a, dtype=torch.int32, device="cuda")
    pos = torch.full((T,), -9, dtype=torch.int32, device="cuda")
    dn.deinfer_tree_mask(ints(parents), ints(start), ints(cached), mask, pos)
    bits, want = cs.tree(parents, start, cached, words)
    n = int(start[-1])
    assert np.array_equal(host(mask)[:n].view(np.uint32), np.array(bits, dtype=np.uint32).reshape(n, words))
    assert np.array_equal(host(pos)[:n], want)
    assert np.all(host(mask)[n:] == 0x5a5a5a) and np.all(host(pos)[n:] == -9)


# ------------------------------------------------------------------ rotary positions into the cache
ROPES = [
    # dtype, rows, q heads, kv heads, head dim, rotated, interleaved, columns more per row
    ("bf16", 5, 4, 2, 128, 128, False, 0),
    ("bf16", 70, 8, 8, 64, 32, False, 8),
    ("f16", 33, 6, 2, 128, 64, True, 0),
    ("f16", 3, 5, 1, 96, 96, True, 16),
    ("f32", 9, 4, 4, 64, 64, False, 4),
    ("f32", 17, 3, 1, 40, 24, True, 0),
    ("bf16", 6, 2, 1, 20, 12, False, 3),        # nothing of whole 16-byte pieces
    ("bf16", 6, 2, 1, 20, 12, True, 1),
    ("f16", 4, 3, 3, 7, 6, False, 0),           # odd heads
    ("f32", 4, 2, 2, 5, 2, False, 1),
    ("bf16", 2, 1, 1, 256, 256, False, 0),
    ("f32", 2, 1, 1, 1100, 1024, False, 0),     # the longest rotated part, more pieces than threads
    ("f32", 2, 1, 1, 1101, 1024, False, 0),
]


def rope_case(dtype, rows, hq, hk, D, rot, inter, extra, seed=7):
    import torch
    kind = kind_of(dtype)
    make = lambda n, s: torch.tensor(normal(s, rows, n * D + extra), device="cuda").to(kind)[:, :n * D]
    q, k, v = make(hq, seed), make(hk, seed + 1), make(hk, seed + 2)
    pos = np.random.default_rng(seed).integers(0, 1 << 20, rows)
    pos[0] = 0
    return q, k, v, pos


def close(got, ref, size, dtype):
    tol = HALF[dtype] * np.abs(ref) * 1.001 + 5e-7 * size + (2.0 ** -25 if dtype == "f16" else 0.0)
    worst = np.max(np.abs(got - ref) / np.maximum(tol, 1e-300)) if got.size else 0.0
    assert np.all(np.abs(got - ref) <= tol), worst


@pytest.mark.parametrize("dtype,rows,hq,hk,D,rot,inter,extra", ROPES)
def test_rope_store(dn, dtype, rows, hq, hk, D, rot, inter, extra):
    import torch
    q, k, v, pos = rope_case(dtype, rows, hq, hk, D, rot, inter, extra)
    f, magnitude = dn.deinfer_rope_frequencies(rot, 10000.0, dn.ROPE_RAMP, 4.0, 4096.0, 1.0, 32.0)
    n_slots = rows + 4
    slots = np.random.default_rng(3).permutation(n_slots)[:rows]
    slots[rows // 2] = -1 if rows % 2 else n_slots                   # a row that is not in use
    pools = [torch.full((n_slots, hk * D + extra), float("nan"), dtype=q.dtype, device="cuda") for _ in range(2)]
    q_out = torch.full((rows, hq * D + extra), float("nan"), dtype=q.dtype, device="cuda")
    dn.deinfer_rope_store(q, k, v, ints(pos), torch.tensor(f, device="cuda"), hq, hk, D, interleaved=inter, magnitude=magnitude, slots=ints(slots),
                          q_out=q_out[:, :hq * D], k_out=pools[0][:, :hk * D], v_out=pools[1][:, :hk * D])
    live = [t for t in range(rows) if 0 <= slots[t] < n_slots]
    dead = [t for t in range(rows) if t not in live]
    mag = np.float64(np.float32(magnitude))
    for x, y, heads, at in ((q, q_out, hq, live), (k, pools[0], hk, slots[live])):
        ref = cs.rotate(wide(x)[live], pos[live], f, heads, D, inter, mag)
        size = np.abs(cs.rotate(np.abs(wide(x)[live]), np.zeros(len(live)), f, heads, D, inter)) + np.max(np.abs(wide(x)[live]))
        got = wide(y)[at]
        close(got[:, :heads * D], ref, 2 * size, dtype)
        rest = np.concatenate([np.arange(h * D + rot, (h + 1) * D) for h in range(heads)])
        assert np.array_equal(got[:, rest.astype(int)], wide(x)[live][:, rest.astype(int)])
        assert np.all(np.isnan(got[:, heads * D:]))
    assert np.array_equal(wide(pools[1])[slots[live], :hk * D], wide(v)[live])
    assert np.all(np.isnan(wide(q_out)[dead]))
    unused = [r for r in range(n_slots) if r not in set(slots[live])]
    assert np.all(np.isnan(wide(pools[0])[unused])) and np.all(np.isnan(wide(pools[1])[unused]))


@pytest.mark.parametrize("dtype,D,rot,inter", [("bf16", 128, 128, False), ("f16", 64, 32, True), ("f32", 20, 12, False)])
def test_rope_in_place_and_alone(dn, dtype, D, rot, inter):
    """In place without slots, q alone, k alone: the same bits as apart; inverse angles turn it back."""
    import torch
    q, k, v, pos = rope_case(dtype, 11, 4, 2, D, rot, inter, 0)
    f = torch.tensor(cs.frequencies(rot, 500000.0)[0], device="cuda")
    apart = [torch.empty_like(t) for t in (q, k, v)]
    dn.deinfer_rope_store(q, k, v, ints(pos), f, 4, 2, D, interleaved=inter, q_out=apart[0], k_out=apart[1], v_out=apart[2])
    a, b = q.clone(), k.clone()
    dn.deinfer_rope_store(a, b, None, ints(pos), f, 4, 2, D, interleaved=inter)
    assert torch.equal(a, apart[0]) and torch.equal(b, apart[1]) and torch.equal(v, apart[2])
    c, d = q.clone(), k.clone()
    dn.deinfer_rope_store(c, None, None, ints(pos), f, 4, 0, D, interleaved=inter)
    dn.deinfer_rope_store(None, d, None, ints(pos), f, 0, 2, D, interleaved=inter)
    assert torch.equal(c, a) and torch.equal(d, b)
    dn.deinfer_rope_store(a, b, None, ints(-pos), f, 4, 2, D, interleaved=inter)
    # two roundings of elements of at most |a| + |b| <= 2 max
    most = max(float(q.abs().max()), float(k.abs().max()))
    assert float((a.double() - q.double()).abs().max()) <= 2 * (2 * HALF[dtype] + 1e-6) * 2 * most
    assert torch.equal(a.view(torch.int16 if dtype != "f32" else torch.int32)[0], q.view(torch.int16 if dtype != "f32" else torch.int32)[0])      # position 0


def test_rope_agrees_with_the_call_in_place(dn):
    """Plain frequencies, whole heads, half layout: deinfer_rope_inplace, to the last step of the type."""
    import torch
    q, _, _, pos = rope_case("bf16", 40, 8, 8, 128, 128, False, 0)
    a, b = q.clone(), q.clone()
    dn.deinfer_rope_inplace(a, 8, 128, ints(pos), 10000.0)
    dn.deinfer_rope_store(b, None, None, ints(pos), torch.tensor(cs.frequencies(128, 10000.0)[0], device="cuda"), 8, 0, 128)
    # the same angles within 1e-7: nearly every element has the same bits, none is off by more than a step of the larger of its pair
    assert float((a != b).float().mean()) < 1e-3
    assert float((a.double() - b.double()).abs().max()) <= 2.0 ** -7 * float(q.abs().max())


@pytest.mark.parametrize("dtype,width,extra", [("bf16", 1638, 2), ("f16", 64, 0), ("f32", 33, 1)])
def test_rows_of_the_low_rank_cache_are_copied(dn, dtype, width, extra):
    import torch
    bits = {"f32": torch.int32}.get(dtype, torch.int16)
    rows, n_slots = 21, 40
    t = torch.randint(-2 ** 15, 2 ** 15 - 1, (rows, width + extra), device="cuda").to(bits).view(kind_of(dtype))[:, :width]      # any bits, NaN among them
    pool = torch.zeros((n_slots, width + extra), dtype=t.dtype, device="cuda")
    slots = np.random.default_rng(5).permutation(n_slots)[:rows]
    dn.deinfer_rope_store(None, t, None, None, None, 0, 1, width, slots=ints(slots), k_out=pool[:, :width])
    want = torch.zeros_like(pool).view(bits)
    want[torch.tensor(slots, device="cuda").long(), :width] = t.contiguous().view(bits)
    assert torch.equal(pool.view(bits), want)


# ------------------------------------------------------------------ attention
def cache_case(seed, cached, new, n_kv, D, bt, dtype, extra_pitch=0, spare=3, scale=1.0):
    """Pools full of NaN but for the slots in use; block table over a shuffled pool."""
    import torch
    rng = np.random.default_rng(seed)
    lengths = [c + m for c, m in zip(cached, new)]
    owned = [-(-n // bt) for n in lengths]
    n_blocks = sum(owned) + spare
    ids = rng.permutation(n_blocks)
    pitch = max(owned + [1]) + 1
    table = np.full((len(cached), pitch), -1)
    at = 0
    for s, n in enumerate(owned):
        table[s, :n] = ids[at:at + n]
        at += n
    w = n_kv * D
    pools = [torch.full((n_blocks * bt, w + extra_pitch), float("nan"), dtype=kind_of(dtype), device="cuda") for _ in range(2)]
    for s, n in enumerate(lengths):
        if n:
            slots = torch.tensor([int(table[s, t // bt]) * bt + t % bt for t in range(n)], device="cuda")
            for i, p in enumerate(pools):
                p[slots, :w] = torch.tensor(normal(seed * 100 + 2 * s + i, n, w) * scale, device="cuda").to(p.dtype)
    return table, pools[0][:, :w], pools[1][:, :w]


def check_attention(dn, q, k, v, table, start, cached, n_q, n_kv, bt, dtype, mask=None, scale=None, out=None, stream=None):
    import torch
    T, D = q.shape[0], q.shape[1] // n_q
    ws = dn.Workspace(dn.deinfer_tree_attention_workspace_bytes(T, len(cached), n_q, n_kv, D))
    if out is None:
        out = torch.full((T, n_q * D), 3.0, dtype=q.dtype, device="cuda")
    sc = D ** -0.5 if scale is None else scale
    dn.deinfer_tree_attention(q, k, v, ints(table), ints(start), ints(cached), ws, n_q, n_kv, bt, scale=scale,
                              mask=None if mask is None else torch.tensor(np.array(mask, dtype=np.uint32).view(np.int32), device="cuda"), out=out)
    torch.cuda.synchronize()
    kh, vh = np.nan_to_num(wide(k)), np.nan_to_num(wide(v))
    ref = cs.attention(wide(q), kh, vh, table, start, cached, n_q, n_kv, bt, sc, mask=mask, out=np.full((T, n_q * D), 3.0))
    size = cs.attention(wide(q), kh, np.abs(vh), table, start, cached, n_q, n_kv, bt, sc, mask=mask, out=np.zeros((T, n_q * D)))
    got = wide(out)
    longest = max([c + int(start[s + 1]) - int(start[s]) for s, c in enumerate(cached)] + [1])
    tol = HALF[dtype] * (np.abs(ref) + size) * 1.01 + 4e-4 * size + (longest * 2.0 ** -25 * np.max(np.abs(vh)) if dtype == "f16" else 0.0)
    n = int(start[-1])
    assert np.all(np.isfinite(got))
    assert np.all(np.abs(got - ref)[:n] <= tol[:n]), float(np.max((np.abs(got - ref) / np.maximum(tol, 1e-30))[:n]))
    assert np.all(got[n:] == 3.0)                                   # padding rows: as they were
    return got


ATTEND = [
    # cached, new, q heads, kv heads, head dim, block tokens, type, tree words (0: causal), more rows
    ([0], [1], 1, 1, 64, 16, "bf16", 0, 0),                          # one token that sees itself
    ([1, 15, 16, 17, 31, 32, 33, 127, 128, 129], [1] * 10, 8, 1, 128, 16, "bf16", 0, 2),
    ([1000, 3, 0, 517], [1, 1, 1, 1], 16, 2, 128, 16, "f16", 0, 0),
    ([700], [1], 7, 1, 80, 32, "bf16", 0, 0),
    ([40, 41], [1, 1], 4, 4, 8, 16, "bf16", 0, 1),
    ([90, 0], [1, 1], 6, 2, 72, 8, "f16", 0, 0),                     # blocks of eight
    ([90, 5], [2, 1], 2, 2, 256, 16, "bf16", 0, 0),
    ([300, 64], [1, 3], 5, 1, 200, 64, "bf16", 0, 0),
    ([50, 60], [1, 1], 4, 2, 64, 1, "bf16", 0, 0),                   # blocks of one
    ([50, 60], [3, 1], 4, 2, 128, 48, "f16", 0, 0),                  # no power of two
    ([5000], [1], 8, 1, 128, 16, "bf16", 0, 0),                      # one sequence over many workgroups
    ([20, 0, 9], [5, 9, 1], 8, 2, 64, 16, "bf16", 1, 3),
    ([300, 77], [33, 20], 8, 2, 128, 16, "bf16", 2, 0),              # more rows than one tile
    ([100, 31, 64], [64, 40, 2], 4, 1, 128, 32, "f16", 2, 5),
    ([17], [100], 3, 1, 96, 16, "bf16", 4, 0),
    ([64, 0], [70, 130], 4, 4, 64, 16, "bf16", 0, 0),                # chunks of prompts
    ([33], [300], 6, 2, 128, 16, "f16", 0, 1),
    ([0], [257], 2, 1, 128, 8, "bf16", 0, 0),
    ([12, 3], [0, 2], 4, 1, 64, 16, "bf16", 0, 0),                   # a sequence without rows
    ([12], [40], 4, 1, 64, 16, "bf16", 1, 0),                        # rows without a bit in the mask's one word
]


def random_mask(rng, new, words, T, own=True):
    m = np.zeros((T, words), dtype=np.uint32)
    at = 0
    for n in new:
        for i in range(n):
            for j in range(min(n, 32 * words)):
                if (own and j == i) or rng.random() < 0.4:
                    m[at + i, j // 32] |= np.uint32(1 << (j % 32))
        at += n
    return m


@pytest.mark.parametrize("cached,new,hq,hk,D,bt,dtype,words,extra", ATTEND)
def test_attention(dn, cached, new, hq, hk, D, bt, dtype, words, extra):
    import torch
    seed = D + len(cached)
    table, k, v = cache_case(seed, cached, new, hk, D, bt, dtype)
    start = np.concatenate([[0], np.cumsum(new)])
    T = int(start[-1]) + extra
    q = torch.tensor(normal(seed, T, hq * D), device="cuda").to(kind_of(dtype))
    mask = random_mask(np.random.default_rng(seed), new, words, T) if words else None
    check_attention(dn, q, k, v, table, start, cached, hq, hk, bt, dtype, mask)


def test_attention_of_many_ragged_sequences(dn):
    """More sequences than threads of a workgroup, and lengths that differ a hundredfold."""
    import torch
    rng = np.random.default_rng(1)
    cached = (np.exp(rng.uniform(0, 6, 300))).astype(int)
    new = rng.integers(0, 3, 300)
    table, k, v = cache_case(3, cached, new, 1, 64, 16, "bf16")
    start = np.concatenate([[0], np.cumsum(new)])
    q = torch.tensor(normal(5, int(start[-1]) + 7, 2 * 64), device="cuda").to(torch.bfloat16)
    check_attention(dn, q, k, v, table, start, cached, 2, 1, 16, "bf16")


def test_attention_strides_and_large_scores(dn):
    """q inside a wider qkv row, keys and values side by side in one pool, out in a wider row; scores up to about 100."""
    import torch
    cached, new, hq, hk, D, bt = [70, 129, 9], [3, 1, 2], 4, 2, 64, 16
    table, k0, v0 = cache_case(4, cached, new, hk, D, bt, "bf16", scale=4.0)
    both = torch.full((k0.shape[0], 2 * hk * D + 8), float("nan"), dtype=torch.bfloat16, device="cuda")
    both[:, :hk * D], both[:, hk * D + 8:] = k0, v0
    rows = torch.tensor(normal(6, 6, 3 * hq * D) * 4.0, device="cuda").to(torch.bfloat16)
    out = torch.full((6, hq * D + 16), 3.0, dtype=torch.bfloat16, device="cuda")
    check_attention(dn, rows[:, hq * D:2 * hq * D], both[:, :hk * D], both[:, hk * D + 8:], table, np.array([0, 3, 4, 6]), cached, hq, hk, bt, "bf16",
                    scale=0.4, out=out[:, :hq * D])
    assert bool((out[:, hq * D:] == 3.0).all())


@pytest.mark.parametrize("words,new", [(1, [4, 3]), (2, [64, 50])])
def test_attention_rows_that_see_nothing(dn, words, new):
    import torch
    cached, hq, hk, D, bt = [0, 40], 4, 1, 64, 16
    table, k, v = cache_case(8, cached, new, hk, D, bt, "bf16")
    start = np.concatenate([[0], np.cumsum(new)])
    T = int(start[-1])
    q = torch.tensor(normal(9, T, hq * D), device="cuda").to(torch.bfloat16)
    mask = random_mask(np.random.default_rng(2), new, words, T, own=False)
    mask[1] = 0                                                      # nothing cached, nothing drafted
    got = check_attention(dn, q, k, v, table, start, cached, hq, hk, bt, "bf16", mask)
    assert np.all(got[1] == 0.0)


@pytest.mark.parametrize("bt", [16, 8])
@pytest.mark.parametrize("new", [[1, 1], [60, 50]])
def test_attention_leaves_out_blocks_outside_the_pool(dn, bt, new):
    import torch
    cached, hq, hk, D = [100, 40], 4, 1, 128
    table, k, v = cache_case(10, cached, new, hk, D, bt, "bf16")
    table[0, 2], table[0, 4], table[1, 0] = -1, k.shape[0] // bt, 1 << 30
    start = np.concatenate([[0], np.cumsum(new)])
    q = torch.tensor(normal(11, int(start[-1]), hq * D), device="cuda").to(torch.bfloat16)
    check_attention(dn, q, k, v, table, start, cached, hq, hk, bt, "bf16")


def test_attention_of_a_table_that_is_too_short(dn):
    """Keys beyond the table's row are not seen, whatever the lengths say."""
    import torch
    table, k, v = cache_case(12, [40, 20], [1, 1], 1, 64, 16, "bf16")
    q = torch.tensor(normal(13, 2, 64), device="cuda").to(torch.bfloat16)
    check_attention(dn, q, k, v, table[:, :2], np.array([0, 1, 2]), [40, 20], 1, 1, 16, "bf16")
    check_attention(dn, q, k, v, table[:, :1], np.array([0, 1, 2]), [4000, 20], 1, 1, 16, "bf16")


@pytest.mark.parametrize("bt", [16, 8])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("hq,new", [(2, 4), (8, 40)])
def test_values_and_keys_that_are_no_numbers_stay_with_the_rows_that_see_them(dn, bt, value, hq, new):
    """Token 1 of a drafted tree has such a value and such a key: rows that do not see it are as without it."""
    import torch
    cached, hk, D, dtype = [37], 1, 128, "bf16"
    table, k, v = cache_case(14, cached, [new], hk, D, bt, dtype)
    start = np.array([0, new])
    q = torch.tensor(normal(15, new, hq * D), device="cuda").to(torch.bfloat16)
    mask = np.zeros((new, 2), dtype=np.uint32)
    for i in range(new):
        mask[i, i // 32] = 1 << (i % 32)                             # itself
        if i != 1:
            mask[i, 0] |= 1                                          # and token 0
    mask[3, 0] |= 2                                                  # row 3 sees token 1
    slot = int(table[0, 38 // bt]) * bt + 38 % bt
    ws = dn.Workspace(dn.deinfer_tree_attention_workspace_bytes(new, 1, hq, hk, D))
    m = torch.tensor(mask.view(np.int32), device="cuda")
    call = lambda: wide(dn.deinfer_tree_attention(q, k, v, ints(table), ints(start), ints(cached), ws, hq, hk, bt, mask=m))
    clean = call()
    others = [i for i in range(new) if i not in (1, 3)]
    v[slot, 5] = value
    got = call()
    # (those rows' sums are formed in another order beside such a value: fp32 sums, and an output step)
    assert np.max(np.abs(got[others] - clean[others])) <= 2 ** -7 * np.max(np.abs(clean))
    for r in (1, 3):
        col = got[r].reshape(hq, D)
        assert not np.any(np.isfinite(col[:, 5])) and np.all(np.isfinite(np.delete(col, 5, axis=1)))
        if np.isinf(value):
            assert np.all(col[:, 5] == value)
    k[slot, 7] = float("nan")
    got = call()
    assert np.max(np.abs(got[others] - clean[others])) <= 2 ** -7 * np.max(np.abs(clean))
    assert np.all(np.isnan(got[[1, 3]]))


def test_a_query_that_is_no_number_stays_in_its_row(dn):
    import torch
    cached, new, hq, hk, D = [300, 20], [1, 2], 8, 1, 64
    table, k, v = cache_case(16, cached, new, hk, D, 16, "bf16")
    q = torch.tensor(normal(17, 3, hq * D), device="cuda").to(torch.bfloat16)
    ws = dn.Workspace(dn.deinfer_tree_attention_workspace_bytes(3, 2, hq, hk, D))
    call = lambda x: wide(dn.deinfer_tree_attention(x, k, v, ints(table), ints([0, 1, 3]), ints(cached), ws, hq, hk, 16)).reshape(3, hq, D)
    clean = call(q)
    bad = q.clone()
    bad[0, 2 * D + 3] = float("nan")
    got = call(bad)
    assert np.all(np.isnan(got[0, 2]))
    got[0, 2] = clean[0, 2]
    assert np.array_equal(got, clean)


def test_attention_is_the_same_every_time(dn):
    import torch
    cached, new, hq, hk, D = [3000, 10, 700], [1, 1, 1], 8, 2, 128
    table, k, v = cache_case(18, cached, new, hk, D, 16, "bf16")
    q = torch.tensor(normal(19, 3, hq * D), device="cuda").to(torch.bfloat16)
    ws = dn.Workspace(dn.deinfer_tree_attention_workspace_bytes(3, 3, hq, hk, D))
    ws.buf.fill_(255)                                                # whatever the workspace holds
    outs = [dn.deinfer_tree_attention(q, k, v, ints(table), ints([0, 1, 2, 3]), ints(cached), ws, hq, hk, 16) for _ in range(5)]
    assert all(torch.equal(outs[0], o) for o in outs[1:])
    assert bool(torch.isfinite(outs[0].float()).all())


# ------------------------------------------------------------------ the calls together
def test_steps_under_one_graph(dn):
    """Lengths in, attention out: kv_step, tree_mask, rope_store, tree_attention captured once and replayed over steps whose lengths,
    trees and block counts differ, on a stream of its own, with eager work between; against the oracle after every replay."""
    import torch
    seqs, bt, hq, hk, D, T, words, n_pool, pitch = 3, 16, 4, 2, 64, 24, 1, 40, 12
    dtype, dev = torch.bfloat16, "cuda"
    z = lambda *s, t=torch.int32: torch.zeros(s, dtype=t, device=dev)
    cached, new, parents, free, first = z(seqs), z(seqs), z(T), z(n_pool), z(1)
    table = torch.full((seqs, pitch), -1, dtype=torch.int32, device=dev)
    qkv = z(T, (hq + 2 * hk) * D, t=dtype)
    q, k, v = qkv[:, :hq * D], qkv[:, hq * D:(hq + hk) * D], qkv[:, (hq + hk) * D:]
    pools = [torch.full((n_pool * bt, hk * D), float("nan"), dtype=dtype, device=dev) for _ in range(2)]
    step = dn.KvStep(z(seqs + 1), z(T), z(T), z(4))
    mask, q_rot, out = z(T, words), z(T, hq * D, t=dtype), z(T, hq * D, t=dtype)
    f, _ = dn.deinfer_rope_frequencies(D, 10000.0, dn.ROPE_BANDS, 8.0, 256.0, 1.0, 4.0)
    freqs = torch.tensor(f, device=dev)
    ws = dn.Workspace(dn.deinfer_tree_attention_workspace_bytes(T, seqs, hq, hk, D))
    stream = torch.cuda.Stream()

    def enqueue():
        dn.deinfer_kv_step(cached, new, table, free, bt, n_pool, T, free_first=first, out=step, stream=stream)
        dn.deinfer_tree_mask(parents, step.row_start, cached, mask, step.positions, stream=stream)
        dn.deinfer_rope_store(q, k, v, step.positions, freqs, hq, hk, D, slots=step.slots, q_out=q_rot, k_out=pools[0], v_out=pools[1], stream=stream)
        dn.deinfer_tree_attention(q_rot, pools[0], pools[1], table, step.row_start, cached, ws, hq, hk, bt, mask=mask, out=out, stream=stream)

    torch.cuda.synchronize()
    stream.wait_stream(torch.cuda.current_stream())
    enqueue()                                                        # nothing to do yet: lengths of zero
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        enqueue()
    free.copy_(ints(np.random.default_rng(0).permutation(n_pool)))
    held = np.zeros(seqs, dtype=int)                                 # tokens in the cache
    used = 0
    for n, lengths in enumerate(([20, 3, 0], [1, 1, 1], [5, 8, 2], [1, 0, 12], [7, 6, 7])):
        rng = np.random.default_rng(n + 50)
        total = sum(lengths)
        j = np.concatenate([np.arange(m) for m in lengths] + [np.zeros(T - total, dtype=int)])
        par = np.maximum(-1, j - (1 if n == 0 else rng.integers(1, 4, T)))
        cached.copy_(ints(held)); new.copy_(ints(lengths)); parents.copy_(ints(par)); first.fill_(used)
        qkv.copy_(torch.tensor(rng.standard_normal(tuple(qkv.shape)), device=dev))
        out.fill_(3.0)
        before = host(table).copy()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = cs.kv_step(held, lengths, before, host(free), used, n_pool, bt, T)
        assert np.array_equal(host(step.slots), want[1]) and np.array_equal(host(table), want[3]) and np.array_equal(host(step.counts), want[4])
        bits, pos = cs.tree(par, want[0], held, words)
        assert np.array_equal(host(step.positions)[:total], pos)
        ref_q = cs.rotate(wide(q)[:total], pos, f, hq, D, False)
        ref_k = cs.rotate(wide(k)[:total], pos, f, hk, D, False)
        close(wide(q_rot)[:total], ref_q, 4 * np.max(np.abs(wide(qkv))), "bf16")
        close(wide(pools[0])[want[1][:total]], ref_k, 4 * np.max(np.abs(wide(qkv))), "bf16")
        assert np.array_equal(wide(pools[1])[want[1][:total]], wide(v)[:total])
        kh, vh = np.nan_to_num(wide(pools[0])), np.nan_to_num(wide(pools[1]))      # (the rotated keys as they are stored)
        ref = cs.attention(wide(q_rot), kh, vh, host(table), want[0], held, hq, hk, bt, D ** -0.5, mask=bits, out=np.full((T, hq * D), 3.0))
        size = cs.attention(wide(q_rot), kh, np.abs(vh), host(table), want[0], held, hq, hk, bt, D ** -0.5, mask=bits, out=np.zeros((T, hq * D)))
        got = wide(out)
        assert np.all(np.abs(got - ref) <= HALF["bf16"] * (np.abs(ref) + size) * 1.01 + 4e-4 * size)
        held = held + (np.array(lengths) if n == 0 else np.minimum(lengths, 1))     # drafted tokens: the first is kept
        used = int(want[4][3])
        # eager work of the program between the replays, on its own stream
        assert int(torch.arange(1000, device=dev).sum()) == 499500
        # a rejected draft's blocks stay in the table beyond the kept tokens: the next step writes those entries anew


def test_attention_over_the_low_rank_cache(dn):
    """The low-rank cache's way on the device alone: rows of t_k, t_v stored by slot, plan, compacting copies, keys rebuilt and
    rotated, values rebuilt, attention with the remapped table; against the oracle on the rebuilt keys and values."""
    import torch
    bt, r, D, hq, hk, d_in, n_pool, buf_blocks = 16, 40, 128, 4, 2, 64, 32, 20
    cached, new = [37, 5, 90], [2, 1, 3]
    T = sum(new)
    pair = lambda s: dn.deinfer_pack_factors(dn.raw_pair(torch.tensor(normal(s, d_in, r) / 8, device="cuda").to(torch.bfloat16),
                                                        torch.tensor(normal(s + 1, r, hk * D) / 6, device="cuda").to(torch.bfloat16)))
    fk, fv = pair(30), pair(32)
    pools = [torch.zeros((n_pool * bt, r), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    free = ints(np.arange(12, 30))
    everything = [torch.tensor(normal(40 + i, sum(cached) + T, r), device="cuda").to(torch.bfloat16) for i in range(2)]
    # what earlier steps have stored, then this step's rows
    zero = ints([0, 0, 0])
    empty = torch.full((3, 9), -1, dtype=torch.int32, device="cuda")
    first = dn.deinfer_kv_step(zero, ints(cached), empty, ints(np.arange(12)), bt, n_pool, sum(cached))
    dn.deinfer_rope_store(None, everything[0][:sum(cached)], everything[1][:sum(cached)], None, None, 0, 1, r, slots=first.slots, k_out=pools[0], v_out=pools[1])
    step = dn.deinfer_kv_step(ints(cached), ints(new), empty, free, bt, n_pool, T)
    dn.deinfer_rope_store(None, everything[0][sum(cached):], everything[1][sum(cached):], None, None, 0, 1, r, slots=step.slots, k_out=pools[0], v_out=pools[1])
    plan, remap, pos = dn.deinfer_kv_compact_plan_device(empty, ints(cached), n_pool, buf_blocks, bt, n_new=ints(new))
    bufs = [torch.zeros((buf_blocks * bt, r), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for p, b in zip(pools, bufs):
        dn.deinfer_kv_compact_copy(p, bt * r * 2, plan, b)
    n_tok = buf_blocks * bt
    ws = dn.Workspace(max(dn.deinfer_workspace_bytes(n_tok, [fk, fv]), dn.deinfer_tree_attention_workspace_bytes(T, 3, hq, hk, D)))
    keys = dn.deinfer_lowrank_up_rope(bufs[0], fk, dn.deinfer_rope_table(pos, D), ws)
    values = dn.deinfer_lowrank_up(bufs[1], fv, ws)
    q = torch.tensor(normal(50, T, hq * D), device="cuda").to(torch.bfloat16)
    got = wide(dn.deinfer_tree_attention(q, keys, values, remap, step.row_start, ints(cached), ws, hq, hk, bt))
    torch.cuda.synchronize()
    # every row of the cache is where the walk says
    order = np.concatenate([np.concatenate([np.arange(sum(cached[:s]), sum(cached[:s + 1])), sum(cached) + np.arange(sum(new[:s]), sum(new[:s + 1]))]) for s in range(3)])
    at = np.concatenate([[int(host(remap)[s, t // bt]) * bt + t % bt for t in range(cached[s] + new[s])] for s in range(3)])
    assert np.array_equal(wide(bufs[0])[at], wide(everything[0])[order]) and np.array_equal(wide(bufs[1])[at], wide(everything[1])[order])
    args = (host(remap), [0, 2, 3, 6], cached, hq, hk, bt, D ** -0.5)
    ref, size = cs.attention(wide(q), wide(keys), wide(values), *args), cs.attention(wide(q), wide(keys), np.abs(wide(values)), *args)
    assert np.all(np.abs(got - ref) <= HALF["bf16"] * (np.abs(ref) + size) * 1.01 + 4e-4 * size)
    assert np.array_equal(host(pos)[at], np.concatenate([np.arange(c + m) for c, m in zip(cached, new)]))
