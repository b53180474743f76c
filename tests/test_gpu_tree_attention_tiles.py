"""Attention over the paged cache where a sequence and key head has more than 16 rows: tiles of 128 and 256 rows, long contexts,
many tiles per workgroup; and pools whose offsets pass 32 bits.  Against the 64-bit oracle, with the tolerances of
``check_attention``: the output's rounding, that of the probabilities, and 32-bit arithmetic."""
import numpy as np
import pytest

from test_gpu_cache_step import cache_case, check_attention, dn, ints, kind_of, normal, random_mask  # noqa: F401

pytestmark = pytest.mark.gpu


def queries(seed, T, width, dtype):
    import torch
    return torch.tensor(normal(seed, T, width), device="cuda").to(kind_of(dtype))


LONG = [
    # cached, new, q heads, kv heads, head dim, block tokens, type, tree words
    ([3000], [60], 8, 1, 64, 1, "bf16", 2),                          # more blocks than are looked up at a time
    ([3000, 70], [10, 30], 8, 1, 128, 1, "f16", 0),
    ([5000, 4999], [30, 33], 4, 1, 128, 3, "bf16", 2),               # no power of two, a block that ends inside a row of loads
    ([2500], [20], 4, 1, 256, 2, "bf16", 1),
    ([1500], [130], 2, 1, 256, 16, "f16", 0),
    ([900, 0, 2100], [64, 64, 64], 4, 1, 128, 16, "bf16", 2),        # 256 rows: one tile each
    ([900, 0, 2100], [30, 20, 25], 4, 1, 128, 16, "f16", 1),         # up to 128
    ([130, 640], [400, 300], 4, 2, 64, 16, "bf16", 0),               # several tiles, each with keys of its own
    ([70], [520], 8, 2, 128, 32, "f16", 0),
    ([255, 256, 257, 63, 64, 65], [17] * 6, 4, 2, 128, 16, "bf16", 1),
    ([100, 2], [1024, 40], 1, 1, 40, 16, "bf16", 32),                # the widest mask
]


@pytest.mark.parametrize("cached,new,hq,hk,D,bt,dtype,words", LONG)
def test_tiles(dn, cached, new, hq, hk, D, bt, dtype, words):
    table, k, v = cache_case(D + bt, cached, new, hk, D, bt, dtype)
    start = np.concatenate([[0], np.cumsum(new)])
    T = int(start[-1]) + 3
    mask = random_mask(np.random.default_rng(D), new, words, T) if words else None
    check_attention(dn, queries(1, T, hq * D, dtype), k, v, table, start, cached, hq, hk, bt, dtype, mask)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("new,D", [([3], 128), ([40], 128), ([30], 64), ([40], 256)])
def test_scores_that_rise_along_the_keys(dn, dtype, new, D):
    """Every later key scores higher, by up to 60 in all: each stage wants a new reference, and early keys come to weigh nothing."""
    import torch
    cached, hq, hk, bt = [700], 4, 1, 16
    table, k, v = cache_case(31, cached, new, hk, D, bt, dtype)
    total = cached[0] + new[0]
    slots = torch.tensor([int(table[0, t // bt]) * bt + t % bt for t in range(total)], device="cuda")
    rise = torch.arange(total, device="cuda", dtype=torch.float32)[:, None] / total
    k[slots] = (0.1 * k[slots].float() + rise * 8.0 / D ** 0.5).to(k.dtype)
    T = new[0]
    q = (0.1 * queries(2, T, hq * D, dtype).float() + 8.0).to(kind_of(dtype))
    start = np.array([0, T])
    check_attention(dn, q, k, v, table, start, cached, hq, hk, bt, dtype, scale=60.0 / (64.0 * D ** 0.5))
    check_attention(dn, -q, k, v, table, start, cached, hq, hk, bt, dtype, scale=60.0 / (64.0 * D ** 0.5))


@pytest.mark.parametrize("D,new", [(128, [50, 40]), (128, [20, 8]), (256, [40, 20])])
def test_missing_blocks_in_the_middle(dn, D, new):
    cached, hq, hk, bt = [900, 333], 4, 1, 16
    table, k, v = cache_case(33, cached, new, hk, D, bt, "bf16")
    for page in list(range(8, 13)) + [20, 31, 56]:                   # a whole stage of keys among them
        table[0, page] = -1
    table[1, 0], table[1, 20] = k.shape[0] // bt, -(1 << 31)
    start = np.concatenate([[0], np.cumsum(new)])
    check_attention(dn, queries(3, int(start[-1]), hq * D, "bf16"), k, v, table, start, cached, hq, hk, bt, "bf16")


@pytest.mark.parametrize("D,new", [(128, 50), (128, 20), (256, 40), (64, 100)])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_drafted_values_that_are_no_numbers(dn, D, new, value):
    """A drafted token's value row is infinite or NaN: rows whose mask leaves it out are exactly what they are without it."""
    import torch
    cached, hq, hk, bt, bad = [200], 4, 1, 16, 7
    table, k, v = cache_case(35, cached, [new], hk, D, bt, "bf16")
    q, start = queries(4, new, hq * D, "bf16"), np.array([0, new])
    mask = random_mask(np.random.default_rng(6), [new], 4, new)
    sees = (mask[:, 0] >> np.uint32(bad)) & 1 != 0
    assert sees.any() and not sees.all()
    slot = int(table[0, (cached[0] + bad) // bt]) * bt + (cached[0] + bad) % bt
    ws = dn.Workspace(dn.deinfer_tree_attention_workspace_bytes(new, 1, hq, hk, D))
    run = lambda: dn.deinfer_tree_attention(q, k, v, ints(table), ints(start), ints(cached), ws, hq, hk, bt, mask=ints(mask.view(np.int32)))
    without = run()
    v[slot, ::3] = value
    got = run()
    hidden = torch.tensor(~sees, device="cuda")
    assert torch.equal(got[hidden], without[hidden])
    hit = got[~hidden].view(-1, hq, D)[:, :, ::3].float()
    assert bool((torch.isnan(hit) if value != value else torch.isinf(hit) & (hit > 0)).all())
    rest = torch.ones(D, dtype=torch.bool, device="cuda")
    rest[::3] = False
    assert bool(torch.isfinite(got.view(-1, hq, D)[:, :, rest].float()).all())


def test_more_sequences_than_a_workgroup_has_threads(dn):
    rng = np.random.default_rng(8)
    cached = (np.exp(rng.uniform(0, 5, 700))).astype(int)
    new = rng.integers(0, 30, 700)
    new[:3] = [70, 0, 150]
    table, k, v = cache_case(37, cached, new, 1, 64, 16, "bf16")
    start = np.concatenate([[0], np.cumsum(new)])
    check_attention(dn, queries(5, int(start[-1]), 2 * 64, "bf16"), k, v, table, start, cached, 2, 1, 16, "bf16")


@pytest.mark.parametrize("new", [1, 50])
def test_offsets_past_32_bits(dn, new):
    """The same blocks at the far end of a pool of 5 GB and in one of their own: bit for bit the same."""
    import torch
    cached, hq, hk, D, bt = 300, 16, 16, 128, 16
    table, k, v = cache_case(39, [cached], [new], hk, D, bt, "bf16")
    q = queries(6, new, hq * D, "bf16")
    ws = dn.Workspace(dn.deinfer_tree_attention_workspace_bytes(new, 1, hq, hk, D))
    want = dn.deinfer_tree_attention(q, k, v, ints(table), ints([0, new]), ints([cached]), ws, hq, hk, bt)
    far = 5 * (1 << 30) // (hk * D * 2) // bt
    at = far - k.shape[0] // bt
    big = torch.empty((2, far * bt, hk * D), dtype=torch.bfloat16, device="cuda")
    big[0, at * bt:], big[1, at * bt:] = k, v
    got = dn.deinfer_tree_attention(q, big[0], big[1], ints(np.where(table >= 0, table + at, table)), ints([0, new]), ints([cached]), ws, hq, hk, bt)
    assert torch.equal(got, want)
    # and what is stored there
    slots = ints([(at + 1) * bt + i for i in range(new)])
    rows = queries(7, new, hk * D, "bf16")
    f, _ = dn.deinfer_rope_frequencies(D, 10000.0)
    freqs, pos = torch.tensor(f, device="cuda"), ints(range(new))
    alone = rows.clone()
    dn.deinfer_rope_store(None, alone, None, pos, freqs, hq, hk, D)
    dn.deinfer_rope_store(None, rows, rows, pos, freqs, hq, hk, D, slots=slots, k_out=big[0], v_out=big[1])
    assert torch.equal(big[0][slots.long()], alone) and torch.equal(big[1][slots.long()], rows)


def test_two_graphs_over_one_workspace(dn):
    """Replayed in turn on one stream, with eager calls between: each gives what it gives alone."""
    import torch
    cached, new, hq, hk, D, bt = [500, 40], [40, 1], 8, 2, 128, 16
    table, k, v = cache_case(41, cached, new, hk, D, bt, "bf16")
    start, T = np.array([0, 40, 41]), 41
    ws = dn.Workspace(dn.deinfer_tree_attention_workspace_bytes(T, 2, hq, hk, D))
    one = dn.Workspace(dn.deinfer_tree_attention_workspace_bytes(2, 2, hq, hk, D))
    assert one.nbytes <= ws.nbytes
    qs = [queries(8, T, hq * D, "bf16"), queries(9, 2, hq * D, "bf16")]
    args = [(ints(table), ints(start), ints(cached)), (ints(table), ints([0, 1, 2]), ints(cached))]
    outs = [torch.zeros_like(q) for q in qs]
    run = lambda i, stream=None: dn.deinfer_tree_attention(qs[i], k, v, *args[i], ws, hq, hk, bt, out=outs[i], stream=stream)
    want = [run(0).clone(), run(1).clone()]
    stream, graphs = torch.cuda.Stream(), []
    stream.wait_stream(torch.cuda.current_stream())
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i], stream=stream):
            run(i, stream)
    for _ in range(3):
        for i in range(2):
            outs[i].fill_(float("nan"))
            graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])
        assert torch.equal(run(0), want[0])
        torch.cuda.synchronize()
