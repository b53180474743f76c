"""Attention over the paged cache where the scores are not those of an ordinary step: one key far above all others (whose
weight may still be nearly all of the output, if that key's value is zero), scores of any size that fp32 has.  Against the
formula in 64 bits.

Tolerance of a long tail, relative to the output itself (all values have one sign): the probabilities' rounding and the output's,
half a step each, h = 2^-11 for fp16 and 2^-8 for bf16, and the numerator's and the sum's additions in fp32: one per 32 keys,
4100 2^-24 = 2.5e-4 each for the longest case.  Scores are exact products, their exponents' arguments below 32 in size: 2^-20."""
import numpy as np
import pytest

from test_gpu_cache_step import HALF, cache_case, check_attention, dn, ints, kind_of, random_mask, wide  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("spread", [0.0, 1.0])
@pytest.mark.parametrize("first", [True, False])
@pytest.mark.parametrize("keys,above", [(16384, 16.0), (131072, 17.5)])
@pytest.mark.parametrize("new,D,dtype,seqs", [(1, 64, "f16", 512), (1, 128, "bf16", 512), (20, 64, "f16", 256), (40, 128, "f16", 256), (20, 256, "f16", 256), (40, 64, "bf16", 256)])
def test_the_tail_below_one_key_that_has_no_value(dn, new, D, dtype, seqs, keys, above, first, spread):
    """Many sequences over the same blocks, so that a workgroup has a whole sequence: what lies `above` nats below the first
    (the last) key makes up the output."""
    import torch
    hq, bt = 4, 16
    kind = kind_of(dtype)
    rng = np.random.default_rng(keys + new)
    total = keys + new
    sink = 0 if first else keys - 1
    kk = np.zeros((total, D))
    kk[:, 1] = np.round(rng.uniform(-spread, spread, total) * 64) / 64
    kk[sink, 0], kk[sink, 1] = above, 0.0
    vv = rng.uniform(0.5, 1.5, (total, D))
    vv[sink] = 0.0
    pages = -(-total // bt)
    ids = rng.permutation(pages)
    slots = torch.tensor(ids[np.arange(total) // bt] * bt + np.arange(total) % bt, device="cuda")
    k, v = (torch.zeros((pages * bt, D), dtype=kind, device="cuda") for _ in range(2))
    k[slots], v[slots] = torch.tensor(kk, device="cuda").to(kind), torch.tensor(vv, device="cuda").to(kind)
    q = torch.zeros((seqs * new, hq * D), dtype=kind, device="cuda")
    q.view(seqs * new, hq, D)[:, :, :2] = 1.0
    table = ints(np.tile(ids, (seqs, 1)))
    ws = dn.Workspace(dn.deinfer_tree_attention_workspace_bytes(seqs * new, seqs, hq, 1, D))
    got = wide(dn.deinfer_tree_attention(q, k, v, table, ints(np.arange(seqs + 1) * new), ints([keys] * seqs), ws, hq, 1, bt, scale=1.0)).reshape(seqs, new, hq, D)
    kh, vh = wide(k[slots]), wide(v[slots])
    w = np.exp(kh[:, 0] + kh[:, 1] - above)
    for i in range(new):
        n = keys + i + 1
        ref = w[:n] @ vh[:n] / np.sum(w[:n])
        off = np.max(np.abs(got[:, i] - ref) / ref)
        assert off <= 2.02 * HALF[dtype] + 6e-4, (i, off)


@pytest.mark.parametrize("words", [0, 2])
@pytest.mark.parametrize("new,D", [([1, 1], 64), ([3, 2], 128), ([20, 9], 128), ([40, 33], 64), ([40, 33], 128), ([20, 30], 256)])
@pytest.mark.parametrize("dtype,sizes", [("bf16", [1.0, 100.0, 1e6, 1e9, 1e12, 1e20, 1e30, 5e36]), ("f16", [1e-3, 0.1, 10.0, 1000.0, 60000.0])])
def test_scores_of_any_size(dn, dtype, sizes, new, D, words):
    """A row's scores are one factor of its own, up to 5e36 and of either sign, times a number of the key: from an ordinary
    softmax to one key (or a few with the same number) that has all the weight.  The scores are exact in fp32, and where they are large
    any two that differ are a weight of nothing apart, so the tolerance is that of ordinary ones."""
    import torch
    cached, hq, hk, bt = [700, 130], 4, 1, 16
    table, k, v = cache_case(51, cached, new, hk, D, bt, dtype)
    rng = np.random.default_rng(4)
    start = np.concatenate([[0], np.cumsum(new)])
    T = int(start[-1])
    kk = torch.zeros((k.shape[0], D), dtype=torch.float64)
    kk[:, 3] = torch.tensor(np.clip(rng.standard_normal(k.shape[0]), -4, 4) * (8000.0 if dtype == "f16" else 1.0))
    k[:] = torch.where(torch.isnan(k), k, kk.to(k.dtype).cuda())
    q = torch.zeros((T, hq, D), dtype=torch.float64)
    q[:, :, 3] = torch.tensor(rng.choice(sizes, (T, hq)) * rng.choice([-1.0, 1.0], (T, hq)))
    mask = random_mask(rng, new, words, T) if words else None
    check_attention(dn, q.view(T, hq * D).to(k.dtype).cuda(), k, v, table, start, cached, hq, hk, bt, dtype, mask, scale=1.0)


@pytest.mark.parametrize("new,D", [([1], 64), ([20], 128), ([40], 64), ([20], 256)])
@pytest.mark.parametrize("dtype,q_value,k_value", [("bf16", 1e16, -1e16), ("bf16", 1e9, 2.0), ("bf16", 2.0 ** 62, -2.0 ** 63), ("f16", 60000.0, -30000.0), ("f16", 60000.0, 400.0)])
def test_equal_scores_of_any_size(dn, dtype, q_value, k_value, new, D):
    """Every score of a row is the same number, however large: every key that it sees has the same weight."""
    import torch
    cached, hq, hk, bt = [500], 4, 1, 16
    table, k, v = cache_case(53, cached, new, hk, D, bt, dtype)
    kk = torch.zeros_like(k)
    kk[:, 0] = k_value
    k[:] = torch.where(torch.isnan(k), k, kk)
    q = torch.zeros((new[0], hq, D), dtype=k.dtype, device="cuda")
    q[:, :, 0] = q_value
    check_attention(dn, q.view(new[0], hq * D), k, v, table, np.array([0, new[0]]), cached, hq, hk, bt, dtype, scale=1.0)


@pytest.mark.parametrize("D,new,hq", [(64, 4, 2), (128, 4, 4), (128, 20, 4), (64, 50, 4), (256, 40, 4)])
@pytest.mark.parametrize("value", [float("inf"), -float("inf"), float("nan")])
def test_fp16_values_that_are_no_numbers(dn, D, new, hq, value):
    """A drafted token's value is no number: rows whose mask leaves it out stay within the tolerance of finite values of the formula
    (those of ``check_attention``), the others have it in that feature alone."""
    cached, bt, bad = [90], 16, 1
    table, k, v = cache_case(55, cached, [new], 1, D, bt, "f16")
    rng = np.random.default_rng(7)
    mask = random_mask(rng, [new], 2, new)
    mask[0, 0] &= ~np.uint32(1 << bad)
    mask[new - 1, 0] |= np.uint32(1 << bad)
    import torch
    q = torch.tensor(rng.standard_normal((new, hq * D)), device="cuda").half()
    want = check_attention(dn, q, k, v, table, np.array([0, new]), cached, hq, 1, bt, "f16", mask).reshape(new, hq, D)
    slot = int(table[0, (cached[0] + bad) // bt]) * bt + (cached[0] + bad) % bt
    v[slot, 3] = value
    ws = dn.Workspace(dn.deinfer_tree_attention_workspace_bytes(new, 1, hq, 1, D))
    got = wide(dn.deinfer_tree_attention(q, k, v, ints(table), ints([0, new]), ints(cached), ws, hq, 1, bt, mask=ints(mask.view(np.int32)))).reshape(new, hq, D)
    sees = (mask[:, 0] >> np.uint32(bad)) & 1 != 0
    assert sees.any() and not sees.all()
    # (beside such a value the sums are formed one key at a time: fp32 sums in another order, 123 keys 2^-24, and a step of the output)
    close = lambda a, b: np.all(np.abs(a - b) <= 2 * HALF["f16"] * np.abs(b) + 2e-5 * np.max(np.abs(want)) + 2.0 ** -24)
    assert close(got[~sees], want[~sees])
    assert close(np.delete(got[sees], 3, axis=2), np.delete(want[sees], 3, axis=2))
    assert np.all(np.isnan(got[sees][:, :, 3]) if value != value else got[sees][:, :, 3] == value)
