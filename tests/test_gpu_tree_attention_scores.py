"""Attention over the paged cache where the scores are not those of an ordinary step: one key far above all others (whose
weight may still be nearly all of the output, if that key's value is zero).  Against the formula in 64 bits.

Tolerance of a long tail, relative to the output itself (all values have one sign): the probabilities' rounding and the output's,
half a step each, h = 2^-11 for fp16 and 2^-8 for bf16, and the numerator's and the sum's additions in fp32: one per 32 keys,
4100 2^-24 = 2.5e-4 each for the longest case.  Scores are exact products, their exponents' arguments below 32 in size: 2^-20."""
import numpy as np
import pytest

from test_gpu_cache_step import HALF, dn, ints, kind_of, wide  # noqa: F401

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
