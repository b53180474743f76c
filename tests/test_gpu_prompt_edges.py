"""The calls between the projections of a prompt where they can go wrong.  Tolerances: as in test_gpu_prompt.py."""
import numpy as np
import pytest

from oracle import prompt as op
from test_gpu_cache_step import HALF, dn, ints, kind_of, wide  # noqa: F401
from test_gpu_prompt import packed

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
