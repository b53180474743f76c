"""The calls between the projections of a prompt where they can go wrong.  Tolerances: as in test_gpu_prompt.py."""
import numpy as np
import pytest

from oracle import prompt as op
from test_gpu_cache_step import HALF, dn, host, ints, kind_of, normal, wide  # noqa: F401
from test_gpu_prompt import angles_of, check_norm, packed

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
