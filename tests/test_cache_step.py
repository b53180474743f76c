"""Host side of the calls around a paged cache: refusals (no call here reaches a launch) and the frequencies of rotary
positions, which are formed on the host."""
import ctypes

import numpy as np
import pytest

import paper_2604_17709_amd as dn
from oracle import cache_step as cs

FAKE = 0x7f0000000000        # 256-byte aligned, never dereferenced
N = [FAKE + 0x100000 * i for i in range(12)]


def step(cached=N[0], n_new=N[1], n_seqs=4, free=N[2], n_free=8, first=None, pool=64, bt=16, table=N[3], pitch=8, T=32,
         row_start=N[4], slots=N[5], positions=N[6], counts=N[7]):
    return dn.lib().deinfer_kv_step(cached, n_new, n_seqs, free, n_free, first, pool, bt, table, pitch, T, row_start, slots, positions, counts, None)


def test_step_refusals():
    for bad in (dict(n_seqs=-1), dict(n_free=-1), dict(pool=-1), dict(bt=0), dict(pitch=-1), dict(T=-1), dict(cached=None), dict(n_new=None),
                dict(table=None), dict(free=None), dict(row_start=None), dict(slots=None), dict(positions=None), dict(counts=None),
                dict(first=N[7] + 12), dict(pool=1 << 28, bt=16), dict(pitch=1 << 28, bt=16)):
        assert step(**bad) == dn.ERR_INVALID_ARG, bad
    assert step(n_seqs=8193) == dn.ERR_UNSUPPORTED and "8192" in dn.last_error()
    assert step(T=(1 << 28) + 1) == dn.ERR_UNSUPPORTED
    assert step(slots=N[5] + 2) == dn.ERR_MISALIGNED
    assert step(T=0, row_start=None, slots=None, positions=None, counts=None) == dn.OK


def plan(table=N[0], n_seqs=4, pitch=8, tokens=N[1], new=None, pool=64, buf=32, bt=16, out=N[2], cap=32, remap=N[3], rpitch=8, pos=N[4]):
    return dn.lib().deinfer_kv_compact_plan_device(table, n_seqs, pitch, tokens, new, pool, buf, bt, out, cap, remap, rpitch, pos, None)


def test_plan_refusals():
    for bad in (dict(n_seqs=-1), dict(pitch=-1), dict(pool=-1), dict(buf=-1), dict(cap=-1), dict(rpitch=-1), dict(bt=0), dict(table=None),
                dict(tokens=None), dict(out=None), dict(buf=1 << 27), dict(cap=1 << 30)):
        assert plan(**bad) == dn.ERR_INVALID_ARG, bad
    assert plan(n_seqs=8193) == dn.ERR_UNSUPPORTED
    for bad in (dict(out=N[2] + 1), dict(remap=N[3] + 2), dict(pos=N[4] + 1), dict(new=N[5] + 3)):
        assert plan(**bad) == dn.ERR_MISALIGNED, bad


def mask(parents=N[0], row_start=N[1], cached=N[2], n_seqs=4, T=32, out=N[3], words=2, pos=N[4]):
    return dn.lib().deinfer_tree_mask(parents, row_start, cached, n_seqs, T, out, words, pos, None)


def test_tree_mask_refusals():
    for bad in (dict(n_seqs=-1), dict(T=-1), dict(words=0), dict(parents=None), dict(row_start=None), dict(cached=None), dict(out=None)):
        assert mask(**bad) == dn.ERR_INVALID_ARG, bad
    assert mask(words=33) == dn.ERR_UNSUPPORTED
    assert mask(n_seqs=8193) == dn.ERR_UNSUPPORTED
    assert mask(out=N[3] + 2) == dn.ERR_MISALIGNED
    assert mask(T=0, parents=None) == dn.OK and mask(n_seqs=0, cached=None) == dn.OK


def rope(q=N[0], ldq=64, nq=2, k=N[1], ldk=32, v=N[2], ldv=32, nkv=1, T=4, D=32, rot=32, inter=0, pos=N[3], freqs=N[4], mag=1.0,
         slots=N[5], n_slots=64, qo=N[6], ldqo=64, ko=N[7], ldko=32, vo=N[8], ldvo=32, dtype=dn.BF16):
    return dn.lib().deinfer_rope_store(q, ldq, nq, k, ldk, v, ldv, nkv, T, D, rot, inter, pos, freqs, mag, slots, n_slots, qo, ldqo, ko, ldko,
                                       vo, ldvo, dtype, None)


def test_rope_store_refusals():
    for bad in (dict(T=-1), dict(nq=-1), dict(nkv=-1), dict(D=0), dict(n_slots=-1), dict(rot=31), dict(rot=34), dict(rot=-2), dict(mag=float("nan")),
                dict(mag=float("inf")), dict(qo=None), dict(q=None), dict(ko=None), dict(vo=None), dict(nq=0), dict(nkv=0), dict(ldq=63),
                dict(ldqo=63), dict(ldk=31), dict(ldko=31), dict(ldv=31), dict(ldvo=31), dict(pos=None), dict(freqs=None), dict(ko=N[1]),
                dict(vo=N[2]), dict(qo=N[0], ldqo=72)):
        assert rope(**bad) == dn.ERR_INVALID_ARG, bad
    assert rope(dtype=7) == dn.ERR_UNSUPPORTED
    assert rope(D=2048, rot=1026, ldq=4096, ldqo=4096, ldk=2048, ldko=2048, ldv=2048, ldvo=2048) == dn.ERR_UNSUPPORTED
    assert rope(D=33, rot=2, inter=1, ldq=66, ldqo=66, ldk=33, ldko=33, ldv=33, ldvo=33) == dn.ERR_UNSUPPORTED
    for bad in (dict(q=N[0] + 1), dict(ko=N[7] + 1), dict(pos=N[3] + 2), dict(freqs=N[4] + 4), dict(slots=N[5] + 2)):
        assert rope(**bad) == dn.ERR_MISALIGNED, bad
    assert rope(T=0) == dn.OK


def attend(q=N[0], T=8, ldq=256, nq=4, nkv=2, D=64, row_start=N[1], cached=N[2], n_seqs=2, mask=None, words=0, k=N[3], ldk=128, v=N[4], ldv=128,
           pool=64, bt=16, table=N[5], pitch=8, scale=0.125, out=N[6], ldo=256, dtype=dn.BF16, ws=N[7], nbytes=None):
    if nbytes is None:
        nbytes = 1 << 33
    return dn.lib().deinfer_tree_attention(q, T, ldq, nq, nkv, D, row_start, cached, n_seqs, mask, words, k, ldk, v, ldv, pool, bt, table, pitch,
                                           scale, out, ldo, dtype, ws, nbytes, None)


def test_attention_refusals():
    for bad in (dict(T=-1), dict(nq=0), dict(nkv=0), dict(nkv=3), dict(n_seqs=-1), dict(pool=-1), dict(pitch=-1), dict(bt=0), dict(scale=0.0),
                dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(mask=N[8], words=0), dict(mask=N[8], words=33), dict(ldq=255),
                dict(ldo=255), dict(ldk=127), dict(ldv=127), dict(pool=0), dict(pitch=0), dict(q=None), dict(k=None), dict(v=None), dict(out=None),
                dict(row_start=None), dict(cached=None), dict(table=None), dict(out=N[0]), dict(pool=1 << 28, bt=16)):
        assert attend(**bad) == dn.ERR_INVALID_ARG, bad
    for bad in (dict(dtype=dn.F32), dict(dtype=5), dict(D=60), dict(D=264, ldq=1056, ldo=1056, ldk=528, ldv=528), dict(D=0), dict(n_seqs=8193), dict(T=(1 << 28) + 1),
                dict(ldk=(1 << 26) + 8), dict(ldv=(1 << 26) + 8)):
        assert attend(**bad) == dn.ERR_UNSUPPORTED, bad
    for bad in (dict(q=N[0] + 8), dict(k=N[3] + 2), dict(v=N[4] + 8), dict(out=N[6] + 8), dict(ldq=260), dict(ldo=257), dict(ldk=132), dict(ldv=132),
                dict(table=N[5] + 2), dict(mask=N[8] + 1, words=1), dict(ws=N[7] + 128)):
        assert attend(**bad) == dn.ERR_MISALIGNED, bad
    assert attend(ws=None) == dn.ERR_WORKSPACE
    need = dn.deinfer_tree_attention_workspace_bytes(8, 2, 4, 2, 64)
    assert need > 0
    assert attend(nbytes=need - 1) == dn.ERR_WORKSPACE and str(need) in dn.last_error()
    assert attend(T=0, q=None) == dn.OK and attend(n_seqs=0, q=None) == dn.OK


def test_attention_refuses_a_scale_that_fp32_cannot_hold():
    for scale in (1e-46, 1e-39, 3e38, 1e300):
        assert attend(scale=scale) == dn.ERR_UNSUPPORTED, scale


def test_a_call_with_fewer_sequences_may_need_a_larger_workspace():
    """More rows per sequence take larger tiles; with as many sequences, more rows never need less."""
    sizes = [dn.deinfer_tree_attention_workspace_bytes(T, 8, 32, 8, 128) for T in (1, 8, 33, 300, 600, 5000)]
    assert sizes == sorted(sizes)
    assert dn.deinfer_tree_attention_workspace_bytes(600, 2, 32, 8, 128) > dn.deinfer_tree_attention_workspace_bytes(600, 600, 32, 8, 128)


def test_attention_workspace_refusals():
    for bad in ((-1, 1, 1, 1, 64), (1, -1, 1, 1, 64), (1, 1, 0, 1, 64), (1, 1, 4, 3, 64), (1, 1, 1, 1, 0)):
        with pytest.raises(dn.DeinferError) as e:
            dn.deinfer_tree_attention_workspace_bytes(*bad)
        assert e.value.code == dn.ERR_INVALID_ARG
    with pytest.raises(dn.DeinferError) as e:
        dn.deinfer_tree_attention_workspace_bytes(1, 1, 1, 1, 512)
    assert e.value.code == dn.ERR_UNSUPPORTED
    assert dn.lib().deinfer_tree_attention_workspace_bytes(1, 1, 1, 1, 64, None) == dn.ERR_INVALID_ARG


@pytest.mark.parametrize("rot_dim,theta,kind,factor,context,low,high", [
    (128, 10000.0, "plain", 1.0, 0.0, 0.0, 0.0),
    (2, 10000.0, "plain", 1.0, 0.0, 0.0, 0.0),
    (64, 500000.0, "linear", 4.0, 0.0, 0.0, 0.0),
    (128, 10000.0, "base", 8.0, 0.0, 0.0, 0.0),
    (128, 500000.0, "bands", 8.0, 8192.0, 1.0, 4.0),
    (20, 10000.0, "bands", 2.0, 100.0, 1.0, 4.0),
    (128, 10000.0, "ramp", 16.0, 4096.0, 1.0, 32.0),
    (64, 10000.0, "ramp", 0.5, 64.0, 1.0, 32.0),         # shorter, magnitude 1
    (8, 1.0e6, "ramp", 4.0, 7.0, 1.0, 1.0001),           # both borders in one pair
])
def test_frequencies(rot_dim, theta, kind, factor, context, low, high):
    kinds = {"plain": dn.ROPE_PLAIN, "linear": dn.ROPE_LINEAR, "base": dn.ROPE_BASE, "bands": dn.ROPE_BANDS, "ramp": dn.ROPE_RAMP}
    got, magnitude = dn.deinfer_rope_frequencies(rot_dim, theta, kinds[kind], factor, context, low, high)
    want, m = cs.frequencies(rot_dim, theta, kind, factor, context, low, high)
    # powers, logarithms and a handful of products in 64 bits: a few parts in 1e16 each, the blend's difference of a few
    # hundred turns included
    assert np.max(np.abs(got / want - 1)) <= 1e-12 and abs(magnitude - m) <= 1e-12
    assert got.shape == (rot_dim // 2,)
    if kind in ("bands", "ramp"):                         # fast pairs stay, slow ones are divided
        plain, _ = cs.frequencies(rot_dim, theta)
        assert np.all(got <= plain * (1 + 1e-12) if factor > 1 else got >= plain * (1 - 1e-12))
        assert abs(got[-1] / (plain[-1] / factor) - 1) <= 1e-12


def test_frequencies_refusals():
    L = dn.lib()
    f = (ctypes.c_double * 64)()
    sc = dn.RopeScaling(dn.ROPE_RAMP, 4.0, 4096.0, 1.0, 32.0)
    ok = lambda rot=64, theta=1e4, s=sc, to=f: L.deinfer_rope_frequencies(rot, theta, None if s is None else ctypes.byref(s), to, None)
    assert ok() == dn.OK and ok(s=None) == dn.OK
    for rot in (0, -2, 3, 1026):
        assert ok(rot=rot) == dn.ERR_INVALID_ARG
    for theta in (0.0, -1.0, float("nan"), float("inf"), 0.5):
        assert ok(theta=theta) == dn.ERR_INVALID_ARG
    assert ok(to=None) == dn.ERR_INVALID_ARG
    R = dn.RopeScaling
    for s in (R(dn.ROPE_LINEAR, 0.0, 0, 0, 0), R(dn.ROPE_LINEAR, float("nan"), 0, 0, 0), R(dn.ROPE_BANDS, 4.0, 0.0, 1, 4), R(dn.ROPE_BANDS, 4.0, 100.0, 4, 4),
              R(dn.ROPE_RAMP, 4.0, 100.0, 0, 4), R(dn.ROPE_RAMP, 4.0, 100.0, 1, float("inf"))):
        assert ok(s=s) == dn.ERR_INVALID_ARG
    assert ok(s=R(9, 2.0, 0, 0, 0)) == dn.ERR_UNSUPPORTED
    assert ok(rot=2, s=R(dn.ROPE_BASE, 2.0, 0, 0, 0)) == dn.ERR_INVALID_ARG


def test_the_binding_refuses_host_tensors_and_wrong_shapes():
    torch = pytest.importorskip("torch")
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    with pytest.raises(ValueError, match="current device"):
        dn.deinfer_kv_step(i(2), i(2), i(2, 4), i(8), 16, 64, 8)
    with pytest.raises(ValueError, match="n_new"):
        dn.deinfer_kv_step(i(2), i(1), i(2, 4), i(8), 16, 64, 8)
    with pytest.raises(ValueError, match="block_table"):
        dn.deinfer_kv_step(i(2), i(2), i(1, 4), i(8), 16, 64, 8)
    with pytest.raises(ValueError, match="cached"):
        dn.deinfer_kv_step(i(2).long(), i(2), i(2, 4), i(8), 16, 64, 8)
    with pytest.raises(ValueError, match="mask"):
        dn.deinfer_tree_mask(i(8), i(3), i(2), i(4, 1))
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="pools"):
        dn.deinfer_rope_store(x, x, x, i(4), torch.zeros(16, dtype=torch.float64), 2, 2, 32, slots=i(4), q_out=x)
    with pytest.raises(ValueError, match="freqs"):
        dn.deinfer_rope_store(x, x, x, i(4), torch.zeros(16), 2, 2, 32)
    with pytest.raises(ValueError, match="current device"):
        dn.deinfer_rope_store(x, x, x, i(4), torch.zeros(16, dtype=torch.float64), 2, 2, 32)

    class NoWorkspace:
        buf, nbytes = torch.zeros(256, dtype=torch.uint8), 256

    with pytest.raises(ValueError, match="share a dtype"):
        dn.deinfer_tree_attention(x, x.float(), x, i(2, 4), i(3), i(2), NoWorkspace, 2, 2, 4)
    with pytest.raises(ValueError, match="current device"):
        dn.deinfer_tree_attention(x, x, x, i(2, 4), i(3), i(2), NoWorkspace, 2, 2, 4)
