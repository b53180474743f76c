"""Host code of the calls between the projections of a prompt: refusals, workspace sizes, axes of rotary pairs.  No GPU."""
import ctypes

import numpy as np
import pytest

import paper_2604_17709_amd as dn
from oracle import prompt as op

A = [0x10000 * (i + 1) for i in range(12)]       # addresses that are never read


def places(segments=A[0], n_segments=4, segment_start=A[1], row_start=A[2], cached=A[3], n_seqs=2, T=8, positions=A[4], pitch=8):
    return dn.lib().deinfer_axis_positions(segments, n_segments, segment_start, row_start, cached, n_seqs, T, positions, pitch, None)


def test_axis_positions_refusals():
    for bad in (dict(n_segments=-1), dict(n_seqs=-1), dict(T=-1), dict(pitch=-1), dict(pitch=7), dict(segments=None), dict(segment_start=None),
                dict(row_start=None), dict(positions=None)):
        assert places(**bad) == dn.ERR_INVALID_ARG, bad
    for bad in (dict(n_seqs=8193), dict(T=(1 << 28) + 1, pitch=1 << 30), dict(n_segments=(1 << 28) + 1)):
        assert places(**bad) == dn.ERR_UNSUPPORTED, bad
    for bad in (dict(segments=A[0] + 8), dict(segment_start=A[1] + 2), dict(row_start=A[2] + 1), dict(cached=A[3] + 2), dict(positions=A[4] + 2)):
        assert places(**bad) == dn.ERR_MISALIGNED, bad
    assert places(T=0, positions=None) == dn.OK and places(n_seqs=0, row_start=None) == dn.OK


@pytest.mark.parametrize("pairs", [[8], [3, 5], [16, 24, 24], [0, 4, 1], [1, 2, 3, 4], [40, 0, 0]])
@pytest.mark.parametrize("turns", [False, True])
def test_axes_of_pairs(pairs, turns):
    got = dn.deinfer_rope_axes(2 * sum(pairs), pairs, turns)
    assert got.tolist() == op.rope_axes(pairs, turns)


def test_axes_refusals():
    L, out = dn.lib(), (ctypes.c_uint8 * 64)()
    def axes(rot=16, n=2, pairs=(4, 4), turns=0, to=out):
        return L.deinfer_rope_axes(rot, n, None if pairs is None else (ctypes.c_int32 * 4)(*pairs), turns, to)
    assert axes() == dn.OK
    for bad in (dict(rot=0), dict(rot=15), dict(rot=1026), dict(n=0), dict(n=5), dict(pairs=None), dict(to=None), dict(pairs=(4, 5)), dict(pairs=(9, -1)), dict(pairs=(4, 3))):
        assert axes(**bad) == dn.ERR_INVALID_ARG, bad


def norm(q=A[0], ldq=256, hq=4, k=A[1], ldk=128, v=A[2], ldv=128, hk=2, T=3, D=64, rot=64, inter=0, qw=A[3], kw=A[4], eps=1e-6, pos=A[5], pitch=3, axes=1,
         axis_of=None, freqs=A[6], magnitude=1.0, slots=A[7], n_slots=9, qo=A[8], ldqo=256, ko=A[9], ldko=128, vo=A[10], ldvo=128, dtype=dn.BF16):
    return dn.lib().deinfer_norm_rope_store(q, ldq, hq, k, ldk, v, ldv, hk, T, D, rot, inter, qw, kw, eps, pos, pitch, axes, axis_of, freqs, magnitude, slots, n_slots,
                                            qo, ldqo, ko, ldko, vo, ldvo, dtype, None)


def test_norm_rope_store_refusals():
    for bad in (dict(T=-1), dict(hq=-1), dict(D=0), dict(n_slots=-1), dict(rot=63), dict(rot=66), dict(magnitude=float("nan")), dict(eps=-1e-6), dict(eps=float("nan")),
                dict(eps=float("inf")), dict(eps=1e300), dict(axes=0), dict(axes=5), dict(axes=2), dict(axes=2, axis_of=A[11], pitch=2), dict(qo=None), dict(ko=None), dict(v=None),
                dict(hq=0), dict(hk=0), dict(ldq=255), dict(ldko=127), dict(pos=None), dict(freqs=None), dict(ko=A[1]), dict(qo=A[0], ldqo=264)):
        assert norm(**bad) == dn.ERR_INVALID_ARG, bad
    for bad in (dict(dtype=7), dict(D=2056, ldq=1 << 14, ldk=1 << 14, ldv=1 << 14, ldqo=1 << 14, ldko=1 << 14, ldvo=1 << 14), dict(T=(1 << 28) + 1),
                dict(D=63, rot=62, inter=1)):
        assert norm(**bad) == dn.ERR_UNSUPPORTED, bad
    for bad in (dict(q=A[0] + 1), dict(qw=A[3] + 1), dict(kw=A[4] + 1), dict(vo=A[10] + 1), dict(pos=A[5] + 2), dict(slots=A[7] + 2), dict(freqs=A[6] + 4)):
        assert norm(**bad) == dn.ERR_MISALIGNED, bad
    assert norm(T=0, q=None, k=None) == dn.OK and norm(q=None, qo=None, k=None, ko=None, v=None, vo=None) == dn.OK


def attend(q=A[0], T=8, ldq=256, hq=4, hk=2, D=64, q_start=A[1], k=A[2], ldk=128, v=A[3], ldv=128, n_keys=9, k_start=A[4], n_seqs=2, left=-1, right=0, scale=0.125,
           out=A[5], ldo=256, dtype=dn.BF16, ws=A[6], nbytes=1 << 40):
    return dn.lib().deinfer_prompt_attention(q, T, ldq, hq, hk, D, q_start, k, ldk, v, ldv, n_keys, k_start, n_seqs, left, right, scale, out, ldo, dtype, ws, nbytes, None)


def test_prompt_attention_refusals():
    for bad in (dict(T=-1), dict(n_keys=-1), dict(n_seqs=-1), dict(hq=0), dict(hk=0), dict(hk=3), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
                dict(ldq=248), dict(ldk=120), dict(ldv=120), dict(ldo=248), dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(q_start=None),
                dict(out=A[0]), dict(out=A[2]), dict(out=A[3])):
        assert attend(**bad) == dn.ERR_INVALID_ARG, bad
    big = dict(ldq=4096, ldk=4096, ldv=4096, ldo=4096)
    for bad in (dict(dtype=dn.F32), dict(dtype=9), dict(D=0), dict(D=60), dict(D=264, **big), dict(scale=1e-46), dict(scale=3e38), dict(T=(1 << 28) + 1), dict(n_keys=(1 << 28) + 1),
                dict(n_seqs=8193), dict(ldk=(1 << 26) + 8)):
        assert attend(**bad) == dn.ERR_UNSUPPORTED, bad
    for bad in (dict(q=A[0] + 8), dict(k=A[2] + 8), dict(v=A[3] + 2), dict(out=A[5] + 8), dict(ldq=260), dict(ldk=132), dict(ldv=130), dict(ldo=257), dict(q_start=A[1] + 2),
                dict(k_start=A[4] + 1), dict(ws=A[6] + 64)):
        assert attend(**bad) == dn.ERR_MISALIGNED, bad
    need = dn.deinfer_prompt_attention_workspace_bytes(8, 2, 4, 2, 64)
    assert attend(ws=None) == dn.ERR_WORKSPACE and attend(nbytes=need - 1) == dn.ERR_WORKSPACE and str(need) in dn.last_error()
    assert attend(T=0, q=None) == dn.OK and attend(n_seqs=0, q=None) == dn.OK


def test_prompt_attention_workspace():
    sizes = [dn.deinfer_prompt_attention_workspace_bytes(T, 8, 32, 8, 128) for T in (1, 8, 33, 300, 600, 5000)]
    assert sizes == sorted(sizes)
    for bad in ((-1, 1, 1, 1, 64), (1, -1, 1, 1, 64), (1, 1, 0, 1, 64), (1, 1, 4, 3, 64), (1, 1, 1, 1, 0)):
        with pytest.raises(dn.DeinferError) as e:
            dn.deinfer_prompt_attention_workspace_bytes(*bad)
        assert e.value.code == dn.ERR_INVALID_ARG
    with pytest.raises(dn.DeinferError) as e:
        dn.deinfer_prompt_attention_workspace_bytes(1, 1, 1, 1, 264)
    assert e.value.code == dn.ERR_UNSUPPORTED
    assert dn.lib().deinfer_prompt_attention_workspace_bytes(1, 1, 1, 1, 64, None) == dn.ERR_INVALID_ARG


def test_the_binding_refuses_host_tensors_and_wrong_shapes():
    torch = pytest.importorskip("torch")
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    with pytest.raises(ValueError, match="current device"):
        dn.deinfer_axis_positions(i(4, 4), i(3), i(3), i(2), 8)
    with pytest.raises(ValueError, match="segments"):
        dn.deinfer_axis_positions(i(4, 3), i(3), i(3), i(2), 8)
    with pytest.raises(ValueError, match="row_start"):
        dn.deinfer_axis_positions(i(4, 4), i(3), i(2), i(2), 8)
    with pytest.raises(ValueError, match="positions"):
        dn.deinfer_axis_positions(i(4, 4), i(3), i(3), i(2), 8, positions=i(2, 8))
    x, f = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(16, dtype=torch.float64)
    w = torch.zeros(32, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="q_weight"):
        dn.deinfer_norm_rope_store(x, x, None, i(4), f, 2, 2, 32, q_weight=w.float())
    with pytest.raises(ValueError, match="k_weight"):
        dn.deinfer_norm_rope_store(x, x, None, i(4), f, 2, 2, 32, k_weight=w[:30])
    with pytest.raises(ValueError, match="axis_of"):
        dn.deinfer_norm_rope_store(x, x, None, i(3, 4), f, 2, 2, 32)
    with pytest.raises(ValueError, match="axis_of"):
        dn.deinfer_norm_rope_store(x, x, None, i(3, 4), f, 2, 2, 32, axis_of=torch.zeros(15, dtype=torch.uint8))
    with pytest.raises(ValueError, match="positions"):
        dn.deinfer_norm_rope_store(x, x, None, i(3, 3), f, 2, 2, 32, axis_of=torch.zeros(16, dtype=torch.uint8))
    with pytest.raises(ValueError, match="pools"):
        dn.deinfer_norm_rope_store(x, x, x, i(4), f, 2, 2, 32, slots=i(4), q_out=x)
    with pytest.raises(ValueError, match="current device"):
        dn.deinfer_norm_rope_store(x, x, x, i(4), f, 2, 2, 32, q_weight=w)

    class NoWorkspace:
        buf, nbytes = torch.zeros(256, dtype=torch.uint8), 256

    with pytest.raises(ValueError, match="share a dtype"):
        dn.deinfer_prompt_attention(x, x.float(), x, i(3), NoWorkspace, 2, 2)
    with pytest.raises(ValueError, match="key rows"):
        dn.deinfer_prompt_attention(x, x, x[:3], i(3), NoWorkspace, 2, 2)
    with pytest.raises(ValueError, match="k_start"):
        dn.deinfer_prompt_attention(x, x, x, i(3), NoWorkspace, 2, 2, k_start=i(2))
    with pytest.raises(ValueError, match="current device"):
        dn.deinfer_prompt_attention(x, x, x, i(3), NoWorkspace, 2, 2)
