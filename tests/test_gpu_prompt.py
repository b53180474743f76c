"""The calls between the projections of a prompt on the GPU through the C ABI, each against the 64-bit oracle: positions
exactly, norms with rotation and attention within what their roundings can make.

Tolerances.  h = half a step of the output type relative to the value (bf16 2^-8, fp16 2^-11, fp32 2^-24).
  norms      the factor 1 / sqrt(mean + eps): a sum of D squares in fp32, D 2^-24 at most, halved by the root, and a handful of
             roundings of 2^-24 each: 1e-6 + D 2^-25; the rotation 5e-7 (as in test_gpu_cache_step.py); both times |a| + |b| of the pair; and h |y|
             for the output's rounding (fp16: 2^-25 for its small numbers).
  attention  as in test_gpu_cache_step.py: with A = sum_j p_j |v_j|: h A for the probabilities, h |o| for the output, 4e-4 A for scores in
             fp32; fp16 probabilities that are small numbers n 2^-25 max |v|."""
import numpy as np
import pytest

from oracle import prompt as op
from test_gpu_cache_step import HALF, dn, host, ints, kind_of, normal, wide  # noqa: F401

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ positions of several axes
def text(n):
    return [n, 0, 0, 0]


SEGMENTS = {
    # segments of every request, tokens cached (None: no list), new rows
    "one_token": ([[text(5)]], [2], [1]),
    "image": ([[text(3), [1, 4, 6, 1], text(2)]], None, [40]),
    "video": ([[[5, 2, 3, 2], text(4), [3, 7, 1, 0]], [text(1)], [[2, 1, 9, 100]]], [0, 0, 3], [70, 9, 30]),
    "decode": ([[text(9), [2, 4, 4, 3], text(2)]] * 4, [0, 20, 43, 60], [1, 1, 1, 1]),
    "nothing": ([[], [text(0), text(-4)], [[0, 3, 3, 1], [-2, 5, 5, 1], [4, -1, 5, 1], [2, 2, 2, -7]]], [5, 0, 1], [3, 4, 30]),
    "no_rows": ([[text(3)], [text(3)], [text(3)]], [0, 1, -5], [0, 2, 0]),
    "many_segments": ([[[1 + i % 3, i % 5, i % 4, i % 6] for i in range(700)], [text(1)] * 256, [text(2)] * 257], [100, 0, 0], [3000, 300, 600]),
    "far": ([[text(2 ** 31 - 1), text(2 ** 31 - 1)], [[2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1], text(9)], [text(7), [2, 65536, 65536, 9]]],
            [2 ** 31 - 4, 2 ** 31 - 5, 2 ** 31 - 100], [9, 5, 20]),
    "steps": ([[text(2), [4, 2, 2, 2 ** 30], text(5)]], [0], [30]),
}


def lists(of):
    return [seg for one in of for seg in one], np.concatenate([[0], np.cumsum([len(one) for one in of])])


@pytest.mark.parametrize("name", SEGMENTS)
@pytest.mark.parametrize("extra", [0, 5])
def test_axis_positions(dn, name, extra):
    import torch
    of, cached, new = SEGMENTS[name]
    segments, start = lists(of)
    rows = np.concatenate([[0], np.cumsum(new)])
    T = int(rows[-1]) + extra
    seg = ints(segments).reshape(-1, 4)
    out = torch.full((3, T + extra), -9, dtype=torch.int32, device="cuda")
    got = dn.deinfer_axis_positions(seg, ints(start), ints(rows), None if cached is None else ints(cached), T, positions=out[:, :T])
    want = op.axis_positions(segments, start, rows, cached, T, np.full((3, T), -9))
    assert np.array_equal(host(got), want)
    assert bool((out[:, T:] == -9).all())


def test_axis_positions_of_many_requests_and_lists_that_do_not_fit(dn):
    import torch
    rng = np.random.default_rng(4)
    of = [[[int(x) for x in rng.integers(-1, 6, 4)] for _ in range(rng.integers(0, 9))] for _ in range(1500)]
    segments, start = lists(of)
    new, cached = rng.integers(0, 12, 1500), rng.integers(-1, 90, 1500)
    rows = np.concatenate([[0], np.cumsum(new)])
    T = int(rows[-1]) - 40                                           # the last requests' rows are not there
    rows, start = rows.copy(), start.copy()
    rows[0], start[0] = -7, -3                                       # (from 0 on)
    start[-1] += 50                                                  # more segments than there are
    got = dn.deinfer_axis_positions(ints(segments), ints(start), ints(rows), ints(cached), T, positions=torch.full((3, T), 1, dtype=torch.int32, device="cuda"))
    assert np.array_equal(host(got), op.axis_positions(segments, start, rows, cached, T, np.ones((3, T))))


def test_axis_positions_of_requests_that_end_far_ahead_of_their_start(dn):
    """Ends of -2^31 are ends ahead of the start, whatever the start is."""
    import torch
    rows, T, low = [3, -2 ** 31, 2, 9], 12, -2 ** 31
    segments = [[5, 0, 0, 0], [1, 2, 2, 1]]
    for start in ([0, 1, 2, 2], [1, low, 0, 2]):
        got = dn.deinfer_axis_positions(ints(segments), ints(start), ints(rows), None, T, positions=torch.full((3, T), -4, dtype=torch.int32, device="cuda"))
        assert np.array_equal(host(got), op.axis_positions(segments, start, rows, None, T, np.full((3, T), -4)))


def test_axis_positions_of_long_prompts(dn):
    of = [[text(70000), [40, 60, 50, 2], text(100)], [[9, 30, 30, 1]]]
    segments, start = lists(of)
    rows = np.array([0, 190000, 190100])
    got = host(dn.deinfer_axis_positions(ints(segments), ints(start), ints(rows), None, 190100))
    at = np.concatenate([np.arange(0, 190000, 997), np.arange(69990, 70010), np.arange(189990, 190100)])
    want = op.axis_positions(segments, start, np.array([0, 190000, 190100]), None, 190100, np.zeros((3, 190100)))
    assert np.array_equal(got, want) and len(at)


# ------------------------------------------------------------------ norms with rotation
NORMS = [
    # type, rows, q heads, kv heads, head dim, rotated, interleaved, pairs of each axis, turns, pitch beyond the row
    ("bf16", 1, 1, 1, 8, 8, False, [4], False, 0),
    ("bf16", 33, 8, 2, 128, 128, False, [64], False, 0),
    ("f16", 9, 4, 4, 128, 64, True, [32], False, 0),
    ("f32", 17, 3, 1, 64, 64, False, [12, 10, 10], True, 0),
    ("f32", 5, 2, 2, 64, 32, True, [8, 8], False, 0),
    ("bf16", 21, 5, 1, 80, 80, False, [20, 20], False, 0),
    ("f16", 11, 4, 2, 72, 72, False, [9, 9, 9, 9], True, 4),
    ("bf16", 11, 4, 2, 72, 36, False, [18], False, 2),
    ("bf16", 7, 2, 2, 96, 48, True, [8, 8, 8], False, 1),            # rows at odd elements
    ("f32", 7, 2, 1, 20, 12, False, [3, 3], True, 3),
    ("bf16", 6, 3, 1, 7, 4, False, [2], False, 0),                   # an odd head
    ("f16", 6, 3, 1, 256, 256, True, [32, 48, 48], True, 0),
    ("bf16", 3, 2, 1, 1000, 500, False, [125, 125], False, 0),       # more pieces than lanes
    ("f32", 3, 2, 1, 2048, 1024, False, [512], False, 1),
    ("bf16", 4, 2, 2, 2048, 1024, True, [500, 12], True, 0),
    ("f16", 300, 40, 8, 64, 64, False, [8, 12, 12], True, 8),
    ("bf16", 4, 6, 2, 64, 0, False, [], False, 0),                   # norms alone
]


def norm_case(dtype, rows, hq, hk, D, extra, seed=0):
    import torch
    def rows_of(i, heads, scale):
        x = torch.full((rows, heads * D + extra), float("nan"), device="cuda")
        x[:, :heads * D] = torch.tensor(normal(seed * 10 + i, rows, heads * D) * scale, device="cuda")
        return x.to(kind_of(dtype))[:, :heads * D]
    weights = [torch.tensor(1.0 + 0.3 * normal(seed * 10 + 5 + i, D), device="cuda").to(kind_of(dtype)) for i in range(2)]
    return rows_of(1, hq, 3.0), rows_of(2, hk, 0.2), rows_of(3, hk, 1.0), weights


def angles_of(positions, axis_of, freqs):
    return np.asarray(positions, dtype=np.float64)[np.asarray(axis_of, dtype=int)].T * freqs if len(freqs) else np.zeros((np.asarray(positions).shape[1], 0))


def check_norm(got, x, heads, weight, eps, angles, magnitude, inter, dtype):
    ref = op.norm_rope(x, heads, weight, eps, angles, magnitude, inter)
    T, D, half = x.shape[0], x.shape[1] // heads, angles.shape[1]
    size = np.abs(op.norm_rope(x, heads, weight, eps, np.zeros((T, 0)), 1.0, inter)).reshape(T, heads, D)
    first = np.arange(half) * (2 if inter else 1)
    second = first + (1 if inter else half)
    pair = abs(magnitude) * (size[:, :, first] + size[:, :, second])
    size[:, :, first] = size[:, :, second] = pair
    tol = HALF[dtype] * np.abs(ref) * 1.001 + (1.5e-6 + D * 2.0 ** -25) * size.reshape(T, heads * D) + (2.0 ** -25 if dtype == "f16" else 0.0)
    assert np.all(np.abs(got - ref) <= tol), float(np.max(np.abs(got - ref) / np.maximum(tol, 1e-300)))


@pytest.mark.parametrize("dtype,rows,hq,hk,D,rot,inter,pairs,turns,extra", NORMS)
def test_norm_rope_store(dn, dtype, rows, hq, hk, D, rot, inter, pairs, turns, extra):
    import torch
    q, k, v, (qw, kw) = norm_case(dtype, rows, hq, hk, D, extra, seed=D)
    rng = np.random.default_rng(D)
    axes = max(len(pairs), 1)
    freqs = 10000.0 ** (-2.0 * np.arange(rot // 2) / max(rot, 1))
    axis_of = dn.deinfer_rope_axes(rot, pairs, turns) if rot else np.zeros(0, dtype=np.uint8)
    pos = rng.integers(-5, 1 << 20, (axes, rows))
    n_slots = rows + 4
    slots = rng.permutation(n_slots)[:rows]
    if rows > 1:
        slots[rows // 2] = -1 if rows % 2 else n_slots               # a row that is not in use
    pools = [torch.full((n_slots, hk * D + extra), float("nan"), dtype=q.dtype, device="cuda") for _ in range(2)]
    q_out = torch.full((rows, hq * D + extra), float("nan"), dtype=q.dtype, device="cuda")
    at = torch.full((axes, rows + 3), -7, dtype=torch.int32, device="cuda")
    at[:, :rows] = ints(pos)
    magnitude, eps = 1.25, 1e-5
    dn.deinfer_norm_rope_store(q, k, v, at[:, :rows], torch.tensor(freqs, device="cuda") if rot else None, hq, hk, D, q_weight=qw, k_weight=kw, eps=eps,
                               axis_of=torch.tensor(axis_of, device="cuda") if axes > 1 else None, interleaved=inter, magnitude=magnitude, slots=ints(slots),
                               q_out=q_out[:, :hq * D], k_out=pools[0][:, :hk * D], v_out=pools[1][:, :hk * D])
    live = [t for t in range(rows) if 0 <= slots[t] < n_slots]
    dead = [t for t in range(rows) if t not in live]
    angles = angles_of(pos, axis_of, freqs)[live]
    e = float(np.float32(eps))
    check_norm(wide(q_out)[live][:, :hq * D], wide(q)[live], hq, wide(qw), e, angles, magnitude, inter, dtype)
    check_norm(wide(pools[0])[slots[live]][:, :hk * D], wide(k)[live], hk, wide(kw), e, angles, magnitude, inter, dtype)
    assert np.array_equal(wide(pools[1])[slots[live], :hk * D], wide(v)[live])
    assert np.all(np.isnan(wide(q_out)[dead])) and np.all(np.isnan(wide(q_out)[:, hq * D:])) and np.all(np.isnan(wide(pools[0])[:, hk * D:]))
    unused = [r for r in range(n_slots) if r not in set(slots[live])]
    assert np.all(np.isnan(wide(pools[0])[unused])) and np.all(np.isnan(wide(pools[1])[unused]))


@pytest.mark.parametrize("dtype,D,rot,inter", [("bf16", 128, 128, False), ("f16", 64, 32, True), ("f32", 20, 12, False), ("bf16", 1000, 1000, False)])
def test_norm_in_place_and_alone(dn, dtype, D, rot, inter):
    """In place without slots, q alone, k alone: the same bits as apart."""
    import torch
    q, k, v, (qw, kw) = norm_case(dtype, 11, 4, 2, D, 0, seed=3)
    f, pos = torch.tensor(500000.0 ** (-2.0 * np.arange(rot // 2) / rot), device="cuda"), ints(np.arange(11) * 37)
    apart = [torch.empty_like(t) for t in (q, k, v)]
    dn.deinfer_norm_rope_store(q, k, v, pos, f, 4, 2, D, q_weight=qw, k_weight=kw, interleaved=inter, q_out=apart[0], k_out=apart[1], v_out=apart[2])
    a, b = q.clone(), k.clone()
    dn.deinfer_norm_rope_store(a, b, None, pos, f, 4, 2, D, q_weight=qw, k_weight=kw, interleaved=inter)
    assert torch.equal(a, apart[0]) and torch.equal(b, apart[1]) and torch.equal(v, apart[2])
    c, d = q.clone(), k.clone()
    dn.deinfer_norm_rope_store(c, None, None, pos[None, :], f, 4, 0, D, q_weight=qw, interleaved=inter)
    dn.deinfer_norm_rope_store(None, d, None, pos, f, 0, 2, D, k_weight=kw, interleaved=inter)
    assert torch.equal(c, a) and torch.equal(d, b)


@pytest.mark.parametrize("dtype,D,rot,inter,extra", [("bf16", 128, 128, False, 0), ("f16", 64, 32, True, 0), ("f32", 20, 12, False, 1), ("bf16", 80, 40, False, 0), ("bf16", 96, 96, True, 1)])
def test_without_weights_it_is_the_rotary_store(dn, dtype, D, rot, inter, extra):
    import torch
    q, k, v, _ = norm_case(dtype, 13, 4, 2, D, extra, seed=4)
    f, pos = torch.tensor(10000.0 ** (-2.0 * np.arange(rot // 2) / rot), device="cuda"), ints(np.arange(13) * 1001)
    slots = ints(np.random.default_rng(1).permutation(20)[:13])
    found = []
    for call in (dn.deinfer_rope_store, dn.deinfer_norm_rope_store):
        out = [torch.zeros_like(q), torch.zeros(20, 2 * D, dtype=q.dtype, device="cuda"), torch.zeros(20, 2 * D, dtype=q.dtype, device="cuda")]
        call(q, k, v, pos, f, 4, 2, D, interleaved=inter, magnitude=1.5, slots=slots, q_out=out[0], k_out=out[1], v_out=out[2])
        found.append(out)
    # the same angles, products and roundings (which products are fused with their sum is the compiler's)
    for a, b in zip(*found):
        assert float((a != b).float().mean()) < 2e-2 or dtype == "f32"
        assert float((a.double() - b.double()).abs().max()) <= 2 * HALF[dtype] * float(a.abs().max()) + 1e-6
    assert torch.equal(found[0][2], found[1][2])


@pytest.mark.parametrize("dtype,scale,eps", [("bf16", 1e25, 1e-6), ("bf16", 1e38, 0.0), ("f32", 1e30, 1e-6), ("f32", 1e-30, 0.0), ("f32", 1e-20, 1e-6), ("bf16", 1e-25, 0.0), ("bf16", 0.0, 1e-6),
                                             ("f16", 6e4, 1e-6), ("f16", 1e-7, 0.0)])
def test_norms_of_very_large_and_small_elements(dn, dtype, scale, eps):
    import torch
    T, H, D = 6, 3, 64
    x = torch.tensor(np.clip(normal(9, T, H * D), -2.0, 2.0) * 0.5 * scale, device="cuda").to(kind_of(dtype))
    x[2] = torch.tensor(normal(10, H * D), device="cuda").to(x.dtype)               # an ordinary row beside them
    w = torch.ones(D, dtype=x.dtype, device="cuda")
    y = torch.empty_like(x)
    f, pos = torch.tensor(10000.0 ** (-2.0 * np.arange(32) / D), device="cuda"), np.arange(T)
    dn.deinfer_norm_rope_store(x, None, None, ints(pos), f, H, 0, D, q_weight=w, eps=eps, q_out=y)
    check_norm(wide(y), wide(x), H, wide(w), float(np.float32(eps)), angles_of(pos[None], np.zeros(32), host(f)), 1.0, False, dtype)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_elements_that_are_no_numbers_stay_in_their_head(dn, bad):
    import torch
    q, _, _, (qw, _) = norm_case("bf16", 5, 6, 1, 80, 0, seed=6)
    f, pos = torch.tensor(10000.0 ** (-2.0 * np.arange(40) / 80), device="cuda"), ints(np.arange(5))
    call = lambda x: dn.deinfer_norm_rope_store(x.clone(), None, None, pos, f, 6, 0, 80, q_weight=qw)[0].view(5, 6, 80)
    clean = call(q)
    q[2, 3 * 80 + 7] = bad
    got = call(q)
    same = torch.ones(5, 6, dtype=torch.bool, device="cuda")
    same[2, 3] = False
    assert torch.equal(got[same], clean[same])
    # infinity: its own pair is no number, the rest of the head is zero (x / infinity)
    hit = torch.isnan(got[2, 3])
    assert bool(hit.all()) if bad != bad else hit.nonzero().flatten().tolist() == [7, 47] and bool((got[2, 3][~hit] == 0).all())


# ------------------------------------------------------------------ attention
def packed(seed, lengths, heads, D, dtype, extra_rows=0, extra_pitch=0, scale=1.0):
    """Rows of the sequences; padding rows and the columns behind a row are NaN."""
    import torch
    n = int(sum(lengths))
    x = torch.full((n + extra_rows, heads * D + extra_pitch), float("nan"), dtype=kind_of(dtype), device="cuda")
    x[:n, :heads * D] = torch.tensor(normal(seed, n, heads * D) * scale, device="cuda").to(x.dtype)
    return x[:, :heads * D]


def check_prompt(dn, q, k, v, q_start, k_start, hq, hk, left, right, dtype, scale=None, out=None, ws=None):
    import torch
    T, D, n = q.shape[0], q.shape[1] // hq, len(q_start) - 1
    ws = ws or dn.Workspace(dn.deinfer_prompt_attention_workspace_bytes(T, n, hq, hk, D))
    if out is None:
        out = torch.full((T, hq * D), 3.0, dtype=q.dtype, device="cuda")
    call = lambda: dn.deinfer_prompt_attention(q, k, v, ints(q_start), ws, hq, hk, k_start=None if k_start is None else ints(k_start), scale=scale, left=left, right=right, out=out)
    call()
    first = out.clone()
    call()
    assert torch.equal(first, out)                                  # whatever was timed how
    sc = D ** -0.5 if scale is None else scale
    qh, kh, vh = np.nan_to_num(wide(q)), np.nan_to_num(wide(k)), np.nan_to_num(wide(v))
    ref = op.attention(qh, kh, vh, q_start, k_start, hq, hk, left, right, sc, np.full((T, hq * D), 3.0))
    size = op.attention(qh, kh, np.abs(vh), q_start, k_start, hq, hk, left, right, sc, np.zeros((T, hq * D)))
    got = wide(out)
    longest = int(np.max(np.diff(q_start if k_start is None else k_start)))
    tol = HALF[dtype] * (np.abs(ref) + size) * 1.01 + 4e-4 * size + (longest * 2.0 ** -25 * np.max(np.abs(vh)) if dtype == "f16" and vh.size else 0.0)
    rows = int(q_start[-1])
    assert np.all(np.isfinite(got))
    assert np.all(np.abs(got - ref)[:rows] <= tol[:rows]), float(np.max((np.abs(got - ref) / np.maximum(tol, 1e-30))[:rows]))
    assert np.all(got[rows:] == 3.0)                                # padding rows: as they were
    return got


def starts(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(int)


ATTEND = [
    # rows, keys (None: the rows'), q heads, kv heads, head dim, type, left, right, padding rows
    ([1], None, 1, 1, 64, "bf16", -1, 0, 0),                         # one token that sees itself
    ([1] * 6, [1, 15, 33, 128, 129, 300], 8, 1, 128, "bf16", -1, 0, 2),
    ([1] * 4, [0, 700, 5, 64], 7, 1, 80, "f16", -1, 0, 1),           # a sequence without keys
    ([1, 1], [90, 41], 4, 4, 8, "bf16", -1, 0, 0),
    ([1, 1, 1], [300, 20, 4], 5, 1, 256, "bf16", 16, 0, 0),          # windows that leave out most
    ([1, 2], [5000, 3000], 8, 1, 128, "f16", -1, 0, 0),              # keys over many workgroups
    ([3, 0, 2], [70, 9, 0], 6, 2, 72, "bf16", -1, -1, 3),
    ([5, 9, 1], None, 8, 2, 64, "bf16", -1, 0, 3),
    ([33, 20], None, 8, 2, 128, "f16", -1, 0, 0),
    ([100, 31, 64, 0, 7], None, 4, 4, 128, "bf16", -1, 0, 5),
    ([17], [200], 3, 1, 96, "bf16", -1, 0, 0),
    ([64, 130], None, 4, 4, 64, "f16", -1, 0, 0),
    ([300], [333], 6, 2, 128, "bf16", -1, 0, 1),                     # a chunk behind other keys
    ([257], None, 2, 1, 128, "bf16", -1, 0, 0),
    ([150, 80], None, 4, 2, 80, "f16", -1, 0, 0),
    ([150, 80], None, 4, 2, 72, "bf16", -1, 0, 2),
    ([150, 80], None, 4, 2, 96, "bf16", -1, 0, 0),
    ([150, 80], None, 4, 2, 88, "f16", 40, 9, 0),
    ([150, 80], None, 4, 2, 120, "bf16", -1, 0, 0),
    ([150, 80], None, 4, 2, 40, "bf16", -1, 0, 0),
    ([150, 80], None, 4, 2, 256, "bf16", -1, 0, 0),
    ([60, 200], None, 2, 2, 200, "f16", -1, 0, 0),
    ([60, 200], None, 2, 2, 256, "f16", 50, 0, 0),
    ([196, 196, 49], None, 3, 3, 64, "bf16", -1, -1, 0),             # images
    ([196, 400], None, 3, 3, 80, "f16", -1, -1, 2),
    ([400, 90], None, 2, 1, 128, "bf16", 63, 0, 0),                  # windows
    ([400, 90], None, 2, 2, 128, "f16", 0, 0, 0),                    # each row itself alone
    ([400, 90], None, 2, 1, 64, "bf16", 20, 33, 0),
    ([300, 90], None, 2, 1, 128, "bf16", 0, -1, 0),                  # what follows
    ([300, 100, 40], [200, 0, 39], 4, 2, 128, "bf16", -1, 0, 1),     # rows ahead of the first key see nothing
    ([300, 100, 40], [200, 0, 39], 4, 2, 256, "f16", 30, 0, 1),
    ([90, 10], [20, 3], 2, 1, 64, "bf16", -1, 0, 0),
    ([20, 3], [5, 2], 1, 1, 128, "f16", 2, 0, 0),
    ([40, 25], None, 40, 1, 64, "bf16", -1, 0, 0),                   # a tile of few tokens
    ([9, 2], None, 150, 1, 64, "bf16", -1, 0, 0),                    # more query heads than rows of a tile
    ([3, 2], [40, 2], 300, 1, 128, "f16", -1, 0, 0),
    ([1, 1], [40, 77], 600, 2, 40, "bf16", -1, 0, 0),
    ([700], None, 1, 1, 128, "bf16", -1, 0, 0),
    ([64, 0, 0, 0, 900], None, 2, 1, 64, "f16", -1, 0, 4),
    ([20] * 30, [400] * 30, 8, 4, 128, "bf16", 100, 0, 0),
]


@pytest.mark.parametrize("rows,keys,hq,hk,D,dtype,left,right,extra", ATTEND)
def test_prompt_attention(dn, rows, keys, hq, hk, D, dtype, left, right, extra):
    seed = D + len(rows) + hq
    q = packed(seed, rows, hq, D, dtype, extra)
    k, v = (packed(seed + 1 + i, rows if keys is None else keys, hk, D, dtype, extra) for i in range(2))
    check_prompt(dn, q, k, v, starts(rows), None if keys is None else starts(keys), hq, hk, left, right, dtype)


def test_prompt_attention_of_many_ragged_sequences(dn):
    """More sequences than threads of a workgroup, and lengths that differ a hundredfold."""
    rng = np.random.default_rng(1)
    for hq, D, most in ((2, 64, 30), (4, 64, 3)):
        keys = np.exp(rng.uniform(0, 5, 700)).astype(int)
        rows = rng.integers(0, most, 700)
        rows[:3] = [70, 0, 150]
        q, k, v = packed(1, rows, hq, D, "bf16", 3), packed(2, keys, 1, D, "bf16", 1), packed(3, keys, 1, D, "bf16", 1)
        check_prompt(dn, q, k, v, starts(rows), starts(keys), hq, 1, -1, 0, "bf16")


@pytest.mark.parametrize("n_seqs", [1, 2, 63, 64, 65, 128, 129])
@pytest.mark.parametrize("most,hq", [(2, 4), (40, 4), (200, 2)])
def test_prompt_attention_of_as_many_sequences_as_a_wavefront_has_lanes(dn, n_seqs, most, hq):
    """Sequences without rows, without keys or with neither among them, also the first and the last."""
    rng = np.random.default_rng(n_seqs)
    rows, keys = rng.integers(0, most, n_seqs), rng.integers(0, 300, n_seqs)
    rows[0], rows[n_seqs // 2] = 0, most
    keys[n_seqs // 3] = 0
    q, k, v = packed(4, rows, 2 * hq, 64, "f16", 2), packed(5, keys, 2, 64, "f16", 5), packed(6, keys, 2, 64, "f16", 5)
    check_prompt(dn, q, k, v, starts(rows), starts(keys), 2 * hq, 2, -1, 0, "f16")


@pytest.mark.parametrize("n", [70, 20000])
def test_pairs_of_tiles_beyond_a_wavefront(dn, n):
    """A sequence with more pairs of tiles than a wavefront has lanes: every row with its own key alone, and with a few around it."""
    import torch
    hq, D = 16, 64
    rows = [n, 3, n // 3]
    q, k, v = (packed(s, rows, h, D, "bf16") for s, h in ((7, hq), (8, 1), (9, 1)))
    ws = dn.Workspace(dn.deinfer_prompt_attention_workspace_bytes(sum(rows), 3, hq, 1, D))
    got = dn.deinfer_prompt_attention(q, k, v, ints(starts(rows)), ws, hq, 1, left=0, right=0)
    assert torch.equal(got.view(-1, hq, D), v.view(-1, 1, D).expand(-1, hq, D))          # p = 1: the value itself
    got = dn.deinfer_prompt_attention(q, k, v, ints(starts(rows)), ws, hq, 1, left=5, right=2).view(-1, hq, D).double()
    of = torch.repeat_interleave(torch.arange(3, device="cuda"), torch.tensor(rows, device="cuda"))
    at = torch.arange(sum(rows), device="cuda")[:, None] + torch.arange(-5, 3, device="cuda")          # the keys of every row
    held = at.clamp(0, sum(rows) - 1)
    seen = (at == held) & (of[held] == of[:, None])
    x = (q.double().view(-1, 1, hq, D) * k.double()[held][:, :, None]).sum(3) * D ** -0.5
    prob = torch.softmax(x.masked_fill(~seen[:, :, None], -float("inf")), 1)[:, :, :, None]
    vs = v.double()[held][:, :, None]
    want, size = (prob * vs).sum(1), (prob * vs.abs()).sum(1)
    assert bool(((got - want).abs() <= HALF["bf16"] * (want.abs() + size) * 1.01 + 4e-4 * size).all())


@pytest.mark.parametrize("D,dtype", [(64, "bf16"), (80, "f16"), (96, "bf16"), (128, "bf16"), (128, "f16"), (200, "f16"), (256, "bf16")])
@pytest.mark.parametrize("most,left,right", [(300, -1, 0), (300, 70, 0), (700, -1, -1), (90, -1, 0)])
def test_prompt_attention_with_many_tiles_for_every_workgroup(dn, D, dtype, most, left, right):
    """Odd lengths, a head for every query head: tiles that end inside a stage follow one another in a workgroup."""
    rng = np.random.default_rng(D + most)
    rows = rng.integers(most // 2, most, 9000 // most)
    rows[3] = 0
    keys = rows + rng.integers(-20, 50, len(rows)).clip(-rows, None)
    hq = 2048 // D
    q, k, v = packed(1, rows, hq, D, dtype, 3), packed(2, keys, hq, D, dtype, 1), packed(3, keys, hq, D, dtype, 1)
    check_prompt(dn, q, k, v, starts(rows), starts(keys), hq, hq, left, right, dtype)


@pytest.mark.parametrize("rows", [[3, 1, 2], [60, 100, 9], [300, 20, 200]])
def test_prompt_attention_strides_and_large_scores(dn, rows):
    """q, k and v side by side in one wide row, out in a wider row; scores up to about 100."""
    import torch
    hq, hk, D = 4, 2, 64
    n = sum(rows)
    wide_row = packed(7, rows, hq + 2 * hk, D, "bf16", 2, 8, scale=4.0)
    q, k, v = wide_row[:, :hq * D], wide_row[:, hq * D:(hq + hk) * D], wide_row[:, (hq + hk) * D:]
    out = torch.full((n + 2, hq * D + 16), 3.0, dtype=torch.bfloat16, device="cuda")
    check_prompt(dn, q, k, v, starts(rows), None, hq, hk, -1, 0, "bf16", scale=0.4, out=out[:, :hq * D])
    assert bool((out[:, hq * D:] == 3.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n,D", [(3, 128), (40, 128), (30, 64), (40, 256), (200, 128)])
def test_prompt_scores_that_rise_along_the_keys(dn, dtype, n, D):
    """Every later key scores higher (or lower), by up to 60 in all: each stage wants a new reference, and early keys come to weigh nothing."""
    import torch
    keys, hq, hk = 700, 4, 1
    k, v = packed(31, [keys], hk, D, dtype), packed(32, [keys], hk, D, dtype)
    rise = torch.arange(keys, device="cuda", dtype=torch.float32)[:, None] / keys
    k = (0.1 * k.float() + rise * 8.0 / D ** 0.5).to(k.dtype)
    q = (0.1 * packed(33, [n], hq, D, dtype).float() + 8.0).to(k.dtype)
    for x in (q, -q):
        check_prompt(dn, x, k, v, starts([n]), starts([keys]), hq, hk, -1, 0, dtype, scale=60.0 / (64.0 * D ** 0.5))


@pytest.mark.parametrize("dtype,D,n", [("bf16", 128, 2), ("f16", 128, 2), ("bf16", 128, 60), ("f16", 64, 60), ("bf16", 64, 300), ("f16", 256, 60)])
@pytest.mark.parametrize("size", [2.0 ** 25, 2.0 ** 40, 2.0 ** 100])
def test_prompt_scores_of_any_size(dn, dtype, D, n, size):
    """Scores of +-size times whole numbers: a row's largest ones share the weight alike, whatever their size."""
    import torch
    keys, hq = 200, 2
    rng = np.random.default_rng(D + n)
    level = rng.integers(-3, 4, keys)
    k = torch.zeros(keys, D, dtype=kind_of(dtype), device="cuda")
    k[:, 0] = torch.tensor(level, device="cuda").to(k.dtype)
    v = packed(5, [keys], 1, D, dtype)
    q = torch.zeros(n, hq * D, dtype=k.dtype, device="cuda")
    q[:, 0], q[:, D] = 1.0, -1.0
    ws = dn.Workspace(dn.deinfer_prompt_attention_workspace_bytes(n, 1, hq, 1, D))
    got = wide(dn.deinfer_prompt_attention(q, k, v, ints([0, n]), ws, hq, 1, k_start=ints([0, keys]), scale=size, right=-1)).reshape(n, hq, D)
    for h, best in ((0, level.max()), (1, level.min())):
        want = wide(v)[level == best].mean(0)
        # equal probabilities: exact in the type; the sum in fp32, and the output's rounding
        assert np.all(np.abs(got[:, h] - want) <= HALF[dtype] * np.abs(want) * 1.01 + 1e-6)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("n,hq,D", [(6, 2, 128), (40, 4, 128), (150, 2, 64), (300, 2, 128), (60, 2, 256), (90, 2, 80)])
def test_keys_and_values_that_are_no_numbers_stay_with_the_rows_that_see_them(dn, value, n, hq, D):
    """Such a value, then such a key, in the middle of a prompt: the rows ahead of it are as without it."""
    import torch
    bad = n // 2
    q, k, v = packed(41, [n, 3], hq, D, "bf16"), packed(42, [n, 3], 1, D, "bf16"), packed(43, [n, 3], 1, D, "bf16")
    ws = dn.Workspace(dn.deinfer_prompt_attention_workspace_bytes(n + 3, 2, hq, 1, D))
    call = lambda: wide(dn.deinfer_prompt_attention(q, k, v, ints([0, n, n + 3]), ws, hq, 1))
    clean = call()
    v[bad, 5] = value
    got = call()
    # (these rows' sums may be formed in another order beside such a value: fp32 sums, and an output step)
    other = np.r_[np.arange(bad), np.arange(n, n + 3)]
    assert np.max(np.abs(got[other] - clean[other])) <= 2 ** -7 * np.max(np.abs(clean))
    hit = got[bad:n].reshape(n - bad, hq, D)
    assert not np.any(np.isfinite(hit[:, :, 5])) and np.all(np.isfinite(np.delete(hit, 5, axis=2)))
    if np.isinf(value):
        assert np.all(hit[:, :, 5] == value)
    k[bad, 7] = float("nan")
    got = call()
    assert np.max(np.abs(got[other] - clean[other])) <= 2 ** -7 * np.max(np.abs(clean))
    assert np.all(np.isnan(got[bad:n]))


@pytest.mark.parametrize("n", [2, 40, 200])
def test_a_query_that_is_no_number_leaves_the_other_rows(dn, n):
    import torch
    q, k, v = packed(44, [n], 4, 128, "bf16"), packed(45, [n], 2, 128, "bf16"), packed(46, [n], 2, 128, "bf16")
    ws = dn.Workspace(dn.deinfer_prompt_attention_workspace_bytes(n, 1, 4, 2, 128))
    call = lambda: dn.deinfer_prompt_attention(q, k, v, ints([0, n]), ws, 4, 2).view(n, 4, 128)
    clean = call()
    q[n // 2, 128 + 3] = float("nan")
    got = call()
    same = torch.ones(n, 4, dtype=torch.bool, device="cuda")
    same[n // 2, 1] = False
    assert bool(torch.isnan(got[n // 2, 1]).all())
    assert float((got[same].double() - clean[same].double()).abs().max()) <= 2 ** -7 * float(clean.abs().max())


@pytest.mark.parametrize("hq,T", [(2, 4), (8, 12), (4, 400)])
def test_lists_that_do_not_fit_are_cut(dn, hq, T):
    """Starts outside the tensors, and ends before starts: what is left of the sequences, and the other rows as they were."""
    import torch
    D = 64
    q, k, v = packed(51, [T], hq, D, "bf16"), packed(52, [T], 1, D, "bf16"), packed(53, [T], 1, D, "bf16")
    q_start, k_start = [-5, T // 2, T // 4, T + 100], [T // 3, T + 9, 2, 2 ** 31 - 1]
    ws = dn.Workspace(dn.deinfer_prompt_attention_workspace_bytes(T, 3, hq, 1, D))
    out = torch.full((T, hq * D), 3.0, dtype=q.dtype, device="cuda")
    dn.deinfer_prompt_attention(q, k, v, ints(q_start), ws, hq, 1, k_start=ints(k_start), right=-1, out=out)
    # (rows T / 4 .. T / 2 belong to two sequences: either's, or in between no matter)
    ref = op.attention(wide(q), wide(k), wide(v), q_start, k_start, hq, 1, -1, -1, D ** -0.5, np.full((T, hq * D), 3.0))
    got = wide(out)
    alone = np.r_[np.arange(T // 4), np.arange(T // 2, T)]
    assert np.max(np.abs(got - ref)[alone]) <= 3 * 2.0 ** -8 * np.max(np.abs(wide(v)))


@pytest.mark.parametrize("n", [1, 50, 200])
def test_prompt_offsets_past_32_bits(dn, n):
    """The same keys at the far end of 5 GB of rows and in tensors of their own: bit for bit the same."""
    import torch
    keys, hq, hk, D = 300, 16, 16, 128
    q, k, v = packed(61, [n], hq, D, "bf16"), packed(62, [keys], hk, D, "bf16"), packed(63, [keys], hk, D, "bf16")
    ws = dn.Workspace(dn.deinfer_prompt_attention_workspace_bytes(n, 1, hq, hk, D))
    want = dn.deinfer_prompt_attention(q, k, v, ints([0, n]), ws, hq, hk, k_start=ints([0, keys]))
    far = 5 * (1 << 30) // (hk * D * 2)
    big = torch.empty((2, far, hk * D), dtype=torch.bfloat16, device="cuda")
    big[0, far - keys:], big[1, far - keys:] = k, v
    got = dn.deinfer_prompt_attention(q, big[0], big[1], ints([0, n]), ws, hq, hk, k_start=ints([far - keys, far]))
    assert torch.equal(got, want)


# ------------------------------------------------------------------ together
def prompt_path(dn, s, rows):
    """The calls of one layer between its projections, for whatever lengths s holds."""
    dn.deinfer_axis_positions(s["segments"], s["segment_start"], s["row_start"], s["cached"], rows, positions=s["positions"])
    dn.deinfer_norm_rope_store(s["q"], s["k"], None, s["positions"], s["freqs"], s["hq"], s["hk"], s["D"], q_weight=s["qw"], k_weight=s["kw"], axis_of=s["axis_of"],
                               q_out=s["q_rot"], k_out=s["k_rot"])
    dn.deinfer_prompt_attention(s["q_rot"], s["k_rot"], s["v"], s["row_start"], s["ws"], s["hq"], s["hk"], out=s["out"])


def prompt_state(dn, rows, n_seqs, hq=8, hk=2, D=128, seed=70):
    import torch
    q, k, v, (qw, kw) = norm_case("bf16", rows, hq, hk, D, 0, seed=seed)
    pairs = [D // 8, D // 4 - D // 16, D // 4 - D // 16]
    return dict(hq=hq, hk=hk, D=D, q=q, k=k, v=v, qw=qw, kw=kw, q_rot=torch.zeros_like(q), k_rot=torch.zeros_like(k), out=torch.zeros_like(q),
                freqs=torch.tensor(10000.0 ** (-2.0 * np.arange(D // 2) / D), device="cuda"), axis_of=torch.tensor(dn.deinfer_rope_axes(D, pairs, True), device="cuda"),
                positions=torch.zeros(3, rows, dtype=torch.int32, device="cuda"), cached=ints([0] * n_seqs), row_start=ints([0] * (n_seqs + 1)),
                segments=ints([[0, 0, 0, 0]] * 12), segment_start=ints([0] * (n_seqs + 1)),
                ws=dn.Workspace(dn.deinfer_prompt_attention_workspace_bytes(rows, n_seqs, hq, hk, D)))


def set_lengths(s, of, new):
    import torch
    segments, start = lists(of)
    s["segments"][:len(segments)] = ints(segments)
    s["segment_start"].copy_(ints(start))
    s["row_start"].copy_(ints(starts(new)))


STEPS = [([[text(9), [1, 4, 5, 1], text(30)], [text(20)], [[3, 4, 4, 2], text(60)]], [59, 20, 108]),
         ([[text(1)], [text(150)], [[1, 6, 6, 1]]], [1, 150, 36]),
         ([[], [text(2)], [text(3), [2, 3, 3, 1]]], [0, 2, 21])]


def test_the_calls_together(dn):
    """Against the same path in 64 bits, rounded to bf16 where the calls hand over."""
    import torch
    rows = 190
    s = prompt_state(dn, rows, 3)
    for of, new in STEPS:
        set_lengths(s, of, new)
        s["out"].fill_(3.0)
        prompt_path(dn, s, rows)
        n = sum(new)
        segments, start = lists(of)
        pos = op.axis_positions(segments, start, starts(new), None, rows, host(s["positions"]))
        assert np.array_equal(host(s["positions"]), pos)
        angles = angles_of(pos, host(s["axis_of"]), host(s["freqs"]))
        for name, heads, weight in (("q", 8, "qw"), ("k", 2, "kw")):
            check_norm(wide(s[name + "_rot"]), wide(s[name]), heads, wide(s[weight]), float(np.float32(1e-6)), angles, 1.0, False, "bf16")
        ref = op.attention(wide(s["q_rot"]), wide(s["k_rot"]), wide(s["v"]), starts(new), None, 8, 2, -1, 0, 128 ** -0.5, np.full((rows, 1024), 3.0))
        assert np.max(np.abs(wide(s["out"]) - ref)) <= 3 * 2.0 ** -8 * np.max(np.abs(wide(s["v"])))
        assert np.all(wide(s["out"])[n:] == 3.0)


def test_one_graph_serves_steps_of_other_lengths(dn):
    import torch
    rows = 190
    s, eager = prompt_state(dn, rows, 3), prompt_state(dn, rows, 3)
    set_lengths(s, *STEPS[0])
    prompt_path(dn, s, rows)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        prompt_path(dn, s, rows)
    for turn in range(3):
        for of, new in STEPS:
            set_lengths(s, of, new)
            set_lengths(eager, of, new)
            for x in (s, eager):
                x["out"].fill_(float(turn))
            graph.replay()
            prompt_path(dn, eager, rows)
            torch.cuda.synchronize()
            for name in ("out", "q_rot", "k_rot"):
                n = sum(new)
                assert torch.equal(s[name][:n], eager[name][:n]), (turn, new, name)
            assert bool((s["out"][sum(new):] == float(turn)).all())


def test_two_graphs_over_one_workspace_and_another_stream(dn):
    import torch
    a, b = prompt_state(dn, 190, 3), prompt_state(dn, 400, 3, hq=4, hk=4, D=64, seed=71)
    nbytes = max(a["ws"].nbytes, b["ws"].nbytes)
    a["ws"] = b["ws"] = dn.Workspace(nbytes)
    set_lengths(a, *STEPS[0])
    set_lengths(b, *STEPS[1])
    want = []
    for s, rows in ((a, 190), (b, 400)):
        prompt_path(dn, s, rows)
        want.append(s["out"].clone())
    graphs = []
    for s, rows in ((a, 190), (b, 400)):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            prompt_path(dn, s, rows)
    for _ in range(3):
        for g, s, w in zip(graphs, (a, b), want):
            s["out"].zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(s["out"], w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    n = sum(STEPS[0][1])
    got = dn.deinfer_prompt_attention(a["q_rot"], a["k_rot"], a["v"], a["row_start"], a["ws"], 8, 2, stream=side)
    side.synchronize()
    assert torch.equal(got[:n], want[0][:n])


def test_beside_the_projections(dn):
    """qkv call, norms with rotation in place, attention, second sub-layer: a layer's attention part over a packed prompt, against
    the same attention through a paged cache."""
    import torch
    rows, d, hq, hk, D, r = 96, 512, 8, 2, 64, 48
    rng = np.random.default_rng(80)
    t = lambda *s: torch.tensor(rng.standard_normal(s) / s[0] ** 0.5, device="cuda").to(torch.bfloat16)
    fq, fk, fv = (dn.deinfer_pack_factors(dn.raw_pair(t(d, r), t(r, n))) for n in (hq * D, hk * D, hk * D))
    fo = dn.deinfer_pack_factors(dn.raw_pair(t(hq * D, r), t(r, d)))
    ws = dn.Workspace(dn.Workspace.bytes_for(rows, [fq, fk, fv]) + dn.Workspace.bytes_for(rows, [fo]))
    x = torch.tensor(rng.standard_normal((rows, d)), device="cuda").to(torch.bfloat16)
    q, k, v = dn.deinfer_lowrank_qkv(x, fq, fk, fv, ws)[:3]
    w = torch.ones(D, dtype=torch.bfloat16, device="cuda")
    freqs = torch.tensor(10000.0 ** (-2.0 * np.arange(D // 2) / D), device="cuda")
    start, new = ints(starts([60, 36])), [60, 36]
    pos = ints(np.r_[np.arange(60), np.arange(36)])
    # through the cache: block 0 .. 3 and 4 .. 6
    slots = ints(np.r_[np.arange(60), 64 + np.arange(36)])
    pools = [torch.zeros(7 * 16, hk * D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    q_out = torch.empty_like(q)
    dn.deinfer_norm_rope_store(q, k, v, pos, freqs, hq, hk, D, q_weight=w, k_weight=w, slots=slots, q_out=q_out, k_out=pools[0], v_out=pools[1])
    paged = dn.deinfer_tree_attention(q_out, *pools, ints([[0, 1, 2, 3], [4, 5, 6, -1]]), start, ints([0, 0]),
                                      dn.Workspace(dn.deinfer_tree_attention_workspace_bytes(rows, 2, hq, hk, D)), hq, hk, 16)
    # and straight
    dn.deinfer_norm_rope_store(q, k, None, pos, freqs, hq, hk, D, q_weight=w, k_weight=w)
    assert torch.equal(q, q_out)
    o = dn.deinfer_prompt_attention(q, k, v, start, dn.Workspace(dn.deinfer_prompt_attention_workspace_bytes(rows, 2, hq, hk, D)), hq, hk)
    # both round the probabilities and the output once each
    assert float((o.double() - paged.double()).abs().max()) <= 4 * 2.0 ** -8 * float(v.abs().max())
    y = dn.deinfer_lowrank_down(o, fo, ws)
    assert y.shape == (rows, d) and bool(torch.isfinite(y).all())
