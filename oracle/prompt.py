"""Plain 64-bit forms of the calls between the projections of a prompt: positions of several axes, norms of heads with their
rotation, attention of packed sequences.  Written from the formulas, a token, a head and a sequence at a time."""
import math

import numpy as np


def axis_positions(segments, segment_start, row_start, cached, T, positions):
    """positions [3, T] with the columns of the rows in use written; segments: [n, 4] of {t, h, w, step}."""
    out = np.array(positions, dtype=np.int64)
    for s in range(len(segment_start) - 1):
        g0, g1 = max(0, int(segment_start[s])), min(len(segments), int(segment_start[s + 1]))
        r0, r1 = max(0, int(row_start[s])), min(T, int(row_start[s + 1]))
        token = max(0, int(cached[s])) if cached is not None else 0
        for r in range(r0, r1):
            at, p = token + r - r0, 0
            found = None
            for t, h, w, step in (tuple(int(x) for x in seg) for seg in segments[g0:g1]):
                t, step = max(t, 0), max(step, 0)
                text = h <= 0 or w <= 0
                n = t if text else t * h * w
                if at < n:
                    found = (p + at,) * 3 if text else (p + at // (h * w) * step, p + at % (h * w) // w, p + at % w)
                    break
                at -= n
                if t:
                    p += t if text else max(step * (t - 1), h - 1, w - 1) + 1
            out[:, r] = np.minimum(found if found is not None else (p + at,) * 3, 2 ** 31 - 1)
    return out


def rope_axes(pairs, turns):
    left, out = list(pairs), []
    if not turns:
        return [a for a, n in enumerate(left) for _ in range(n)]
    while any(left):
        for a in range(len(left)):
            if left[a]:
                out.append(a)
                left[a] -= 1
    return out


def norm_rope(x, heads, weight, eps, angles, magnitude, interleaved):
    """x [T, heads * D] normed for each head (weight None: not) and rotated by angles [T, rot_dim / 2]."""
    T, D, half = x.shape[0], x.shape[1] // heads, angles.shape[1]
    y = np.array(x, dtype=np.float64).reshape(T, heads, D)
    if weight is not None:
        with np.errstate(all="ignore"):
            y = np.asarray(weight, dtype=np.float64) * (y / np.sqrt(np.mean(y * y, axis=2, keepdims=True) + eps))
    first = np.arange(half) * (2 if interleaved else 1)
    second = first + (1 if interleaved else half)
    a, b = y[:, :, first], y[:, :, second]
    c, s = magnitude * np.cos(angles)[:, None, :], magnitude * np.sin(angles)[:, None, :]
    out = y.copy()
    out[:, :, first], out[:, :, second] = a * c - b * s, b * c + a * s
    return out.reshape(T, heads * D)


def attention(q, k, v, q_start, k_start, n_q, n_kv, left, right, scale, out):
    """Rows of the packed sequences; the others as in ``out``."""
    out = np.array(out, dtype=np.float64)
    D, group = q.shape[1] // n_q, n_q // n_kv
    if k_start is None:
        k_start = q_start
    for s in range(len(q_start) - 1):
        r0, r1 = max(0, int(q_start[s])), min(q.shape[0], int(q_start[s + 1]))
        j0, j1 = max(0, int(k_start[s])), min(k.shape[0], int(k_start[s + 1]))
        rows, keys = max(0, r1 - r0), max(0, j1 - j0)
        place = keys - rows + np.arange(rows)[:, None]
        j = np.arange(keys)[None, :]
        sees = np.ones((rows, keys), dtype=bool)
        if left >= 0:
            sees &= j >= place - left
        if right >= 0:
            sees &= j <= place + right
        for h in range(n_q):
            of = slice(h // group * D, (h // group + 1) * D)
            at = slice(h * D, (h + 1) * D)
            if rows == 0:
                continue
            x = np.where(sees, scale * (q[r0:r0 + rows, at] @ k[j0:j0 + keys, of].T), -math.inf) if keys else np.full((rows, 1), -math.inf)
            top = np.max(x, axis=1, keepdims=True)
            p = np.exp(x - np.where(top == -math.inf, 0.0, top))
            total = np.sum(p, axis=1, keepdims=True)
            out[r0:r0 + rows, at] = (p / np.where(total > 0.0, total, 1.0)) @ v[j0:j0 + keys, of] if keys else 0.0
    return out
