"""CPU oracle for one step over a paged cache: slots from lengths, drafted trees, rotary positions, attention.

TEST INFRASTRUCTURE ONLY: imported by ``tests/`` (and nothing in the GPU package); it imports nothing from the
GPU package.  Plain Python loops and numpy in float64 / exact integers, written for reading, not for speed.
"""
from __future__ import annotations

import math

import numpy as np


def kv_step(cached, n_new, table, free_list, free_first, n_pool, bt, T):
    """(row_start, slots, positions, table, counts); table: [n_seqs][pitch], copied."""
    table = np.array(table, dtype=np.int64).copy()
    pitch = table.shape[1]
    row_start, slots, positions = [0], [-1] * T, [0] * T
    have = max(0, len(free_list) - free_first) if free_first >= 0 else 0
    asked = taken = wanted = rows = total = 0
    for s in range(len(cached)):
        c, m = max(0, int(cached[s])), max(0, int(n_new[s]))
        total += m
        m = min(m, T - rows)
        first, last = -(-c // bt), -(-(c + m) // bt)
        wanted += last - first
        for b in range(first, min(last, pitch)):
            block = -1
            if asked < have:
                block = int(free_list[free_first + asked])
                taken += 1
                if not 0 <= block < n_pool:
                    block = -1
            asked += 1
            table[s][b] = block
        for j in range(m):
            b = (c + j) // bt
            positions[rows] = c + j
            if b < pitch and 0 <= table[s][b] < n_pool:
                slots[rows] = int(table[s][b]) * bt + (c + j) % bt
            rows += 1
        row_start.append(rows)
    return np.array(row_start), np.array(slots), np.array(positions), table, np.array([total, taken, wanted - taken, free_first + taken])


def tree(parents, row_start, cached, words):
    """(bits [rows][words] as Python ints, positions) of the rows in use, in order."""
    bits, positions = [], []
    for s in range(len(cached)):
        n = int(row_start[s + 1]) - int(row_start[s])
        for j in range(n):
            mask, depth, at = 0, 0, j
            if j < 32 * words:
                mask = 1 << j
                while 0 <= int(parents[row_start[s] + at]) < at:
                    at = int(parents[row_start[s] + at])
                    mask |= 1 << at
                    depth += 1
            bits.append([(mask >> (32 * w)) & 0xFFFFFFFF for w in range(words)])
            positions.append(max(0, int(cached[s])) + depth)
    return bits, positions


def frequencies(rot_dim, theta, kind="plain", factor=1.0, context=0.0, low=0.0, high=0.0):
    """(angle per position of every pair, magnitude)."""
    out = []
    base = theta * factor ** (rot_dim / (rot_dim - 2)) if kind == "base" else theta
    for i in range(rot_dim // 2):
        f = base ** (-2.0 * i / rot_dim)
        if kind == "linear":
            f = f / factor
        elif kind == "bands":
            turns = context / (2 * math.pi / f)
            if turns <= low:
                f = f / factor
            elif turns < high:
                b = (turns - low) / (high - low)
                f = (1 - b) * f / factor + b * f
        elif kind == "ramp":
            pair = lambda t: rot_dim * math.log(context / (2 * math.pi * t)) / (2 * math.log(theta))
            lo, hi = max(0, math.floor(pair(high))), min(rot_dim - 1, math.ceil(pair(low)))
            r = min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001)))
            f = f * (1 - r) + f / factor * r
        out.append(f)
    return np.array(out), (0.1 * math.log(factor) + 1.0 if kind == "ramp" and factor > 1 else 1.0)


def rotate(x, positions, freqs, heads, head_dim, interleaved, magnitude=1.0):
    """x [rows][heads * head_dim] in float64, the first 2 len(freqs) elements of every head rotated."""
    y = np.array(x, dtype=np.float64).copy()
    half = len(freqs)
    for t in range(y.shape[0]):
        a = float(positions[t]) * np.asarray(freqs, dtype=np.float64)
        for h in range(heads):
            for i in range(half):
                u = h * head_dim + (2 * i if interleaved else i)
                w = h * head_dim + (2 * i + 1 if interleaved else i + half)
                p, q = x[t][u], x[t][w]
                y[t][u] = magnitude * (p * math.cos(a[i]) - q * math.sin(a[i]))
                y[t][w] = magnitude * (q * math.cos(a[i]) + p * math.sin(a[i]))
    return y


def attention(q, k_pool, v_pool, table, row_start, cached, n_q, n_kv, bt, scale, mask=None, out=None):
    """Rows in use of the output in float64; mask: [rows][words] of ints (None: causal); out: what padding rows hold."""
    T, D = q.shape[0], q.shape[1] // n_q
    n_blocks = k_pool.shape[0] // bt
    y = np.zeros((T, n_q * D)) if out is None else np.array(out, dtype=np.float64)
    for s in range(len(cached)):
        c = int(cached[s])
        for i in range(int(row_start[s + 1]) - int(row_start[s])):
            row = int(row_start[s]) + i
            slots = []
            for t in range(c + int(row_start[s + 1]) - int(row_start[s])):
                if t >= c:
                    j = t - c
                    if mask is None:
                        if j > i:
                            continue
                    elif j >= 32 * len(mask[row]) or not (int(mask[row][j // 32]) >> (j % 32)) & 1:
                        continue
                if t // bt < len(table[s]) and 0 <= int(table[s][t // bt]) < n_blocks:
                    slots.append(int(table[s][t // bt]) * bt + t % bt)
            for h in range(n_q):
                g = h // (n_q // n_kv)
                at = slice(h * D, (h + 1) * D)
                y[row, at] = 0.0
                if slots:
                    x = scale * (k_pool[slots, g * D:(g + 1) * D] @ q[row, at])
                    e = np.exp(x - np.max(x))
                    y[row, at] = (e / np.sum(e)) @ v_pool[slots, g * D:(g + 1) * D]
    return y
