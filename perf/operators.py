"""Performance cases of one step over the paged cache: from the requests' lengths to the attention that reads the cache.

Five kinds of case, each one public entry point of the library:
  step    block tables, slots and positions of the step's tokens from the lengths, ``deinfer_kv_step``;
  plan    the runs of the compacting copy from the block tables on the device, ``deinfer_kv_compact_plan_device``;
  tree    visibility bits and positions of drafted trees from their parents, ``deinfer_tree_mask``;
  rope    queries rotated, keys rotated into their slots of the cache, values stored beside them, ``deinfer_rope_store``;
  attend  attention of the step's tokens over the paged cache, ``deinfer_tree_attention``.

Lengths go by the case (their order among the sequences by the seed), everything else by the seed.  Row buffers are a little
longer than the rows in use, as in a program that replays one captured graph for every step.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
MAX_SCORES = 1.0e9        # padded scores of a drawn attention case (the largest listed one: 1.08e9)
MAX_CACHE = 5.0e8         # padded key values of a drawn attention case (the largest listed one: 5.4e8)


def listed():
    return [
        # eight users, one token each: the latency of a step's bookkeeping
        {"name": "step_8_seqs", "op": "step", "seqs": 8, "cached": 2000, "new": 1, "block": 16},
        # a large batch of requests that mixes prompts, chunks and single tokens
        {"name": "step_2048_seqs", "op": "step", "seqs": 2048, "cached": 4000, "new": 500, "block": 16},
        # the benchmark's rebuild state: 16 sequences of 32 blocks
        {"name": "plan_16_seqs", "op": "plan", "seqs": 16, "tokens": 512, "block": 16},
        # a full cache: 1024 sequences, about 33000 blocks
        {"name": "plan_1024_seqs", "op": "plan", "seqs": 1024, "tokens": 1040, "block": 16},
        # a few drafted tokens for each of 16 users
        {"name": "tree_16_seqs", "op": "tree", "seqs": 16, "drafted": 8},
        # wide drafts for a large batch
        {"name": "tree_256_seqs", "op": "tree", "seqs": 256, "drafted": 256},
        # one token for each of 8 users, grouped heads of the 70B shape
        {"name": "rope_8_rows", "op": "rope", "rows": 8, "q_heads": 64, "kv_heads": 8, "head": 128, "rotated": 128, "interleaved": False, "type": "bf16", "block": 16},
        # a prompt of 8191 tokens, neighbouring pairs, half of every head rotated
        {"name": "rope_8191_rows", "op": "rope", "rows": 8191, "q_heads": 32, "kv_heads": 32, "head": 128, "rotated": 64, "interleaved": True, "type": "f16", "block": 32},
        # one token for each of 8 users over short contexts: latency
        {"name": "attend_8_x_1k", "op": "attend", "seqs": 8, "cached": 1000, "new": 1, "tree": False, "q_heads": 64, "kv_heads": 8, "head": 128, "type": "bf16", "block": 16},
        # a decode batch over long, ragged contexts: the cache read once
        {"name": "attend_64_x_8k", "op": "attend", "seqs": 64, "cached": 8191, "new": 1, "tree": False, "q_heads": 64, "kv_heads": 8, "head": 128, "type": "bf16", "block": 16},
        # drafted trees verified over long contexts
        {"name": "attend_tree_16_x_16k", "op": "attend", "seqs": 16, "cached": 16384, "new": 64, "tree": True, "q_heads": 64, "kv_heads": 8, "head": 128, "type": "f16", "block": 32},
        # chunks of two prompts, a head for every query head
        {"name": "attend_chunk_2_x_2k", "op": "attend", "seqs": 2, "cached": 6000, "new": 2048, "tree": False, "q_heads": 32, "kv_heads": 32, "head": 128, "type": "bf16", "block": 16},
    ]


def _spread(rng, lo, hi):
    """A whole number whose logarithm is spread evenly over [lo, hi]."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["step", "plan", "tree", "rope", "rope", "attend", "attend", "attend", "attend"])
    block = rng.choice([8, 16, 16, 32, 64])
    if op == "step":
        seqs = _spread(rng, 1, 2048)
        return {"op": op, "seqs": seqs, "cached": _spread(rng, 16, 16384), "new": min(_spread(rng, 1, 4096), 1000000 // seqs), "block": block}
    if op == "plan":
        seqs = _spread(rng, 1, 1024)
        return {"op": op, "seqs": seqs, "tokens": max(1, min(_spread(rng, 16, 131072), 33000 * block * 2 // seqs)), "block": block}
    if op == "tree":
        return {"op": op, "seqs": _spread(rng, 1, 256), "drafted": _spread(rng, 2, 256)}
    kv_heads = rng.choice([1, 2, 4, 8, 8, 16, 32])
    group = rng.choice([1, 1, 2, 4, 5, 7, 8]) if kv_heads <= 8 else 1
    head = rng.choice([64, 80, 96, 128, 128, 128, 256])
    if op == "rope":
        rotated = rng.choice([head, head, head // 2])
        rows = _spread(rng, 1, 8192)
        kind = rng.choice(["bf16", "bf16", "f16", "f32"])
        while rows * kv_heads * (group + 2) * head > 1.0e8:
            rows = rows * 3 // 4
        return {"op": op, "rows": rows, "q_heads": kv_heads * group, "kv_heads": kv_heads, "head": head, "rotated": rotated,
                "interleaved": rng.random() < 0.4, "type": kind, "block": block}
    shape = rng.choice(["decode", "decode", "tree", "chunk"])
    seqs = _spread(rng, 1, 128) if shape != "chunk" else _spread(rng, 1, 4)
    new = 1 if shape == "decode" else _spread(rng, 2, 128) if shape == "tree" else _spread(rng, 64, 2048)
    cached = _spread(rng, 64, 131072) if shape != "chunk" else _spread(rng, 16, 16384)
    while seqs * (cached + new) * kv_heads * head > MAX_CACHE or seqs * (cached + new) * new * kv_heads * group > MAX_SCORES:
        if cached > new:
            cached = cached * 3 // 4
        else:
            new = max(1, new * 3 // 4)
    return {"op": op, "seqs": seqs, "cached": cached, "new": new, "tree": shape == "tree", "q_heads": kv_heads * group, "kv_heads": kv_heads,
            "head": head, "type": rng.choice(["bf16", "bf16", "f16"]), "block": block}


def _ragged(case, n, lo, hi, tag):
    """n lengths between lo and hi that go by the case alone, the longest among them."""
    rng = random.Random("%s %s" % (tag, sorted((k, v) for k, v in case.items() if k != "name")))
    return [hi] + [rng.randint(lo, hi) for _ in range(n - 1)]


def _lengths(case):
    """(cached, new) of every sequence, before the seed shuffles the sequences."""
    n = case["seqs"]
    if case["op"] == "step":
        return _ragged(case, n, 0, case["cached"], "cached"), _ragged(case, n, min(1, case["new"] // 2), case["new"], "new")
    if case["op"] == "plan":
        return _ragged(case, n, min(case["tokens"], 2) if n < 16 else case["tokens"] // 2, case["tokens"], "tokens"), [0] * n
    if case["op"] == "tree":
        return _ragged(case, n, 0, 4096, "cached"), _ragged(case, n, max(1, case["drafted"] // 2), case["drafted"], "drafted")
    return _ragged(case, n, 0, case["cached"], "cached"), _ragged(case, n, max(1, case["new"] // 2), case["new"], "new")


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _exclusive(values):
    out = [0]
    for v in values:
        out.append(out[-1] + v)
    return out


def _tables(lengths, block, pool_blocks, gen, contiguous):
    """A block table per sequence over a pool: scattered blocks, or the first three quarters of a sequence in one run as a prompt's."""
    owned = [-(-n // block) for n in lengths]
    ids = torch.randperm(pool_blocks, generator=gen, device="cuda", dtype=torch.int32)
    if contiguous:
        runs = [3 * n // 4 for n in owned]
        ids = torch.cat([torch.arange(sum(runs), device="cuda", dtype=torch.int32),
                         torch.randperm(pool_blocks - sum(runs), generator=gen, device="cuda", dtype=torch.int32) + sum(runs)])
    pitch = max(1, max(owned)) + 2
    table = torch.full((len(lengths), pitch), -1, dtype=torch.int32, device="cuda")
    column = torch.arange(pitch, device="cuda")[None, :]
    n = torch.tensor(owned, device="cuda")[:, None]
    if contiguous:
        r = torch.tensor(runs, device="cuda")[:, None]
        base = torch.tensor(_exclusive(runs)[:-1], device="cuda")[:, None]
        rest = torch.tensor(_exclusive([a - b for a, b in zip(owned, runs)])[:-1], device="cuda")[:, None] + sum(runs)
        at = torch.where(column < r, base + column, rest + column - r)
    else:
        at = torch.tensor(_exclusive(owned)[:-1], device="cuda")[:, None] + column
    return torch.where(column < n, ids[at.clamp(max=pool_blocks - 1)], table).contiguous()


def _mask_of_parents(parents, row_start, most, words):
    """Ancestors (and the row itself) as bits, and the depth, for every row: powers of the parents' matrix, two steps further each time."""
    rows = parents.numel()
    seqs = row_start.numel() - 1
    row = torch.arange(rows, device=parents.device)
    seq = torch.searchsorted(row_start[1:].long(), row, right=True)
    inside = seq < seqs
    at = seq.clamp(max=seqs - 1)
    j = row - row_start.long()[at]
    ok = inside & (parents >= 0) & (parents < j) & (j < 32 * words)
    reach = torch.zeros(seqs, most, most + 1, device=parents.device)
    reach[at, j.clamp(max=most - 1), torch.where(ok, parents.long(), most)] += inside.float()
    reach = reach[:, :, :most] + torch.eye(most, device=parents.device)
    length = 1
    while length < most:
        reach = (torch.matmul(reach, reach.contiguous()) > 0).float()
        length *= 2
    bits = torch.zeros(rows, 32 * words, device=parents.device, dtype=torch.int64)
    mine = reach[at, j.clamp(max=most - 1)] * inside[:, None]
    bits[:, :min(most, 32 * words)] = mine[:, :32 * words].long()
    packed = (bits.view(rows, words, 32) << torch.arange(32, device=parents.device)).sum(2)
    packed = torch.where(packed >= 2 ** 31, packed - 2 ** 32, packed).to(torch.int32)
    return packed, mine.sum(1).long() - 1, at, inside


def _frequencies(rotated, gen_scale, device="cuda"):
    """theta^(-2 i / D) with the long wavelengths slowed down by bands of wavelength, in 64 bits."""
    i = torch.arange(rotated // 2, dtype=torch.float64)
    f = 500000.0 ** (-2.0 * i / rotated)
    wave = 2.0 * math.pi / f
    blend = ((8192.0 / wave - 1.0) / (4.0 - 1.0)).clamp(0.0, 1.0)
    return ((1.0 - blend) * f / gen_scale + blend * f).to(device)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]
    s = {"op": op, "case": case}
    if op == "rope":
        kind, rows, heads = DTYPES[case["type"]], case["rows"], case["kv_heads"]
        slots = (rows // case["block"] + 3) * case["block"]
        # one row more than the cache has: where a plain scatter puts the rows that have no slot
        s.update(q=torch.randn(rows, case["q_heads"] * case["head"], generator=gen, device="cuda").to(kind),
                 k=torch.randn(rows, heads * case["head"], generator=gen, device="cuda").to(kind),
                 v=torch.randn(rows, heads * case["head"], generator=gen, device="cuda").to(kind),
                 k_pool=torch.zeros(slots + 1, heads * case["head"], dtype=kind, device="cuda"),
                 v_pool=torch.zeros(slots + 1, heads * case["head"], dtype=kind, device="cuda"),
                 positions=torch.randint(0, 131072, (rows,), generator=gen, device="cuda", dtype=torch.int32),
                 slots=torch.randperm(slots, generator=gen, device="cuda", dtype=torch.int32)[:rows].contiguous(),
                 freqs=_frequencies(case["rotated"], 8.0))
        s["q_out"] = torch.zeros_like(s["q"])
        s["pool"] = (s["k_pool"][:slots], s["v_pool"][:slots])
        return s
    cached, new = _lengths(case)
    order = random.Random(seed).sample(range(case["seqs"]), case["seqs"])
    cached, new = [cached[i] for i in order], [new[i] for i in order]
    starts = _exclusive(new)
    total = starts[-1]
    rows = -(-(total + 1) // 8) * 8
    s.update(cached=_int(cached), new=_int(new), rows=rows)
    if op == "step":
        block = case["block"]
        lengths = [a + b for a, b in zip(cached, new)]
        need = sum(-(-n // block) for n in lengths)
        pool = need + need // 4 + 1
        s["table"] = _tables(cached, block, pool, gen, False)
        pitch = max(-(-n // block) for n in lengths) + 1
        s["table"] = torch.nn.functional.pad(s["table"], (0, max(0, pitch - s["table"].shape[1])), value=-1).contiguous()
        used = sum(-(-n // block) for n in cached)
        s["free"] = (torch.randperm(pool - used, generator=gen, device="cuda", dtype=torch.int32) + used).contiguous()
        s["pool_blocks"] = pool
    elif op == "plan":
        block = case["block"]
        need = sum(-(-n // block) for n in cached)
        s["pool_blocks"] = need + need // 4 + 1
        s["buffer_blocks"] = need + 5
        s["table"] = _tables(cached, block, s["pool_blocks"], gen, True)
    elif op == "tree":
        s["row_start"] = _int(starts)
        words = -(-case["drafted"] // 32)
        j = torch.arange(rows, device="cuda") - s["row_start"].long()[torch.searchsorted(s["row_start"][1:].long(), torch.arange(rows, device="cuda"), right=True).clamp(max=case["seqs"] - 1)]
        back = (torch.rand(rows, generator=gen, device="cuda") * 6).long() + 1        # the parent is one of the six rows before, or the cached text
        s["parents"] = (j - back).clamp(min=-1).to(torch.int32)
        s["mask"] = torch.zeros(rows, words, dtype=torch.int32, device="cuda")
        s["positions"] = torch.zeros(rows, dtype=torch.int32, device="cuda")
    else:
        kind, block, heads, head = DTYPES[case["type"]], case["block"], case["kv_heads"], case["head"]
        lengths = [a + b for a, b in zip(cached, new)]
        need = sum(-(-n // block) for n in lengths)
        pool = need + need // 8 + 1
        s["table"] = _tables(lengths, block, pool, gen, False)
        s["row_start"] = _int(starts)
        s["q"] = torch.randn(rows, case["q_heads"] * head, generator=gen, device="cuda").to(kind)
        s["k_pool"] = torch.randn(pool * block, heads * head, generator=gen, device="cuda", dtype=kind)
        s["v_pool"] = torch.randn(pool * block, heads * head, generator=gen, device="cuda", dtype=kind)
        s["out"] = torch.zeros(rows, case["q_heads"] * head, dtype=kind, device="cuda")
        s["longest"], s["most"] = max(lengths), max(new)
        s["mask"] = None
        if case["tree"]:
            j = torch.cat([torch.arange(n) for n in new] + [torch.zeros(rows - total, dtype=torch.int64)]).cuda()
            back = (torch.rand(rows, generator=gen, device="cuda") * 6).long() + 1
            s["mask"] = _mask_of_parents((j - back).clamp(min=-1).to(torch.int32), s["row_start"], s["most"], -(-s["most"] // 32))[0]
    return s


def _step(s):
    """From the lengths: [row_start, slots, positions, block table, counts]."""
    block, rows, table, free = s["case"]["block"], s["rows"], s["table"], s["free"]
    if own:
        import paper_2604_17709_amd as dn
        step = dn.deinfer_kv_step(s["cached"], s["new"], table, free, block, s["pool_blocks"], rows)
        return [step.row_start, step.slots, step.positions, table, step.counts]
    cached = s["cached"].long()
    pitch = table.shape[1]
    ends = s["new"].long().cumsum(0)
    row_start = torch.cat([ends.new_zeros(1), ends]).clamp(max=rows)
    new = row_start[1:] - row_start[:-1]
    first = (cached + block - 1) // block
    last = (cached + new + block - 1) // block
    need = last.clamp(max=pitch) - first.clamp(max=pitch)
    before = need.cumsum(0) - need
    column = torch.arange(pitch, device=table.device)[None, :]
    at = before[:, None] + column - first[:, None]
    fresh = torch.where(at < free.numel(), free[at.clamp(0, free.numel() - 1)], -1)
    table = torch.where((column >= first[:, None]) & (column < last[:, None]), fresh, table)
    row = torch.arange(rows, device=table.device)
    seq = torch.searchsorted(row_start[1:], row, right=True)
    used = seq < new.numel()
    seq = seq.clamp(max=new.numel() - 1)
    position = torch.where(used, cached[seq] + row - row_start[seq], 0)
    page = position // block
    held = table[seq, page.clamp(max=pitch - 1)].long()
    slot = torch.where(used & (page < pitch) & (held >= 0), held * block + position % block, -1)
    taken = need.sum().clamp(max=free.numel())
    counts = torch.stack([ends[-1], taken, (last - first).sum() - taken, taken]).to(torch.int32)
    return [row_start.to(torch.int32), slot.to(torch.int32), position.to(torch.int32), table, counts]


def _plan(s):
    """From the block tables: [plan of runs, remapped table, positions of the buffer's token slots]."""
    block, table, buffer_blocks, cached = s["case"]["block"], s["table"], s["buffer_blocks"], s["cached"]
    if own:
        import paper_2604_17709_amd as dn
        return list(dn.deinfer_kv_compact_plan_device(table, cached, s["pool_blocks"], buffer_blocks, block))
    blocks = (cached.long() + block - 1) // block
    ends = blocks.cumsum(0)
    d = torch.arange(buffer_blocks, device=table.device)
    seq = torch.searchsorted(ends, d, right=True)
    used = seq < blocks.numel()
    seq = seq.clamp(max=blocks.numel() - 1)
    i = torch.where(used, d - (ends - blocks)[seq], 0)
    held = table[seq, i].long()
    head = used & ((d == 0) | (held != torch.roll(held, 1) + 1))
    run = head.long().cumsum(0) - 1
    plan = torch.zeros(4 + 3 * buffer_blocks + 3, dtype=torch.int64, device=table.device)      # three words more: for what is no head
    to = torch.where(head, 4 + 3 * run, 4 + 3 * buffer_blocks)
    plan[to] = held
    plan[to + 1] = d
    plan.index_add_(0, torch.where(used, 4 + 3 * run, 4 + 3 * buffer_blocks) + 2, torch.ones_like(d))
    plan[0] = head.sum()
    plan[1] = ends[-1]
    column = torch.arange(table.shape[1], device=table.device)[None, :]
    remap = torch.where(column < blocks[:, None], (ends - blocks)[:, None] + column, -1)
    positions = torch.where(used[:, None], i[:, None] * block + torch.arange(block, device=table.device), 0)
    return [plan[:4 + 3 * buffer_blocks].to(torch.int32), remap.to(torch.int32), positions.reshape(-1).to(torch.int32)]


def _tree(s):
    """From the drafted tokens' parents: [visibility bits, positions]; rows in use only are written."""
    if own:
        import paper_2604_17709_amd as dn
        return list(dn.deinfer_tree_mask(s["parents"], s["row_start"], s["cached"], s["mask"], s["positions"]))
    packed, depth, seq, inside = _mask_of_parents(s["parents"], s["row_start"], s["case"]["drafted"], s["mask"].shape[1])
    positions = s["cached"].long()[seq] + depth
    return [torch.where(inside[:, None], packed, s["mask"]), torch.where(inside, positions.to(torch.int32), s["positions"])]


def _rotated(x, heads, head, rotated, interleaved, cos, sin):
    rows = x.shape[0]
    x = x.float().view(rows, heads, head)
    part = x[..., :rotated]
    if interleaved:
        a, b = part[..., 0::2], part[..., 1::2]
    else:
        a, b = part[..., :rotated // 2], part[..., rotated // 2:]
    c, d = cos[:, None, :], sin[:, None, :]
    a, b = a * c - b * d, b * c + a * d
    part = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([part, x[..., rotated:]], -1).reshape(rows, heads * head)


def _rope(s):
    """[rotated queries, key cache, value cache]."""
    c = s["case"]
    if own:
        import paper_2604_17709_amd as dn
        dn.deinfer_rope_store(s["q"], s["k"], s["v"], s["positions"], s["freqs"], c["q_heads"], c["kv_heads"], c["head"],
                              interleaved=c["interleaved"], slots=s["slots"], q_out=s["q_out"], k_out=s["pool"][0], v_out=s["pool"][1])
        return [s["q_out"], *s["pool"]]
    angle = s["positions"].double()[:, None] * s["freqs"]
    cos, sin = angle.cos().float(), angle.sin().float()
    q = _rotated(s["q"], c["q_heads"], c["head"], c["rotated"], c["interleaved"], cos, sin).to(s["q"].dtype)
    k = _rotated(s["k"], c["kv_heads"], c["head"], c["rotated"], c["interleaved"], cos, sin).to(s["k"].dtype)
    to = torch.where(s["slots"] >= 0, s["slots"].long(), s["k_pool"].shape[0] - 1)
    s["k_pool"][to] = k
    s["v_pool"][to] = s["v"]
    return [q, *s["pool"]]


def _attend(s):
    """Attention outputs, one row for every row in use."""
    c = s["case"]
    heads, head, block = c["kv_heads"], c["head"], c["block"]
    if own:
        import paper_2604_17709_amd as dn
        if "ws" not in s:
            s["ws"] = dn.Workspace(dn.deinfer_tree_attention_workspace_bytes(s["rows"], c["seqs"], c["q_heads"], heads, head))
        return dn.deinfer_tree_attention(s["q"], s["k_pool"], s["v_pool"], s["table"], s["row_start"], s["cached"], s["ws"],
                                         c["q_heads"], heads, block, mask=s["mask"], out=s["out"])
    seqs, most, longest, group = c["seqs"], s["most"], s["longest"], c["q_heads"] // heads
    table, start, cached, dev = s["table"], s["row_start"].long(), s["cached"].long(), s["q"].device
    new = start[1:] - start[:-1]
    position = torch.arange(longest, device=dev)
    slot = (table[:, position // block].long() * block + position % block).clamp(min=0)
    live = position[None, :] < (cached + new)[:, None]
    k = s["k_pool"][slot].float().view(seqs, longest, heads, head).permute(0, 2, 3, 1).contiguous()
    v = torch.where(live[:, :, None], s["v_pool"][slot].float(), 0.0).view(seqs, longest, heads, head).permute(0, 2, 1, 3).contiguous()
    i = torch.arange(most, device=dev)
    row = (start[:-1, None] + i).clamp(max=s["rows"] - 1)
    q = s["q"][row].float().view(seqs, most, heads, group, head).permute(0, 2, 1, 3, 4).reshape(seqs, heads, most * group, head)
    drafted = position[None, :] - cached[:, None]                            # index among the step's tokens, negative for cached ones
    if s["mask"] is None:
        seen = drafted[:, None, :] <= i[None, :, None]
    else:
        word = s["mask"][row]
        at = drafted.clamp(min=0, max=32 * word.shape[2] - 1)
        bit = torch.gather(word, 2, (at // 32)[:, None, :].expand(seqs, most, longest)) >> (at % 32)[:, None, :].int()
        seen = (drafted < 0)[:, None, :] | ((bit & 1) > 0)
    seen = (seen & live[:, None, :])[:, None, :, None, :]
    score = (torch.matmul(q, k) * head ** -0.5).view(seqs, heads, most, group, longest)
    score = torch.where(seen, score, -math.inf)
    top = score.amax(-1, keepdim=True)
    score = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    total = score.sum(-1, keepdim=True)
    o = torch.matmul(score.view(seqs, heads, most * group, longest), v).view(seqs, heads, most, group, head)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 2, 1, 3, 4).reshape(seqs, most, heads * group * head).to(s["q"].dtype)
    r = torch.arange(s["rows"], device=dev)
    seq = torch.searchsorted(start[1:], r, right=True)
    used = seq < seqs
    seq = seq.clamp(max=seqs - 1)
    return torch.where(used[:, None], o[seq, (r - start[seq]).clamp(max=most - 1)], s["out"])


def run(state):
    return {"step": _step, "plan": _plan, "tree": _tree, "rope": _rope, "attend": _attend}[state["op"]](state)


def work(case):
    op = case["op"]
    if op == "rope":
        q, kv = case["rows"] * case["q_heads"] * case["head"], case["rows"] * case["kv_heads"] * case["head"]
        size = 4 if case["type"] == "f32" else 2
        return {"bytes": size * (2 * q + 4 * kv) + 8 * case["rows"], "flops": 3 * (q + kv) * case["rotated"] / case["head"]}
    cached, new = _lengths(case)
    n, total = case["seqs"], sum(new)
    if op == "step":
        blocks = sum(-(-(a + b) // case["block"]) - -(-a // case["block"]) for a, b in zip(cached, new))
        return {"bytes": 4 * (3 * n + 2 * blocks + n + 2 * total), "flops": total}
    if op == "plan":
        blocks = sum(-(-a // case["block"]) for a in cached)
        return {"bytes": 4 * (n + 2 * blocks + 3 * blocks / 4 + blocks * case["block"]), "flops": blocks}
    if op == "tree":
        return {"bytes": 4 * (2 * n + total * (2 + -(-case["drafted"] // 32))), "flops": total * -(-case["drafted"] // 32)}
    # attention: all cached tokens, and of the step's own tokens half (a causal chunk) or, in a tree, a few
    pairs = sum(b * (a + (b / 2 if not case["tree"] else min(b, 16))) for a, b in zip(cached, new))
    keys = sum(a + b for a, b in zip(cached, new))
    return {"bytes": 2 * (2 * keys * case["kv_heads"] * case["head"] + 2 * total * case["q_heads"] * case["head"]),
            "flops": 4.0 * pairs * case["q_heads"] * case["head"]}


def exact(case, seed):
    """The rotations and the attention in 64 bits, a sequence and a head at a time; the other outputs are whole numbers."""
    if case["op"] not in ("rope", "attend"):
        return None
    s = prepare(case, seed)
    head, group = case["head"], case["q_heads"] // case["kv_heads"]
    if case["op"] == "rope":
        rotated = case["rotated"]
        i = torch.arange(rotated // 2, device="cuda")
        first = 2 * i if case["interleaved"] else i
        second = 2 * i + 1 if case["interleaved"] else i + rotated // 2
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["positions"].double()[:, None] * s["freqs"])
        found = []
        for name, heads in (("q", case["q_heads"]), ("k", case["kv_heads"])):
            x = s[name].double()
            for h in range(heads):
                z = torch.complex(x[:, h * head + first], x[:, h * head + second]) * turn
                x[:, h * head + first], x[:, h * head + second] = z.real, z.imag
            found.append(x)
        pools = [p.double() for p in s["pool"]]
        pools[0][s["slots"].long()] = found[1]
        pools[1][s["slots"].long()] = s["v"].double()
        return [found[0], *pools]
    out = s["out"].double()
    starts, cached = s["row_start"].tolist(), s["cached"].tolist()
    for n in range(case["seqs"]):
        rows, length = starts[n + 1] - starts[n], cached[n] + starts[n + 1] - starts[n]
        pages = s["table"][n, :-(-length // case["block"])].long()
        slot = (pages[:, None] * case["block"] + torch.arange(case["block"], device="cuda")).reshape(-1)[:length]
        sees = torch.ones(rows, length, dtype=torch.bool, device="cuda")
        if s["mask"] is None:
            sees[:, cached[n]:] = torch.ones(rows, rows, dtype=torch.bool, device="cuda").tril()
        else:
            words = s["mask"][starts[n]:starts[n + 1]]
            for j in range(rows):
                sees[:, cached[n] + j] = (words[:, j // 32] >> (j % 32)) & 1 != 0
        for h in range(case["kv_heads"]):
            k = s["k_pool"][slot, h * head:(h + 1) * head].double()
            v = s["v_pool"][slot, h * head:(h + 1) * head].double()
            for g in range(group):
                at = slice((h * group + g) * head, (h * group + g + 1) * head)
                a = s["q"][starts[n]:starts[n + 1], at].double() @ k.T / math.sqrt(head)
                a[~sees] = -math.inf
                out[starts[n]:starts[n + 1], at] = torch.softmax(a, 1) @ v
    return out
