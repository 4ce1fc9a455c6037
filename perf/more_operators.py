"""Operators of a program that serves prompts of different lengths from one pool of cache pages, as its user calls them.

A case is one pass through one operator of ``paper_1904_10509_amd.sparse_attn`` at one size:

  tables  page tables, first rows, positions and cache slots of a batch, made on the GPU from the sequences' lengths;
  store   the batch's new keys and values (packed, one sequence behind the other) into their slots of the pages;
  packed  attention over whole prompts packed one behind the other: factorized sets or dense causal, shared key heads;
  decode  one new token a sequence over the pages, every sequence at a position of its own.

``own`` chooses between the package's operators and their plain form in elementary torch operations.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
PATTERNS = {"strided": 0, "fixed": 1, "fixed_per_head": 2}
MODES = {"A1": 0, "A2": 1, "merged": 2, "interleaved": 3}


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------
def _tables(sequences, held, fresh, page, ragged, mix):
    """held, fresh: the most tokens that a sequence has in the cache and brings along; ragged: others have fewer."""
    return dict(kind="tables", sequences=sequences, held=held, fresh=fresh, page=page, ragged=ragged, mix=mix)


def _store(sequences, held, fresh, page, ragged, mix, kv_heads, d, dtype):
    return dict(kind="store", sequences=sequences, held=held, fresh=fresh, page=page, ragged=ragged, mix=mix,
                kv_heads=kv_heads, d=d, dtype=dtype)


def _packed(sequences, longest, ragged, mix, heads, kv_heads, d, dtype, pattern, mode, l, c, fused):
    """l = 0: dense causal.  fused: q, k and v are parts of one tensor, as a joint projection leaves them."""
    return dict(kind="packed", sequences=sequences, longest=longest, ragged=ragged, mix=mix, heads=heads,
                kv_heads=kv_heads, d=d, dtype=dtype, pattern=pattern, mode=mode, l=l, c=c, fused=fused)


def _decode(batch, pos, ragged, mix, heads, kv_heads, d, dtype, pattern, mode, l, c, page):
    """pos: the furthest position.  l = 0: dense."""
    return dict(kind="decode", batch=batch, pos=pos, ragged=ragged, mix=mix, heads=heads, kv_heads=kv_heads, d=d,
                dtype=dtype, pattern=pattern, mode=mode, l=l, c=c, page=page)


def listed():
    cases = [
        # the bookkeeping of one step of 32 generating sequences: all latency
        ("tables_step_32", _tables(32, 16384, 1, 64, True, 1)),
        # the bookkeeping of many prompts that arrive together, some of them turns of a longer talk
        ("tables_prompts", _tables(1000, 3000, 2000, 16, True, 2)),
        # the new token of 32 sequences
        ("store_step_32", _store(32, 16384, 1, 64, True, 3, 8, 64, "bf16")),
        # the prompts of a batch, 65,536 tokens and more
        ("store_prompts", _store(24, 5000, 12288, 64, True, 4, 8, 64, "bf16")),
        # four short prompts: latency
        ("packed_short", _packed(4, 200, True, 5, 8, 8, 64, "bf16", "fixed", "merged", 128, 32, True)),
        # text prompts of up to 12,288 tokens, strided
        ("packed_text", _packed(6, 12288, True, 6, 8, 8, 64, "bf16", "strided", "merged", 128, 0, True)),
        # dense causal layers, key heads shared in eights: the most arithmetic
        ("packed_dense", _packed(9, 8192, True, 7, 32, 4, 128, "bf16", "strided", "A1", 0, 0, True)),
        # audio sequences of 65,536, fixed
        ("packed_audio", _packed(2, 65536, True, 8, 8, 8, 64, "bf16", "fixed", "merged", 256, 32, False)),
        # single precision, alternating factors with a summary subblock per head, odd lengths
        ("packed_f32", _packed(5, 2777, True, 9, 8, 4, 128, "f32", "fixed_per_head", "interleaved", 128, 32, False)),
        # sampling one text sequence: the latency of a step
        ("decode_text_one", _decode(1, 9999, False, 10, 8, 8, 64, "bf16", "strided", "merged", 128, 0, 64)),
        # dense layers of 16 sequences, key heads shared in eights: the throughput of a step
        ("decode_dense_16", _decode(16, 32767, True, 11, 32, 4, 128, "bf16", "strided", "A1", 0, 0, 64)),
        # sampling in single precision, heads of alternating factors with a summary subblock each, small pages
        ("decode_subblocks_f32", _decode(3, 12001, True, 12, 8, 8, 128, "f32", "fixed_per_head", "interleaved", 128, 32, 16)),
    ]
    return [dict(name=name, **case) for name, case in cases]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def _pattern(rng, longest):
    """(pattern, mode, l, c); a quarter of them dense."""
    if rng.random() < 0.25:
        return "strided", "A1", 0, 0
    pattern = rng.choice(["strided", "fixed", "fixed", "fixed_per_head"])
    l = rng.choice([128, 256, max(16, int(math.sqrt(longest))), rng.randint(16, 400)])
    c = 0 if pattern == "strided" else max(1, min(l, rng.choice([8, 32, 32, l // 8])))
    if pattern == "fixed_per_head":
        c = max(c, l // 64 + 1)
    return pattern, rng.choice(["merged", "merged", "interleaved", "A1", "A2"]), l, c


def draw(rng):
    """One more case of the listed ranges."""
    kind = rng.choice(["tables", "store", "packed", "packed", "decode", "decode"])
    d, dtype = rng.choice([32, 64, 64, 128]), rng.choice(["bf16", "bf16", "bf16", "f32"])
    kv_heads = rng.choice([1, 2, 3, 4, 8])
    heads = kv_heads * rng.choice([1, 1, 2, 4, 8] if kv_heads <= 4 else [1, 1, 2])
    page, mix, ragged = rng.choice([16, 32, 64, 64, 128, 256]), rng.randint(0, 1 << 30), rng.random() < 0.8
    if kind in ("tables", "store"):
        sequences, held = _log(rng, 1, 2000 if kind == "tables" else 200), rng.choice([0, _log(rng, 1, 20000)])
        fresh = rng.choice([1, _log(rng, 1, 12000)])
        while sequences * fresh * (kv_heads * d if kind == "store" else 40) > 60_000_000:
            sequences, fresh = max(1, sequences // 2), max(1, fresh * 2 // 3)
        while sequences * (held + fresh) * (kv_heads * d if kind == "store" else 4) > 400_000_000:
            held = held * 2 // 3
        if kind == "tables":
            return _tables(sequences, held, fresh, page, ragged, mix)
        return _store(sequences, held, fresh, page, ragged, mix, kv_heads, d, dtype)
    if kind == "packed":
        longest, sequences = _log(rng, 1, 40000), rng.choice([1, 2, 3, 5, 8, 17, 40])
        # the plain form forms every pair: no more of them than the largest listed case has
        while heads * sequences * longest * longest > (20_000_000_000 if dtype == "bf16" else 5_000_000_000):
            sequences, longest = max(1, sequences // 2), max(1, longest * 4 // 5)
        pattern, mode, l, c = _pattern(rng, longest)
        return _packed(sequences, longest, ragged, mix, heads, kv_heads, d, dtype, pattern, mode, l, c, rng.random() < 0.5)
    batch, pos = rng.choice([1, 1, 2, 3, 4, 8, 16, 32]), _log(rng, 1, 100000)
    while batch * heads * pos * d > 1_500_000_000:
        batch, pos = max(1, batch // 2), pos * 2 // 3
    pattern, mode, l, c = _pattern(rng, pos)
    return _decode(batch, pos, ragged, mix, heads, kv_heads, d, dtype, pattern, mode, l, c, page)


def _spread(count, longest, ragged, mix, least=0):
    """Lengths of `count` sequences, the longest among them: every size is as likely as its double; now and then none."""
    rng = random.Random(mix)
    if not ragged:
        return [longest] * count
    out = [longest]
    while len(out) < count:
        out.append(least if rng.random() < 0.08 else _log(rng, max(1, longest // 40), longest) if longest else 0)
    rng.shuffle(out)
    return out


def _lengths(case):
    """(held, fresh) of every sequence of a tables or store case, the lengths of a packed one, the positions of a step."""
    kind, ragged, mix = case["kind"], case["ragged"], case["mix"]
    if kind == "packed":
        return _spread(case["sequences"], case["longest"], ragged, mix)
    if kind == "decode":
        return _spread(case["batch"], case["pos"], ragged, mix, -1)
    fresh = _spread(case["sequences"], case["fresh"], ragged and case["fresh"] > 1, mix)
    held = _spread(case["sequences"], case["held"], ragged, mix + 1)
    return held, fresh


def _stride(case):
    """The stride of the pattern; dense causal is the band of a stride that reaches over everything."""
    return case["l"] if case["l"] else max(case.get("longest", 0), case.get("pos", 0), 1) + 1


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _randn(shape, dtype, gen):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _needed(tokens, page):
    return [-(-t // page) for t in tokens]


def _pages(counts, spare, gen, width):
    """A table whose sequences hold `counts` pages of a pool in use, and the pool's free pages, both in no order."""
    total = sum(counts) + spare
    order = torch.randperm(total, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((len(counts), width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for s, n in enumerate(counts):
        table[s, :n] = order[at:at + n]
        at += n
    return table, order[at:].contiguous(), total


def _cache(pages, case, gen, fill):
    """Pages of keys and values, a token's key and value of one head side by side."""
    shape = (pages, case["kv_heads"], case["page"], 2, case["d"])
    if not fill:
        kv = torch.zeros(shape, dtype=DTYPES[case["dtype"]], device="cuda")
    else:
        kv = torch.empty(shape, dtype=DTYPES[case["dtype"]], device="cuda")
        for p in range(0, pages, 4096):
            kv[p:p + 4096] = torch.randn(kv[p:p + 4096].shape, generator=gen, device="cuda")
    return {"k": kv[:, :, :, 0], "v": kv[:, :, :, 1]}


def prepare(case, seed):
    gen, s = _generator(seed), dict(case=case)
    if case["kind"] in ("tables", "store"):
        held, fresh = _lengths(case)
        both = [a + b for a, b in zip(held, fresh)]
        width = max(1, max(_needed(both, case["page"])) + 3)
        mine = _needed(held, case["page"])
        more = sum(_needed(both, case["page"])) - sum(mine)
        s["table"], s["free"], total = _pages(mine, more + 5, gen, width)
        s.update(held=_ints(held), fresh=_ints(fresh), tokens=max(1, sum(fresh) + 7 * (case["mix"] % 2)))
        if case["kind"] == "tables":
            return s
        s.update(_cache(total, case, gen, False))
        slots = _plain_tables(s)[3]  # (a program has them from the tables' operator)
        s["slots"] = slots
        rows = (s["tokens"], case["kv_heads"], case["d"])
        s["new_k"], s["new_v"] = (_randn(rows, DTYPES[case["dtype"]], gen) for _ in range(2))
        return s
    dtype, d, heads, kv = DTYPES[case["dtype"]], case["d"], case["heads"], case["kv_heads"]
    lengths = _lengths(case)
    if case["kind"] == "packed":
        n = max(1, sum(lengths))
        if case["fused"]:
            x = _randn((n, heads + 2 * kv, d), dtype, gen)
            s.update(q=x[:, :heads], k=x[:, heads:heads + kv], v=x[:, heads + kv:])
        else:
            s.update(q=_randn((n, heads, d), dtype, gen), k=_randn((n, kv, d), dtype, gen), v=_randn((n, kv, d), dtype, gen))
        s.update(lengths=lengths, starts=_ints(np.concatenate([[0], np.cumsum(lengths)]).tolist()))
        return s
    s["table"], _, total = _pages(_needed([p + 1 for p in lengths], case["page"]), 2, gen,
                                  -(-(case["pos"] + 1) // case["page"]) + 1)
    s.update(_cache(total, case, gen, True), q=_randn((case["batch"], heads, d), dtype, gen), positions=_ints(lengths))
    return s


# ---------------------------------------------------------------------------
# The passes
# ---------------------------------------------------------------------------
def run(s):
    return {"tables": _run_tables, "store": _run_store, "packed": _run_packed, "decode": _run_decode}[s["case"]["kind"]](s)


def _run_tables(s):
    if own:
        from paper_1904_10509_amd import sparse_attn as sa
        m = sa.page_tables(s["table"], s["held"], s["fresh"], s["free"], s["case"]["page"], s["tokens"])
        return [s["table"], m.starts, m.positions, m.slots, m.last, m.taken]
    return _plain_tables(s)


def _plain_tables(s):
    """Table, first rows, positions and slots of the new tokens (-1 behind the last), last positions, pages taken."""
    table, held, fresh, free, P = s["table"], s["held"].long(), s["fresh"].long(), s["free"], s["case"]["page"]
    tokens, width = s["tokens"], s["table"].shape[1]
    zero = torch.zeros(1, dtype=torch.long, device=table.device)
    starts = torch.cat([zero, torch.cumsum(fresh, 0)])
    had, wants = (held + P - 1) // P, (held + fresh + P - 1) // P
    before = torch.cat([zero, torch.cumsum(wants - had, 0)])
    column = torch.arange(width, device=table.device)[None]
    new = (column >= had[:, None]) & (column < wants[:, None])
    at = before[:-1, None] + column - had[:, None]
    table.copy_(torch.where(new, free[at.clamp(0, max(0, free.shape[0] - 1))], table))
    row = torch.arange(tokens, device=table.device)
    owner = torch.searchsorted(starts[1:], row, right=True)
    live = owner < held.shape[0]
    owner = owner.clamp(max=held.shape[0] - 1)
    place = held[owner] + row - starts[owner]
    slot = table[owner, (place // P).clamp(max=width - 1)].long() * P + place % P
    out = [starts, torch.where(live, place, -1), torch.where(live, slot, -1), held + fresh - 1, before[-1:]]
    return [table] + [x.to(torch.int32) for x in out]


def _run_store(s):
    if own:
        from paper_1904_10509_amd import sparse_attn as sa
        sa.paged_store(sa.PagedCache(s["k"], s["v"]), s["new_k"], s["new_v"], s["slots"])
    else:
        page = s["case"]["page"]
        row = torch.nonzero(s["slots"] >= 0)[:, 0]
        slot = s["slots"][row].long()
        for pages, new in ((s["k"], s["new_k"]), (s["v"], s["new_v"])):
            pages[slot // page, :, slot % page] = new[row]
    return [s["k"], s["v"]]


def _run_packed(s):
    case = s["case"]
    l, c = _stride(case), case["c"]
    if own:
        from paper_1904_10509_amd import sparse_attn as sa
        return list(sa.packed_forward(s["q"], s["k"], s["v"], s["starts"], l, c, PATTERNS[case["pattern"]],
                                      MODES[case["mode"]]))
    heads, group, d = case["heads"], case["heads"] // case["kv_heads"], case["d"]
    o = torch.zeros(s["q"].shape, dtype=s["q"].dtype, device="cuda")
    lse = torch.full((heads, s["q"].shape[0]), float("-inf"), device="cuda")
    first = 0
    for n in s["lengths"]:
        k = s["k"][first:first + n].float().permute(1, 2, 0).contiguous()  # [kv, d, n]
        v = s["v"][first:first + n].float().transpose(0, 1).contiguous()   # [kv, n, d]
        rows = max(1, min(n, (1 << 28) // max(1, heads * n)))
        for r0 in range(0, n, rows):
            r1 = min(n, r0 + rows)
            q = s["q"][first + r0:first + r1].float().transpose(0, 1)      # [heads, rows, d]
            m = r1 - r0
            q = q.reshape(case["kv_heads"], group * m, d)
            score = torch.bmm(q, k[:, :, :r1]).view(heads, m, r1) * (1.0 / math.sqrt(d))
            _hide(score, case, l, r0)
            top = score.amax(dim=-1, keepdim=True)
            top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
            p = torch.exp_(score.sub_(top))
            total = p.sum(dim=-1)
            x = torch.bmm(p.view(case["kv_heads"], group * m, r1), v[:, :r1]).view(heads, m, d)
            x = x / torch.where(total > 0, total, torch.ones_like(total))[..., None]
            o[first + r0:first + r1] = x.transpose(0, 1).to(o.dtype)
            lse[:, first + r0:first + r1] = torch.log(total) + top[..., 0]
        first += n
    return [o, lse]


def _hide(score, case, l, r0):
    """-inf wherever a head's set leaves a pair out; score [heads, rows from r0, keys from 0]."""
    heads, m, n = score.shape
    i = torch.arange(r0, r0 + m, device="cuda", dtype=torch.int32)[:, None]
    j = torch.arange(n, device="cuda", dtype=torch.int32)[None]
    causal, c = j <= i, case["c"]
    strided, per_head = case["pattern"] == "strided", case["pattern"] == "fixed_per_head"
    a1 = causal & (i - j <= l if strided else i // l == j // l)
    sets = {}
    for h in range(heads):
        part = ("A1", "A2")[h % 2] if case["mode"] == "interleaved" else case["mode"]
        sub = h % (l // c) if per_head and part != "A1" else 0
        if (part, sub) not in sets:
            if part == "A1":
                keep = a1
            else:
                w = l - (sub + 1) * c
                keep = causal & ((i - j) % l == 0 if strided else (j % l >= w) & (j % l < w + c))
                keep = keep | a1 if part == "merged" else keep
            sets[part, sub] = ~keep
        score[h].masked_fill_(sets[part, sub], float("-inf"))


def _run_decode(s):
    case = s["case"]
    l, c, d, heads = _stride(case), case["c"], case["d"], case["heads"]
    if own:
        from paper_1904_10509_amd import sparse_attn as sa
        return list(sa.paged_decode(s["q"], sa.PagedCache(s["k"], s["v"]), s["table"], s["positions"], l, c,
                                    PATTERNS[case["pattern"]], MODES[case["mode"]], max_pos=case["pos"]))
    group = heads // case["kv_heads"]
    h = torch.arange(heads, device="cuda")[:, None] // group
    o, lse = torch.empty_like(s["q"]), torch.empty(case["batch"], heads, device="cuda")
    for b in range(case["batch"]):
        at, valid = _keys(case, l, s["positions"][b].long())  # [heads, most]
        page = s["table"][b][at // case["page"]].long().clamp(min=0)
        k = s["k"][page, h, at % case["page"]].float()
        score = (k * s["q"][b].float()[:, None]).sum(-1) * (1.0 / math.sqrt(d))
        score = score.masked_fill(~valid, float("-inf"))
        top = score.amax(dim=-1, keepdim=True)
        top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
        p = torch.exp(score - top)
        total = p.sum(dim=-1)
        v = s["v"][page, h, at % case["page"]].float()
        x = (p[..., None] * v).sum(dim=1) / torch.where(total > 0, total, torch.ones_like(total))[..., None]
        o[b], lse[b] = x.to(o.dtype), torch.log(total) + top[..., 0]
    return [o, lse]


def _keys(case, l, pos):
    """The attended positions of every head of one sequence, each once: [heads, most] and which of them there are."""
    c, heads = case["c"], case["heads"]
    mode, strided = case["mode"], case["pattern"] == "strided"
    h = torch.arange(heads, device="cuda")
    part = torch.where(h % 2 == 0, 0, 1) if mode == "interleaved" else torch.full_like(h, MODES[mode])  # A1, A2 or both
    sub = h % (l // c) if case["pattern"] == "fixed_per_head" else torch.zeros_like(h)
    window = l - (sub + 1) * c if not strided else torch.zeros_like(h)
    most = case["pos"] + 1
    near, far = min(most, l + 1), case["pos"] // l + 1 if strided else (case["pos"] // l + 1) * c
    t = torch.arange({"A1": near, "A2": far, "merged": near + far, "interleaved": max(near, far)}[mode], device="cuda")
    part, window, t = part[:, None], window[:, None], t[None]
    row = pos // l
    lo = (pos - l).clamp(min=0) if strided else row * l
    near = torch.where(part == 1, 0, pos - lo + 1)  # keys of A1, in front
    u = t - near
    if strided:
        far = torch.where(part == 0, 0, torch.where(part == 1, row + 1, (row - 1).clamp(min=0)))
        there = pos - (u + torch.where(part == 1, 0, 2)) * l
    else:
        here = (pos - row * l - window + 1).clamp(min=0, max=c)
        far = torch.where(part == 0, 0, row * c + torch.where(part == 1, here, 0))
        there = u // c * l + window + u % c
    at = torch.where(t < near, lo + t, there)
    valid = (t < near + far) & (pos >= 0)
    return torch.where(valid, at, 0), valid


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------
def _set_sizes(case, l, pos):
    """Attended positions of A1, of A2, and of both together, for an array of positions (sizes do not depend on the
    summary subblock but for A2's own block, which is taken as the last one's)."""
    c = case["c"]
    if case["pattern"] == "strided":
        a1, a2 = np.minimum(pos, l) + 1, pos // l + 1
        return a1, a2, a1 + np.maximum(pos // l - 1, 0)
    a1 = pos % l + 1
    a2 = pos // l * c + np.maximum(0, pos % l - (l - c) + 1)
    return a1, a2, a1 + pos // l * c


def _per_head(case, l, pos):
    """The sum over the heads of the attended positions."""
    a1, a2, both = (int(x.sum()) for x in _set_sizes(case, l, pos))
    heads = case["heads"]
    return {"A1": a1 * heads, "A2": a2 * heads, "merged": both * heads,
            "interleaved": a1 * ((heads + 1) // 2) + a2 * (heads // 2)}[case["mode"]]


def work(case):
    if case["kind"] in ("tables", "store"):
        held, fresh = _lengths(case)
        tokens = sum(fresh)
        if case["kind"] == "store":
            row = case["kv_heads"] * case["d"] * (2 if case["dtype"] == "bf16" else 4)
            return {"bytes": tokens * (4 * row + 4), "flops": 0}
        taken = sum(_needed([a + b for a, b in zip(held, fresh)], case["page"])) - sum(_needed(held, case["page"]))
        return {"bytes": 8 * len(held) + 8 * taken + 8 * len(held) + 8 * tokens, "flops": tokens}
    d, size, heads, kv, l = case["d"], 2 if case["dtype"] == "bf16" else 4, case["heads"], case["kv_heads"], _stride(case)
    if case["kind"] == "packed":
        lengths = _lengths(case)
        pairs = sum(_per_head(case, l, np.arange(n, dtype=np.int64)) for n in lengths if n)
        return {"bytes": sum(lengths) * (2 * (heads + kv) * d * size + 4 * heads), "flops": 4 * d * pairs}
    pos = np.array([p for p in _lengths(case) if p >= 0], dtype=np.int64)
    pairs, group = _per_head(case, l, pos), heads // kv
    a1, a2, both = (int(x.sum()) for x in _set_sizes(case, l, pos))
    reads = pairs // group  # rows that heads share are read once
    if group > 1 and case["mode"] == "interleaved":
        reads = (a1 + a2) * kv
    if group > 1 and case["pattern"] == "fixed_per_head" and case["mode"] != "A1":
        windows = min(l // case["c"], group if case["mode"] != "interleaved" else (group + 1) // 2)
        reads = kv * ((both - a1 if case["mode"] == "merged" else a2) * windows + (0 if case["mode"] == "A2" else a1))
    return {"bytes": reads * 2 * d * size + len(pos) * heads * (2 * d * size + 4), "flops": 4 * d * pairs}


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"tables": _exact_tables, "store": _exact_store, "packed": _exact_packed, "decode": _exact_decode}[case["kind"]](
        case, s)


def _exact_tables(case, s):
    """Sequence by sequence: pages are taken from the front of the free list as they are needed."""
    P, table, free = case["page"], s["table"].cpu().numpy().copy(), s["free"].cpu().numpy()
    held, fresh = s["held"].tolist(), s["fresh"].tolist()
    starts, last, taken, row = [0], [], 0, 0
    positions, slots = np.full(s["tokens"], -1, np.int32), np.full(s["tokens"], -1, np.int32)
    for b in range(len(held)):
        for place in range(-(-held[b] // P), -(-(held[b] + fresh[b]) // P)):
            table[b, place] = free[taken]
            taken += 1
        place = held[b] + np.arange(fresh[b])
        positions[row:row + fresh[b]] = place
        slots[row:row + fresh[b]] = table[b, place // P] * P + place % P
        row += fresh[b]
        starts.append(row)
        last.append(held[b] + fresh[b] - 1)
    out = [table, starts, positions, slots, last, [taken]]
    return [torch.from_numpy(np.asarray(x, dtype=np.int32)).cuda() for x in out]


def _exact_store(case, s):
    """Pages as flat rows: a slot is a row."""
    out = []
    for pages, new in ((s["k"], s["new_k"]), (s["v"], s["new_v"])):
        flat = pages.double().transpose(1, 2).reshape(-1, case["kv_heads"], case["d"])
        there = s["slots"] >= 0
        flat.index_copy_(0, s["slots"][there].long(), new[there].double())
        out.append(flat.view(pages.shape[0], case["page"], case["kv_heads"], case["d"]).transpose(1, 2))
    return out


def _exact_packed(case, s):
    """Head by head; the set by its defining predicate."""
    l, c, d, group = _stride(case), case["c"], case["d"], case["heads"] // case["kv_heads"]
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full((case["heads"], s["q"].shape[0]), float("-inf"), dtype=torch.float64, device="cuda")
    ends = np.cumsum(s["lengths"])
    for end, n in zip(ends.tolist(), s["lengths"]):
        at = torch.arange(n, device="cuda")
        for h in range(case["heads"]):
            q, k, v = (x[end - n:end, g].double() for x, g in ((s["q"], h), (s["k"], h // group), (s["v"], h // group)))
            part = case["mode"] if case["mode"] != "interleaved" else ("A1", "A2")[h % 2]
            step = max(1, (1 << 26) // max(n, 1))
            for r in range(0, n, step):
                i, j = at[r:r + step, None], at[None, :min(n, r + step)]
                if case["pattern"] == "strided":
                    a1, a2 = i - j <= l, torch.remainder(i - j, l) == 0
                else:
                    w = l - c * (1 + (h % (l // c) if case["pattern"] == "fixed_per_head" else 0))
                    a1, a2 = torch.div(i, l, rounding_mode="floor") == torch.div(j, l, rounding_mode="floor"), \
                        (torch.remainder(j, l) >= w) & (torch.remainder(j, l) < w + c)
                keep = (j <= i) & {"A1": a1, "A2": a2, "merged": a1 | a2}[part]
                score = torch.where(keep, q[r:r + step] @ k[:j.shape[1]].t() / math.sqrt(d), -math.inf)
                z = torch.logsumexp(score, 1)
                lse[h, end - n + r:end - n + r + i.shape[0]] = z
                weight = torch.exp(score - torch.where(torch.isinf(z), torch.zeros_like(z), z)[:, None])
                o[end - n + r:end - n + r + i.shape[0], h] = weight @ v[:j.shape[1]]
    return [o, lse]


def _exact_decode(case, s):
    """Every (sequence, head) by itself; the set by its defining predicate."""
    d, l, c, heads = case["d"], _stride(case), case["c"], case["heads"]
    group, P = heads // case["kv_heads"], case["page"]
    o = torch.zeros(case["batch"], heads, d, dtype=torch.float64, device="cuda")
    lse = torch.full((case["batch"], heads), float("-inf"), dtype=torch.float64, device="cuda")
    for b, pos in enumerate(_lengths(case)):
        j = torch.arange(pos + 1, device="cuda") if pos >= 0 else None
        for h in range(heads if pos >= 0 else 0):
            if case["pattern"] == "strided":
                a1, a2 = pos - j <= l, (pos - j) % l == 0
            else:
                w = l - c * (1 + (h % (l // c) if case["pattern"] == "fixed_per_head" else 0))
                a1, a2 = j // l == pos // l, (j % l >= w) & (j % l < w + c)
            mode = case["mode"] if case["mode"] != "interleaved" else ("A1", "A2")[h % 2]
            at = torch.nonzero({"A1": a1, "A2": a2, "merged": a1 | a2}[mode])[:, 0]
            if at.numel() == 0:
                continue
            page, row = s["table"][b, at // P].long(), at % P
            score = s["k"][page, h // group, row].double() @ s["q"][b, h].double() / math.sqrt(d)
            lse[b, h] = torch.logsumexp(score, 0)
            o[b, h] = torch.exp(score - lse[b, h]) @ s["v"][page, h // group, row].double()
    return [o, lse]
