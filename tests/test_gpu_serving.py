"""Page tables, rotary positions, the paged store, the packed attention and the step over pages together, as a serving program
runs them: prompts of different lengths arrive, then every sequence generates; eager, on streams, and as a replayed graph."""
import numpy as np
import pytest
import torch

import paged_refs as ref
from paper_1904_10509_amd import sparse_attn as sa

from gpu_util import device, to64
from test_gpu_packed import check as check_prompts
from test_gpu_paged_decode import check as check_step

pytestmark = pytest.mark.gpu

H, KV, D, PAGE, WIDTH = 8, 2, 64, 16, 24
CAP = PAGE * WIDTH
PROMPTS = [130, 1, 0, 257, 16]
SETS = [(sa.SA_FIXED, sa.SA_MODE_MERGED, 64, 16), (sa.SA_STRIDED, sa.SA_MODE_MERGED, 24, 0), (sa.SA_STRIDED, sa.SA_MODE_A1, 1000, 0)]


def randn(shape, seed, dtype):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).to(device())


class Program:
    """What a serving program keeps: the pool, its free pages, the table, the lengths."""

    def __init__(self, dtype, batch):
        dev = device()
        self.dtype, self.batch, self.pages = dtype, batch, batch * WIDTH
        self.cache = sa.build_paged_cache(self.pages, KV, PAGE, D, dtype, dev)
        self.cache.k.fill_(float("nan"))
        self.cache.v.fill_(float("nan"))
        self.table = torch.full((batch, WIDTH), -1, dtype=torch.int32, device=dev)
        self.free = torch.randperm(self.pages, generator=torch.Generator().manual_seed(7)).to(torch.int32).to(dev)
        self.held = torch.zeros(batch, dtype=torch.int32, device=dev)

    def admit(self, fresh, tokens, stream=None):
        return sa.page_tables(self.table, self.held, fresh, self.free, PAGE, tokens, stream=stream)


def inputs(program, tokens, seed):
    return (randn((tokens, H, D), seed, program.dtype), randn((tokens, KV, D), seed + 1, program.dtype),
            randn((tokens, KV, D), seed + 2, program.dtype))


def turned(q, k, positions, stream=None):
    """Rotary positions of packed rows: one token a sequence, as the operator takes them."""
    return sa.rotary(q, k, positions[:, None], [D], pairing=sa.SA_ROTARY_HALVES, stream=stream)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pattern,mode,l,c", SETS)
def test_prompts_and_generation(pattern, mode, l, c, dtype):
    """Every step's output equals the attention, in 64 bits, over the keys and values that the program has seen."""
    dev, batch = device(), len(PROMPTS)
    p = Program(dtype, batch)
    tokens = sum(PROMPTS) + 6  # a padded batch
    fresh = torch.tensor(PROMPTS, dtype=torch.int32, device=dev)
    m = p.admit(fresh, tokens)
    q, k, v = inputs(p, tokens, 1)
    q, k = turned(q, k, m.positions)
    sa.paged_store(p.cache, k, v, m.slots)
    o, lse = sa.packed_forward(q, k, v, m.starts, l, c, pattern, mode)
    torch.cuda.synchronize()
    check_prompts(o, lse, q, k, v, m.starts, l, c, pattern, mode)
    seen = [np.full((batch, KV, CAP, D), np.nan) for _ in range(2)]
    at = m.starts.tolist()
    for b in range(batch):
        for s, x in zip(seen, (k, v)):
            s[b, :, :PROMPTS[b]] = to64(x[at[b]:at[b + 1]]).transpose(1, 0, 2)
    one = torch.ones(batch, dtype=torch.int32, device=dev)
    for step in range(40):
        p.free = p.free[int(m.taken[0]):]
        p.held = m.last + 1
        m = p.admit(one, batch)
        q, k, v = inputs(p, batch, 100 + 3 * step)
        q, k = turned(q, k, m.positions)
        sa.paged_store(p.cache, k, v, m.slots)
        o, lse = sa.paged_decode(q, p.cache, p.table, m.last, l, c, pattern, mode)
        now = m.last.tolist()
        assert now == [n + step for n in PROMPTS]
        for b, pos in enumerate(now):
            for s, x in zip(seen, (k, v)):
                s[b, :, pos] = to64(x[b])
        if step % 13 == 0 or step == 39:
            torch.cuda.synchronize()
            assert np.array_equal(ref.gather(to64(p.cache.k), p.table.cpu().numpy(), CAP, PAGE)[0, :, :now[0] + 1],
                                  seen[0][0, :, :now[0] + 1])
            check_step(o, lse, q, seen, now, l, c, pattern, mode)


def test_prompt_rows_and_steps_agree():
    """Row i of the packed attention and a step at position i over the stored keys are one result, within both roundings."""
    for pattern, mode, l, c in SETS:
        p = Program(torch.float32, 2)
        lengths = [300, 77]
        fresh = torch.tensor(lengths, dtype=torch.int32, device=device())
        m = p.admit(fresh, 377)
        q, k, v = inputs(p, 377, 5)
        sa.paged_store(p.cache, k, v, m.slots)
        o, lse = sa.packed_forward(q, k, v, m.starts, l, c, pattern, mode)
        for at in ((0, 0), (5, 76), (150, 30), (299, 64)):
            positions = torch.tensor(at, dtype=torch.int32, device=device())
            rows = positions.long() + m.starts[:2].long()
            got, got_lse = sa.paged_decode(q[rows], p.cache, p.table, positions, l, c, pattern, mode)
            torch.cuda.synchronize()
            # each within 2^-18 of sums of |weights| |values| <= 6 (paged_refs.bounds at these sizes)
            assert torch.all((got - o[rows]).abs() <= 2 * 6 * 2.0 ** -18), (pattern, mode, at)
            assert torch.all((got_lse - lse.t()[rows]).abs() <= 2 * 8 * 2.0 ** -18), (pattern, mode, at)


def step(p, q, k, v, one, m, o, lse, ws, sets, stream=None):
    pattern, mode, l, c = sets
    sa.page_tables(p.table, p.held, one, p.free, PAGE, p.batch, out=m, stream=stream)
    qr, kr = turned(q, k, m.positions, stream)
    sa.paged_store(p.cache, kr, v, m.slots, stream=stream)
    sa.paged_decode(qr, p.cache, p.table, m.last, l, c, pattern, mode, max_pos=CAP - 1, out=o, lse=lse, workspace=ws,
                    stream=stream)


@pytest.mark.parametrize("sets", SETS)
def test_replayed_graph_follows_the_lengths(sets):
    """One captured step, replayed while the program moves lengths, list and inputs: the bits of the eager step on a program of
    the same history, with eager work in between."""
    dev, batch = device(), len(PROMPTS)
    programs = [Program(torch.bfloat16, batch) for _ in range(2)]
    fresh = torch.tensor(PROMPTS, dtype=torch.int32, device=dev)
    for p in programs:
        m = p.admit(fresh, sum(PROMPTS))
        q, k, v = inputs(p, sum(PROMPTS), 3)
        sa.paged_store(p.cache, k, v, m.slots)
        p.held.copy_(m.last + 1)
        p.free.copy_(p.free.roll(-int(m.taken[0])))
    one = torch.ones(batch, dtype=torch.int32, device=dev)
    q, k, v = inputs(programs[0], batch, 9)
    outs = []
    pattern, mode, l, c = sets
    need = sa.sparse_attn_paged_decode_workspace_size(CAP - 1, l, c, pattern, mode, batch, H, KV, D, sa.SA_BF16)
    for p in programs:
        x = torch.zeros(4 * batch + 2, dtype=torch.int32, device=dev)
        m = sa.PageMap(x[:batch + 1], x[batch + 1:2 * batch + 1], x[2 * batch + 1:3 * batch + 1], x[3 * batch + 1:4 * batch + 1],
                       x[4 * batch + 1:])
        outs.append((m, torch.empty_like(q), torch.empty(batch, H, device=dev),
                     torch.full((need + 16,), 0xFF, dtype=torch.uint8, device=dev)))
    side = torch.cuda.Stream(device=dev)
    side.wait_stream(torch.cuda.current_stream(dev))
    with torch.cuda.stream(side):
        step(programs[0], q, k, v, one, *outs[0], sets)
    torch.cuda.current_stream(dev).wait_stream(side)
    step(programs[1], q, k, v, one, *outs[1], sets)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(programs[0], q, k, v, one, *outs[0], sets)
    for rep in range(20):
        for p, out in zip(programs, outs):
            p.held.copy_(out[0].last + 1)
            p.free.copy_(p.free.roll(-int(out[0].taken[0])))
        for i, t in enumerate((q, k, v)):
            t.copy_(randn(t.shape, 50 + 3 * rep + i, t.dtype))
        outs[0][1].fill_(float("nan"))
        outs[0][3].fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        step(programs[1], q, k, v, one, *outs[1], sets)
        torch.cuda.synchronize()
        assert torch.equal(programs[0].table, programs[1].table)
        for a, b in zip(outs[0][1:3], outs[1][1:3]):
            assert torch.equal(a, b) and not torch.isnan(a).any(), rep
        assert outs[0][0].last.tolist() == [n + rep + 1 for n in PROMPTS]


def test_two_streams_at_once():
    """Two programs on streams of their own, enqueued in turn without waiting: each gives the bits it gives alone."""
    dev = device()

    def run(p, seed, stream):
        fresh = torch.tensor(PROMPTS, dtype=torch.int32, device=dev)
        q, k, v = inputs(p, sum(PROMPTS), seed)
        torch.cuda.synchronize()
        yield
        m = sa.page_tables(p.table, p.held, fresh, p.free, PAGE, sum(PROMPTS), stream=stream)
        yield
        sa.paged_store(p.cache, k, v, m.slots, stream=stream)
        o, lse = sa.packed_forward(q, k, v, m.starts, 24, 0, sa.SA_STRIDED, sa.SA_MODE_MERGED, stream=stream)
        yield
        d = sa.paged_decode(q[:len(PROMPTS)], p.cache, p.table, m.last, 64, 16, sa.SA_FIXED, sa.SA_MODE_INTERLEAVED, stream=stream)
        yield o, lse, *d

    alone = [list(run(Program(torch.bfloat16, len(PROMPTS)), seed, None))[-1] for seed in (11, 22)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(device=dev) for _ in range(2)]
    both = [run(Program(torch.bfloat16, len(PROMPTS)), seed, s) for seed, s in zip((11, 22), streams)]
    for _ in range(3):
        for g in both:
            next(g)
    got = [next(g) for g in both]
    torch.cuda.synchronize()
    for a, b in zip(alone, got):
        for x, y in zip(a, b):
            assert torch.equal(x, y)
