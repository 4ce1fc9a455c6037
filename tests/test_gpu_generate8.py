"""Rotary positions, the sparse attention, the 8-bit cache and its decoding step together, as a sampling program runs
them: a prompt, then tokens, sequences of different lengths; eager, on a named stream, and as a replayed graph."""
import numpy as np
import pytest
import torch

import operator_refs as ref
from paper_1904_10509_amd import sparse_attn as sa

from gpu_util import device, to64
from test_gpu_cache8 import state
from test_gpu_decode8 import check as check_step

pytestmark = pytest.mark.gpu

B, H, KV, D, CAP, T = 3, 8, 8, 64, 512, 32
DIMS, L, C = (32, 16, 16), 64, 16
PATTERN, MODE = sa.SA_FIXED, sa.SA_MODE_MERGED


def randn(shape, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).to(device())


def test_prompt_and_generation():
    """Every step's cache equals the definition applied to the turned keys, and its output the attention over that cache."""
    dev, n = device(), 256
    lengths = [256, 130, 1]
    grid = sa.grid_positions((CAP // 64, 8, 8), device=dev)  # [CAP, 3]
    cache = sa.build_cache8(B, KV, CAP, D, T, device=dev)
    cache.k.copy_(torch.zeros_like(cache.k, dtype=torch.uint8).view(torch.float8_e4m3fn))
    cache.v.copy_(torch.zeros_like(cache.v, dtype=torch.uint8).view(torch.float8_e4m3fn))
    cache.k_scale.fill_(1.0)
    cache.v_scale.fill_(1.0)
    want = state(cache)
    # the prompts, padded to one length; the layout's attention takes what the rotary operator made
    q, k, v = (randn((B, H, n, D), 10 + i) for i in range(3))
    q, k = sa.rotary(q, k, grid[:n], DIMS)
    layout = sa.build_layout(n, 32, L, C, PATTERN, MODE, device=dev)
    o, _ = sa.forward(q, k, v, layout)
    assert torch.isfinite(o.float()).all()
    counts = torch.tensor(lengths, dtype=torch.int32, device=dev)
    sa.store8(cache, k, v, None, counts)
    for i, x in enumerate((k, v)):
        ref.store(want[i], want[2 + i], to64(x), [0] * B, lengths, T)
    at = counts.clone()
    for step in range(70):
        places = grid[at.long()]
        q, k, v = (randn((B, H, D), 100 + 3 * step + i) for i in range(3))
        q, k = sa.rotary(q, k, places, DIMS)
        sa.store8(cache, k, v, at)
        o, lse = sa.decode8(q, cache, at, L, C, PATTERN, MODE, max_pos=CAP - 1)
        now = at.tolist()
        for i, x in enumerate((k, v)):
            ref.store(want[i], want[2 + i], to64(x)[:, :, None], now, [1] * B, T)
        if step % 23 == 0 or step == 69:
            torch.cuda.synchronize()
            for got, w in zip(state(cache), want):
                assert np.array_equal(got, w), step
            values = [ref.VALUES[want[i]] * want[2 + i][:, :, np.arange(CAP) // T, None] for i in range(2)]
            check_step(o, lse, q, values, now, L, C, PATTERN, MODE, D ** -0.5)
        at += 1


def steps(cache, at, q, k, v, grid, o, lse, ws, stream=None):
    qr, kr = sa.rotary(q, k, grid[at.long()], DIMS, stream=stream)
    sa.store8(cache, kr, v, at, stream=stream)
    sa.decode8(qr, cache, at, L, C, PATTERN, MODE, max_pos=CAP - 1, out=o, lse=lse, workspace=ws, stream=stream)


def test_replayed_graph_follows_the_positions():
    """One captured step, replayed while the program moves the positions and the inputs: every replay gives the bits of
    the eager step on a cache of the same history, with eager work in between."""
    dev = device()
    grid = sa.grid_positions((CAP // 64, 8, 8), device=dev)
    caches = [sa.build_cache8(B, KV, CAP, D, T, device=dev) for _ in range(2)]
    prompt = [randn((B, KV, 200, D), i) for i in (1, 2)]
    for cache in caches:
        cache.k.copy_(torch.zeros(cache.k.shape, dtype=torch.uint8).view(torch.float8_e4m3fn))
        cache.v.copy_(torch.zeros(cache.v.shape, dtype=torch.uint8).view(torch.float8_e4m3fn))
        cache.k_scale.fill_(1.0)
        cache.v_scale.fill_(1.0)
        sa.store8(cache, *prompt, None, torch.tensor([200, 64, 17], dtype=torch.int32, device=dev))
    at = torch.tensor([200, 64, 17], dtype=torch.int32, device=dev)
    q, k, v = (randn((B, H, D), 5 + i) for i in range(3))
    o, lse = torch.empty_like(q), torch.empty(B, H, device=dev)
    ws = torch.empty(sa.sparse_attn_decode8_workspace_size(CAP - 1, L, C, PATTERN, MODE, B, H, KV, D, sa.SA_BF16) + 16,
                     dtype=torch.uint8, device=dev)
    side = torch.cuda.Stream(device=dev)
    side.wait_stream(torch.cuda.current_stream(dev))
    with torch.cuda.stream(side):
        steps(caches[0], at, q, k, v, grid, o, lse, ws)
    torch.cuda.current_stream(dev).wait_stream(side)
    steps(caches[1], at, q, k, v, grid, torch.empty_like(o), torch.empty_like(lse), None)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        steps(caches[0], at, q, k, v, grid, o, lse, ws)
    for rep in range(6):
        at += 1
        for i, t in enumerate((q, k, v)):
            t.copy_(randn(t.shape, 50 + 3 * rep + i))
        o.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want_o, want_lse = torch.empty_like(o), torch.empty_like(lse)
        steps(caches[1], at, q, k, v, grid, want_o, want_lse, None)
        torch.cuda.synchronize()
        assert torch.equal(o, want_o) and torch.equal(lse, want_lse), rep
        for a, b in zip(state(caches[0]), state(caches[1])):
            assert np.array_equal(a, b)


def test_two_streams_at_once():
    """Two sequences' programs on streams of their own, enqueued in turn without waiting: each gives the bits it gives
    alone.  Named streams allocate their buffers themselves."""
    dev = device()
    grid = sa.grid_positions((CAP // 64, 8, 8), device=dev)
    at = torch.tensor([100, 31, 63], dtype=torch.int32, device=dev)

    def program(seed):
        cache = sa.build_cache8(B, KV, CAP, D, T, device=dev)
        k, v = randn((B, KV, 128, D), seed), randn((B, KV, 128, D), seed + 1)
        tokens = [[randn((B, H, D), seed + 3 * s + i) for i in range(3)] for s in range(4)]
        return cache, k, v, tokens

    def run(p, stream, n):
        cache, k, v, tokens = p
        if n == 0:
            sa.store8(cache, k, v, None, at, stream=stream)
            return None
        q, kk, vv = tokens[n - 1]
        place = at + (n - 1)
        qr, kr = sa.rotary(q, kk, grid[place.long()], DIMS, stream=stream)
        sa.store8(cache, kr, vv, place, stream=stream)
        return sa.decode8(qr, cache, place, L, C, PATTERN, MODE, stream=stream)

    alone = []
    for seed in (1000, 2000):
        p = program(seed)
        alone.append([run(p, None, n) for n in range(5)])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(device=dev) for _ in range(2)]
    programs = [program(1000), program(2000)]
    torch.cuda.synchronize()
    got = [[], []]
    for n in range(5):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(run(programs[i], streams[i] if n % 2 else None, n))
    torch.cuda.synchronize()
    for i in range(2):
        for n in range(1, 5):
            assert torch.equal(got[i][n][0], alone[i][n][0]) and torch.equal(got[i][n][1], alone[i][n][1]), (i, n)


def test_training_step_with_rotary():
    """Rotary and sparse attention under autograd: gradients of q and k are the inverse rotation of the attention's."""
    dev, n = device(), 256
    grid = sa.grid_positions((4, 8, 8), device=dev)
    layout = sa.build_layout(n, 32, L, C, PATTERN, MODE, device=dev)
    q, k, v, w = (randn((2, 4, n, D), 30 + i) for i in range(4))
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    qr, kr = sa.Rotary.apply(leaves[0], leaves[1], grid, DIMS)
    o = sa.SparseAttention.apply(qr, kr, leaves[2], layout)
    grads = torch.autograd.grad(o, leaves, w)
    q1, k1 = sa.rotary(q, k, grid, DIMS)
    o1, lse = sa.forward(q1, k1, v, layout)
    dq, dk, dv = sa.backward(q1, k1, v, o1, w, lse, layout)
    dq, dk = sa.rotary(dq, dk, grid, DIMS, inverse=True)
    assert torch.equal(o, o1)
    for g, want in zip(grads, (dq, dk, dv)):
        assert torch.equal(g, want)
