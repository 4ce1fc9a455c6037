"""Page tables from lengths, and storing into the pages, bit for bit against their definitions."""
import numpy as np
import pytest
import torch

import paged_refs as ref
from paper_1904_10509_amd import sparse_attn as sa

from gpu_util import device

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float32


def ints(x, dev):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=dev)


def check_tables(held, fresh, page, max_pages, tokens, spare=0, seed=0, stride=None):
    dev, rng = device(), np.random.RandomState(seed)
    n = len(held)
    had = [-(-min(max(0, h), max_pages * page) // page) for h in held]
    pool = rng.permutation(sum(had) + 100000)
    want = np.full((n, max_pages), -7)
    at = 0
    for s in range(n):
        want[s, :had[s]] = pool[at:at + had[s]]
        at += had[s]
    needs = sum(min(-(-(max(0, h) + max(0, f)) // page), max_pages) - a for h, f, a in zip(held, fresh, had))
    free = pool[at:at + max(0, needs + spare)]
    table = torch.full((n, stride or max_pages), -7, dtype=torch.int32, device=dev)[:, :max_pages]
    table.copy_(ints(want, dev))
    m = sa.page_tables(table, ints(held, dev), ints(fresh, dev), ints(free, dev), page, tokens)
    torch.cuda.synchronize()
    expect = ref.page_tables(want, held, fresh, free, page, tokens)
    assert np.array_equal(table.cpu().numpy(), want)
    for name, w in zip(("starts", "positions", "slots", "last", "taken"), expect):
        assert np.array_equal(getattr(m, name).cpu().numpy(), w), name
    return m


@pytest.mark.parametrize("sequences", [1, 2, 63, 64, 65, 1000, 1023, 1025, 4097, 8000])
@pytest.mark.parametrize("page", [16, 64])
def test_generating_steps(sequences, page):
    rng = np.random.RandomState(sequences + page)
    held = rng.randint(0, 500, sequences)
    check_tables(held, np.ones(sequences, int), page, 40, sequences, 3, 1)


@pytest.mark.parametrize("sequences,most,page,tokens", [
    (1, 1, 16, 1), (1, 5000, 32, 5000), (3, 700, 16, 2000), (7, 3000, 256, 30000), (300, 900, 128, 100003),
    (2000, 300, 64, 300001), (40, 20000, 64, 500000)])
def test_prompts(sequences, most, page, tokens):
    """Ragged prompts, some empty, some behind held tokens that end inside a page; rows left over are padding."""
    rng = np.random.RandomState(most)
    fresh = rng.randint(0, most + 1, sequences) * (rng.rand(sequences) < 0.9)
    held = rng.randint(0, 300, sequences) * (rng.rand(sequences) < 0.5)
    fresh = fresh * min(1.0, tokens / max(1, fresh.sum()))
    check_tables(held, fresh.astype(int), page, -(-(most + 300) // page), tokens, 5, 2, stride=-(-(most + 300) // page) + 3)


def test_lengths_that_do_not_fit():
    # rows beyond `tokens`, tables that are full, a list that is short, negative lengths
    check_tables([0, 10, 0], [50, 50, 50], 16, 8, 120)
    check_tables([0, 100, 5000, -3], [300, 100, 3, -9], 16, 8, 700)
    check_tables([10, 20, 30], [100, 100, 100], 16, 10, 300, spare=-5)
    check_tables([10, 20, 30], [100, 100, 100], 16, 10, 300, spare=-100)
    check_tables([0, 0], [0, 0], 16, 10, 5)
    check_tables([2 ** 31 - 1] * 3, [2 ** 31 - 1] * 3, 16, 4, 100)


def test_all_sequences_end_at_page_borders():
    check_tables([16, 32, 0, 15, 17, 31], [16, 1, 32, 1, 15, 2], 16, 6, 70)


def test_given_outputs_streams_and_graphs():
    """The outputs that a program keeps, a stream of its own, and a captured step whose lengths the program moves."""
    dev = device()
    n, page, width = 5, 16, 20
    held, fresh = ints([3, 15, 16, 17, 0], dev), ints([1] * n, dev)
    free = torch.arange(100, 200, dtype=torch.int32, device=dev)
    table = torch.arange(n * width, dtype=torch.int32, device=dev).view(n, width)
    other = torch.zeros(4 * n + 3, dtype=torch.int32, device=dev)
    out = sa.PageMap(other[:n + 1], other[n + 1:2 * n + 1], other[2 * n + 1:3 * n + 1], other[3 * n + 1:4 * n + 1],
                     other[4 * n + 1:4 * n + 2])
    versions = [t._version for t in (table, out.slots)]
    side = torch.cuda.Stream(device=dev)
    side.wait_stream(torch.cuda.current_stream(dev))
    assert sa.page_tables(table, held, fresh, free, page, n, out=out, stream=side) is out
    torch.cuda.current_stream(dev).wait_stream(side)
    torch.cuda.synchronize()
    assert [t._version for t in (table, out.slots)] > versions
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sa.page_tables(table, held, fresh, free, page, n, out=out)
    for step in range(20):
        want = table.cpu().numpy().astype(np.int64)
        expect = ref.page_tables(want, held.tolist(), [1] * n, free.tolist(), page, n)
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(table.cpu().numpy(), want)
        for name, w in zip(("starts", "positions", "slots", "last", "taken"), expect):
            assert np.array_equal(getattr(out, name).cpu().numpy(), w), (step, name)
        held += 1
        free += 7
        torch.cuda.synchronize()
    assert other[4 * n + 2] == 0


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d,heads,tokens,page,pages", [
    (32, 1, 1, 16, 1), (64, 8, 33, 64, 3), (128, 3, 1000, 16, 100), (64, 5, 257, 256, 2), (32, 17, 4099, 32, 200)])
def test_store(dtype, d, heads, tokens, page, pages):
    """Every row at its slot and no other byte of the cache moved: interleaved and separate caches, rows of larger
    tensors, padding, slots outside the pool."""
    dev = device()
    g = torch.Generator().manual_seed(d + tokens)
    x = torch.randn((tokens, 3 * heads, d), generator=g).to(dtype).to(dev)
    k, v = x[:, heads:2 * heads], torch.randn((tokens, heads, d), generator=g).to(dtype).to(dev)
    slots = torch.randperm(pages * page, generator=g)[:tokens]
    slots = torch.cat([slots, torch.full((tokens - len(slots),), -1)]).to(torch.int32)
    if tokens > 3:
        slots[1], slots[2], slots[tokens // 2] = pages * page, 2 ** 31 - 1, -5
    inter = sa.build_paged_cache(pages, heads, page, d, dtype, dev)
    plain = sa.PagedCache(*(torch.empty(pages, page, heads, d, dtype=dtype, device=dev).transpose(1, 2) for _ in range(2)))
    for cache in (inter, plain):
        cache.k.fill_(3.0)
        cache.v.fill_(5.0)
        want = [t.clone() for t in (cache.k, cache.v)]
        version = cache.k._version
        sa.paged_store(cache, k, v, slots.to(dev))
        torch.cuda.synchronize()
        assert cache.k._version > version
        for t, s in enumerate(slots.tolist()):
            if 0 <= s < pages * page:
                want[0][s // page, :, s % page], want[1][s // page, :, s % page] = k[t], v[t]
        assert torch.equal(cache.k, want[0]) and torch.equal(cache.v, want[1])


def test_store_keeps_every_bit():
    """Infinities, NaN payloads and subnormals are moved, not computed with."""
    dev = device()
    bits = torch.arange(0, 65536, dtype=torch.int32).to(torch.int16).view(BF).view(1024, 1, 64).to(dev)
    cache = sa.build_paged_cache(8, 1, 128, 64, BF, dev)
    slots = torch.arange(1024, dtype=torch.int32, device=dev)
    sa.paged_store(cache, bits, bits.flip(0), slots)
    torch.cuda.synchronize()
    assert torch.equal(cache.k.reshape(1024, 64).view(torch.int16), bits.view(1024, 64).view(torch.int16))
    assert torch.equal(cache.v.reshape(1024, 64).view(torch.int16), bits.flip(0).view(1024, 64).view(torch.int16))


def test_store_beyond_32_bits():
    """Pages whose addresses pass 4 GiB."""
    dev = device()
    pages, heads, page, d = 36000, 8, 64, 64  # 4.4 GiB of keys, as much of values
    kv = torch.empty((pages, heads, page, 2, d), dtype=BF, device=dev)
    cache = sa.PagedCache(kv[..., 0, :], kv[..., 1, :])
    x = torch.randn((3, heads, d), device=dev).to(BF)
    slots = torch.tensor([pages * page - 1, 64 * 20000 + 5, 0], dtype=torch.int32, device=dev)
    sa.paged_store(cache, x, -x, slots)
    torch.cuda.synchronize()
    for t, s in enumerate(slots.tolist()):
        assert torch.equal(cache.k[s // page, :, s % page], x[t]) and torch.equal(cache.v[s // page, :, s % page], -x[t])


def test_lengths_between_the_rows_of_a_table():
    """Lengths and outputs that lie between a table's rows are no part of it; a call whose `last` is its `held` is
    refused, and nothing is written."""
    dev = device()
    buf = torch.full((4, 32), -9, dtype=torch.int32, device=dev)
    table, held, fresh = buf[:3, :4], buf[0, 4:7], buf[0, 7:10]
    free = buf[1, 4:12]
    out = sa.PageMap(buf[2, 4:8], buf[1, 12:32], buf[3, :20], buf[2, 8:11], buf[2, 11:12])
    held.copy_(ints([5, 16, 0], dev))
    fresh.copy_(ints([12, 3, 2], dev))
    free.copy_(torch.arange(50, 58))
    table.copy_(ints([[40, -9, -9, -9], [41, -9, -9, -9], [-9] * 4], dev))
    want, lengths = table.cpu().numpy().astype(np.int64), [5, 16, 0]
    torch.cuda.synchronize()
    before = buf.clone()
    with pytest.raises(sa.SparseAttnError):
        sa.page_tables(table, held, fresh, free, 16, 20, out=sa.PageMap(out.starts, out.positions, out.slots, held, out.taken))
    torch.cuda.synchronize()
    assert torch.equal(buf, before)
    sa.page_tables(table, held, fresh, free, 16, 20, out=out)
    torch.cuda.synchronize()
    expect = ref.page_tables(want, lengths, [12, 3, 2], list(range(50, 58)), 16, 20)
    assert np.array_equal(table.cpu().numpy(), want) and held.tolist() == lengths
    for name, w in zip(("starts", "positions", "slots", "last", "taken"), expect):
        assert np.array_equal(getattr(out, name).cpu().numpy(), w), name
