"""The 8-bit cache's store, bit for bit against its definition in 64 bits: codes, scales, and every byte that a call
does not own.  The reference rounds float64 values that are exact (inputs times powers of two), so there is no tolerance."""
import numpy as np
import pytest
import torch

import operator_refs as ref
from paper_1904_10509_amd import sparse_attn as sa

from gpu_util import device, to64

pytestmark = pytest.mark.gpu


def make(shape, dtype, seed, spread=3.0):
    """Values over many magnitudes, zeros among them."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g) * torch.exp2(spread * torch.randn(shape[:-1] + (1,), generator=g))
    return (x * (torch.rand(shape, generator=g) > 0.05)).to(dtype)


def fresh(batch, heads, capacity, d, block, seed=0):
    """A cache in which every byte and scale is known: random codes, scales of exponents -9 .. 3."""
    cache = sa.build_cache8(batch, heads, capacity, d, block, device=device())
    g = torch.Generator().manual_seed(seed)
    for t in (cache.k, cache.v):
        codes = torch.randint(0, 255, t.shape, generator=g, dtype=torch.uint8)
        codes[(codes & 127) == 127] = 5
        t.copy_(codes.to(t.device).view(torch.float8_e4m3fn))
    for t in (cache.k_scale, cache.v_scale):
        t.copy_(torch.exp2(torch.randint(-9, 4, t.shape, generator=g).float()))
    return cache


def state(cache):
    return [cache.k.view(torch.uint8).cpu().numpy().copy(), cache.v.view(torch.uint8).cpu().numpy().copy(),
            cache.k_scale.cpu().numpy().astype(np.float64), cache.v_scale.cpu().numpy().astype(np.float64)]


def store_and_check(cache, k, v, start, counts):
    want = state(cache)
    b, n = k.shape[0], k.shape[2]
    for i, x in enumerate((k, v)):
        ref.store(want[i], want[2 + i], to64(x), [0] * b if start is None else start, [n] * b if counts is None else counts,
                  cache.block)
    dev = cache.k.device
    as_ints = [None if t is None else torch.tensor(t, dtype=torch.int32, device=dev) for t in (start, counts)]
    sa.store8(cache, k.to(dev), v.to(dev), *as_ints)
    torch.cuda.synchronize()
    for got, w, name in zip(state(cache), want, ("k", "v", "k_scale", "v_scale")):
        assert np.array_equal(got, w), (name, np.argwhere(got != w)[:3])


# (batch, heads, capacity, d, block, dtype, n, start, counts): every workgroup shape; one token at a block's first, middle
# and last place; chunks that begin inside blocks and end inside them; lengths of 0 and beyond n; a cache that is full;
# sequences without a place; several blocks of a prompt
CASES = [
    (1, 1, 1, 32, 16, torch.bfloat16, 1, None, None),
    (4, 2, 40, 32, 16, torch.bfloat16, 1, [0, 15, 16, 39], None),
    (3, 3, 100, 64, 32, torch.float32, 1, [31, 40, 99], [1, 1, 0]),
    (3, 2, 300, 64, 64, torch.bfloat16, 150, [0, 37, 130], [150, 1, 149]),
    (2, 1, 200, 128, 64, torch.float32, 77, [63, 64], None),
    (2, 2, 500, 128, 128, torch.bfloat16, 257, [100, -1], [257, 257]),
    (2, 1, 500, 128, 128, torch.float32, 300, [1, 250], [10 ** 6, 200]),
    (2, 2, 70, 32, 128, torch.bfloat16, 90, [0, 65], [60, 90]),
    (3, 1, 64, 64, 16, torch.float32, 20, [60, 64, 2 ** 31 - 1], [20, 20, 20]),
    (2, 2, 96, 32, 32, torch.float32, 33, [-2 ** 31, 5], [33, -7]),
    (1, 5, 1000, 64, 64, torch.bfloat16, 1000, None, None),
]


@pytest.mark.parametrize("batch,heads,capacity,d,block,dtype,n,start,counts", CASES)
def test_store_matches_definition(batch, heads, capacity, d, block, dtype, n, start, counts):
    cache = fresh(batch, heads, capacity, d, block, seed=n)
    k, v = make((batch, heads, n, d), dtype, n + d), make((batch, heads, n, d), dtype, n + d + 1)
    store_and_check(cache, k, v, start, counts)


# 512 blocks and more: K and V by one workgroup, in every shape of it
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d,block", [(32, 16), (64, 16), (64, 32), (64, 64), (128, 64), (128, 128)])
def test_many_blocks(d, block, dtype):
    batch, heads, n = 16, 16, block + 2  # up to three blocks each
    cache = fresh(batch, heads, 3 * block, d, block, seed=d)
    k, v = make((batch, heads, n, d), dtype, d + block), make((batch, heads, n, d), dtype, d + block + 1)
    k[3, 2, 1, 4], v[5, 5, 0, 0] = float("nan"), float("inf")
    store_and_check(cache, k, v, [b * (block // 16) for b in range(batch)], [n - b % 3 for b in range(batch)])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_token_by_token(dtype):
    """Tokens that grow and shrink, one at a time over two blocks: scales only grow inside a block, old codes follow."""
    cache = fresh(2, 2, 40, 64, 32)
    x = make((2, 2, 40, 64), dtype, 8, spread=5.0)
    for i in range(40):
        store_and_check(cache, x[:, :, i:i + 1], -x[:, :, i:i + 1], [i, i], None)
    again = state(cache)
    store_and_check(cache, x[:, :, 39:], -x[:, :, 39:], [39, 39], None)  # the same token once more changes nothing
    assert all(np.array_equal(a, b) for a, b in zip(state(cache), again))


def test_first_store_inside_a_block():
    """A new cache (scales of 0) whose first token lies inside a block: the scale is the new tokens' own."""
    cache = sa.build_cache8(2, 2, 64, 32, 32, device=device())
    cache.k.copy_(torch.full(cache.k.shape, 0x7B, dtype=torch.uint8).view(torch.float8_e4m3fn))  # what was there before
    cache.v.copy_(torch.full(cache.v.shape, 0x7B, dtype=torch.uint8).view(torch.float8_e4m3fn))
    x = make((2, 2, 9, 32), torch.bfloat16, 6)
    sa.store8(cache, x.to(device()), x.to(device()), torch.tensor([5, 30], dtype=torch.int32, device=device()))
    torch.cuda.synchronize()
    for b, start in enumerate((5, 30)):
        for h in range(2):
            for blk in range(start // 32, (start + 8) // 32 + 1):
                r0, r1 = max(start, 32 * blk), min(start + 9, 32 * blk + 32)
                new = to64(x)[b, h, r0 - start:r1 - start]
                e = ref.scale_exponent(np.abs(new).max())
                for codes, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
                    assert float(scale[b, h, blk]) == 2.0 ** e
                    assert np.array_equal(codes[b, h, r0:r1].view(torch.uint8).cpu().numpy(), ref.e4m3_encode(new * 2.0 ** -e))


def test_every_bf16_value():
    """All 65,536 bit patterns: each at the scale of its own row's block (the largest finite ones, subnormals, NaN and
    infinities among them), then all of e4m3's borders at scale 1."""
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    x = bits.reshape(1, 1, 1024, 64)
    store_and_check(fresh(1, 1, 1024, 64, 16), x, x.flip(2), None, None)
    x = x.reshape(4, 4, 64, 64).transpose(0, 2).reshape(1, 1, 1024, 64).contiguous()
    store_and_check(fresh(1, 1, 1024, 64, 32), x, x.flip(3).contiguous(), None, None)
    fine = np.sort(ref.VALUES[np.isfinite(ref.VALUES)])
    mid = (fine[1:] + fine[:-1]) / 2
    x = np.concatenate([mid, mid * (1 + 2.0 ** -20), mid * (1 - 2.0 ** -20), fine, [448.0] * 64])
    x = torch.from_numpy(np.resize(x, 16 * 64)).float().reshape(1, 1, 16, 64)
    store_and_check(fresh(1, 1, 16, 64, 16), x, -x, None, None)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_nonfinite_and_extreme_blocks(dtype):
    cache = fresh(1, 2, 64, 32, 16)
    x = make((1, 2, 64, 32), dtype, 4)
    x[0, 0, 3, 5], x[0, 0, 17], x[0, 1, 20, 1] = float("inf"), float("nan"), -float("inf")
    x[0, 0, 32:48] = 0.0                      # an all-zero block: the least scale
    x[0, 1, 32:48] *= 2.0 ** -120             # below the least scale
    x[0, 1, 48:] = torch.finfo(dtype).max     # the largest magnitude there is
    store_and_check(cache, x, x.flip(2).contiguous(), None, None)
    # a begun block whose scale grows from the least to the largest
    x[0, :, 0] = 3e38
    store_and_check(cache, x[:, :, :1], x[:, :, :1], [40], None)


def test_layouts_strides_and_single_tokens():
    """Keys and values apart, rows with room behind them, tensors cut out of a projection, [b, h, d]: the same codes,
    and no byte beside the rows changes."""
    dev, b, h, d, block, n = device(), 2, 3, 64, 32, 50
    qkv = make((b, n, 3, h, d), torch.bfloat16, 1).to(dev)
    k, v = qkv[:, :, 1].transpose(1, 2), qkv[:, :, 2].transpose(1, 2)
    plain = fresh(b, h, 64, d, block)
    start = torch.tensor([3, 10], dtype=torch.int32, device=dev)
    sa.store8(plain, k.contiguous(), v.contiguous(), start)
    room = [torch.full((b, 64, h, d + 16), 9, dtype=torch.uint8, device=dev) for _ in range(2)]
    apart = sa.Cache8(room[0][..., :d].transpose(1, 2), room[1][..., :d].transpose(1, 2),
                      *(torch.ones(b, h, 2, device=dev) for _ in range(2)), block)
    base = fresh(b, h, 64, d, block)
    for a, t in ((apart.k, base.k), (apart.v, base.v), (apart.k_scale, base.k_scale), (apart.v_scale, base.v_scale)):
        a.copy_(t.view(torch.uint8) if t.element_size() == 1 else t)
    sa.store8(apart, k, v, start)
    torch.cuda.synchronize()
    for got, want in zip(state(apart), state(plain)):
        assert np.array_equal(got, want)
    assert all(torch.all(t[..., d:] == 9) for t in room)
    one, two = fresh(b, h, 64, d, block), fresh(b, h, 64, d, block)
    sa.store8(one, k[:, :, 7], v[:, :, 7], start)
    sa.store8(two, k[:, :, 7:8].contiguous(), v[:, :, 7:8].contiguous(), start)
    assert all(np.array_equal(x, y) for x, y in zip(state(one), state(two)))


def test_offsets_past_32_bits():
    """A cache of 5 GB: rows and new tokens behind 2^31 and 2^32 bytes."""
    dev, d, block, capacity = device(), 128, 128, 20_000_000
    cache = sa.build_cache8(1, 1, capacity, d, block, device=dev)
    x = make((1, 1, 200, d), torch.bfloat16, 3).to(dev)
    for start in (capacity - 200, 2 ** 31 // 256 - 100, 2 ** 32 // 256 - 100):
        sa.store8(cache, x, -x, torch.tensor([start], dtype=torch.int32, device=dev))
        small = fresh(1, 1, 512, d, block)
        at = start % block
        first = start - at
        # the begun block's earlier rows and scale
        for i, (big, little) in enumerate(((cache.k, small.k), (cache.v, small.v))):
            big[:, :, first:start] = little[:, :, :at]
        cache.k_scale[0, 0, first // block] = small.k_scale[0, 0, 0]
        cache.v_scale[0, 0, first // block] = small.v_scale[0, 0, 0]
        sa.store8(cache, x, -x, torch.tensor([start], dtype=torch.int32, device=dev))
        sa.store8(small, x, -x, torch.tensor([at], dtype=torch.int32, device=dev))
        for big, little in ((cache.k, small.k), (cache.v, small.v)):
            assert torch.equal(big[:, :, first:start + 200].view(torch.uint8), little[:, :, :at + 200].view(torch.uint8))
        blocks = (at + 199) // block + 1
        for big, little in ((cache.k_scale, small.k_scale), (cache.v_scale, small.v_scale)):
            assert torch.equal(big[..., first // block:first // block + blocks], little[..., :blocks])
