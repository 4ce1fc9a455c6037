"""The decoding step over an 8-bit cache against 64 bits on the cache's own values.

Bounds.  A score is a sum of d exact products in fp32 (codes times scales and bf16 queries are exact; fp32 queries carry
2^-24), off by e = (d + 8) 2^-24 sum |q||k| scale at most, and so is the log-sum-exp, plus 2^-22 of its own size for the
base-2 units and the logarithm, and count 2^-24 for the sum.  A weight is then off by 2 e + 2^-20 relative (both ends of its
difference; exponentials and rescaling) and the sum by count 2^-24; fp32 outputs may carry their weights in two bf16 pieces
(2^-16), bf16 outputs in one (2^-8), and round themselves (2^-24, 2^-8).  Each times sum p |v|."""
import numpy as np
import pytest
import torch

import operator_refs as ref
from paper_1904_10509_amd import sparse_attn as sa

from gpu_util import device, to64

pytestmark = pytest.mark.gpu
S, F, P = sa.SA_STRIDED, sa.SA_FIXED, sa.SA_FIXED_PER_HEAD
A1, A2, MG, IL = sa.SA_MODE_A1, sa.SA_MODE_A2, sa.SA_MODE_MERGED, sa.SA_MODE_INTERLEAVED
BF, FP = torch.bfloat16, torch.float32


def check(o, lse, q, values, positions, l, c, pattern, mode, scale):
    d = q.shape[-1]
    o_ref, lse_ref, pv, qk, count = ref.decode(to64(q), *values, positions, l, c, pattern, mode, scale)
    e = (d + 8) * 2.0 ** -24 * qk
    o, ls = to64(o), to64(lse)
    none = np.isneginf(lse_ref)
    assert np.array_equal(np.isneginf(ls), none) and np.all(o[none] == 0) and np.all(np.isfinite(o))
    fine = ~none
    lim = e + 2.0 ** -22 * (np.abs(np.where(none, 0, lse_ref)) + 1) + count * 2.0 ** -24
    off = np.abs(ls[fine] - lse_ref[fine]) - lim[fine]
    assert np.all(off <= 0), float(off.max())
    piece, last = (2.0 ** -8, 2.0 ** -8) if q.dtype == BF else (2.0 ** -16, 2.0 ** -24)
    lim = (2 * e + 2.0 ** -20 + 2 * count * 2.0 ** -24 + piece)[..., None] * pv + last * np.abs(o_ref)
    assert np.all(np.abs(o - o_ref) <= lim), float((np.abs(o - o_ref) - lim).max())


def make_cache(batch, kv_heads, capacity, d, block, seed, live):
    """A stored cache whose rows behind each sequence's position hold NaN codes, and scales of unused blocks NaN."""
    g = torch.Generator().manual_seed(seed)
    dev = device()
    cache = sa.build_cache8(batch, kv_heads, capacity, d, block, device=dev)
    cache.k.copy_(torch.full(cache.k.shape, 0x7F, dtype=torch.uint8).view(torch.float8_e4m3fn))
    cache.v.copy_(torch.full(cache.k.shape, 0xFF, dtype=torch.uint8).view(torch.float8_e4m3fn))
    cache.k_scale.fill_(float("nan"))
    cache.v_scale.fill_(float("nan"))
    shape = (batch, kv_heads, capacity, d)
    k, v = (torch.randn(shape, generator=g) * torch.exp2(torch.randn(shape[:3] + (1,), generator=g)) for _ in range(2))
    counts = torch.tensor([max(0, p + 1) for p in live], dtype=torch.int32, device=dev)
    sa.store8(cache, k.to(BF).to(dev), v.to(BF).to(dev), None, counts)
    torch.cuda.synchronize()
    values = []
    for codes, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        at = np.arange(capacity) // block
        with np.errstate(invalid="ignore"):
            values.append(ref.VALUES[codes.view(torch.uint8).cpu().numpy()] * to64(scale)[:, :, at, None])
    return cache, values


def places(capacity, l):
    """First and last positions, block and stride edges, some inside."""
    return sorted({0, 1, l // 2, l - 1, l, l + 1, 2 * l, 3 * l - 1, capacity // 2, capacity - 2, capacity - 1}
                  & set(range(capacity)))


# (pattern, mode, capacity, l, c, d, dtype, heads, kv_heads, scale block)
CASES = [
    (S, MG, 600, 16, 0, 32, FP, 2, 2, 16),
    (S, A2, 600, 16, 0, 64, FP, 3, 1, 32),
    (S, MG, 2048, 128, 0, 64, BF, 4, 4, 64),
    (S, A1, 1000, 100, 0, 64, BF, 4, 2, 128),
    (S, IL, 777, 31, 0, 128, BF, 6, 2, 16),
    (S, MG, 700, 1000, 0, 128, BF, 8, 1, 64),      # dense limit, eight heads of one key head
    (S, MG, 300, 1, 0, 32, BF, 40, 1, 32),         # every position, forty heads of one key head
    (F, MG, 4096, 256, 32, 64, BF, 4, 4, 64),
    (F, A2, 1500, 128, 32, 32, BF, 2, 2, 16),      # empty in the first block
    (F, IL, 1537, 128, 24, 128, BF, 16, 2, 32),
    (F, IL, 900, 96, 40, 64, BF, 3, 1, 64),        # three heads of one key head, alternating
    (F, A1, 900, 96, 40, 64, FP, 2, 1, 128),
    (F, MG, 1100, 48, 48, 128, FP, 20, 4, 64),
    (P, MG, 2048, 128, 32, 64, BF, 8, 2, 64),
    (P, A2, 1500, 128, 32, 64, BF, 5, 5, 32),
    (P, IL, 1000, 48, 12, 128, FP, 16, 2, 16),
    (P, IL, 640, 20, 6, 32, BF, 12, 1, 128),       # three subblocks: sets repeat every six heads
    (P, A1, 500, 20, 6, 32, BF, 12, 3, 16),
    (F, IL, 300, 32, 8, 64, BF, 40, 1, 32),        # forty heads, alternating: two tiles of columns each
    (P, A2, 400, 32, 16, 32, FP, 70, 2, 16),       # thirty-five heads of one key head, two subblocks
]


@pytest.mark.parametrize("pattern,mode,capacity,l,c,d,dtype,heads,kv_heads,block", CASES)
def test_decode8_matches_64_bits(pattern, mode, capacity, l, c, d, dtype, heads, kv_heads, block):
    dev = device()
    at = [-1] + places(capacity, l)  # one sequence per position, and one without
    cache, values = make_cache(len(at), kv_heads, capacity, d, block, capacity + l + d, at)
    q = torch.randn((len(at), heads, d), generator=torch.Generator().manual_seed(l + d)).to(dtype).to(dev)
    positions = torch.tensor(at, dtype=torch.int32, device=dev)
    o, lse = sa.decode8(q, cache, positions, l, c, pattern, mode)
    torch.cuda.synchronize()
    check(o, lse, q, values, at, l, c, pattern, mode, d ** -0.5)
    # repeated: the same bits; with a bound of its own: the same answer
    again = sa.decode8(q, cache, positions, l, c, pattern, mode)
    assert torch.equal(again[0], o) and torch.equal(again[1], lse)
    few = sa.decode8(q, cache, positions, l, c, pattern, mode, max_pos=at[4])
    torch.cuda.synchronize()
    check(few[0][:5], few[1][:5], q[:5], [x[:5] for x in values], at[:5], l, c, pattern, mode, d ** -0.5)
    assert torch.isnan(few[0][5:]).all() and torch.isnan(few[1][5:]).all()  # above the bound


# Launch rules: one range and many, few workgroups and thousands, ranges that do not divide
@pytest.mark.parametrize("batch,heads,kv_heads,d,dtype,keys", [
    (1, 1, 1, 64, BF, 1), (1, 2, 2, 128, FP, 31), (1, 1, 1, 32, BF, 255), (2, 192, 192, 32, FP, 256), (1, 385, 385, 32, BF, 256),
    (1, 192, 192, 32, BF, 257), (1, 1, 1, 64, BF, 5000), (2, 2, 2, 128, BF, 2100), (1, 64, 4, 64, FP, 2100),
    (3, 300, 3, 32, BF, 300), (64, 8, 8, 32, BF, 2100), (64, 16, 16, 32, BF, 2100), (5, 24, 24, 128, FP, 700),
])
def test_launch_rules(batch, heads, kv_heads, d, dtype, keys):
    dev = device()
    at = [keys - 1 - b % 7 if keys > 7 else keys - 1 for b in range(batch)]
    cache, values = make_cache(batch, kv_heads, keys, d, 32, keys + heads, at)
    q = torch.randn((batch, heads, d), generator=torch.Generator().manual_seed(3)).to(dtype).to(dev)
    o, lse = sa.decode8(q, cache, torch.tensor(at, dtype=torch.int32, device=dev), keys + 1, 0, S, A1)
    torch.cuda.synchronize()
    check(o, lse, q, values, at, keys + 1, 0, S, A1, d ** -0.5)


def test_large_and_small_scores():
    """Queries that put all weight on one key, scores far below zero, a zero query: no overflow, no lost maximum."""
    dev, capacity, d = device(), 700, 64
    at = [capacity - 1, 400, 30]
    cache, values = make_cache(3, 2, capacity, d, 32, 5, at)
    for size in (40.0, -40.0, 0.0):
        for dtype in (BF, FP):
            q = (size * torch.randn((3, 2, d), generator=torch.Generator().manual_seed(8))).to(dtype).to(dev)
            o, lse = sa.decode8(q, cache, torch.tensor(at, dtype=torch.int32, device=dev), 50, 0, S, MG, softmax_scale=1.0)
            torch.cuda.synchronize()
            check(o, lse, q, values, at, 50, 0, S, MG, 1.0)


def test_equal_keys_of_large_scores():
    """Keys that are all alike, with scores in the thousands: every weight is the same to the bit, whatever chunk, wave or
    range it falls into, so the output is the mean of the values: off by the sum's own roundings, count 2^-24 of the mean
    |v|, three at the end, and an fp32 weight's third piece (2^-24)."""
    dev, d, capacity = device(), 64, 3000
    cache = sa.build_cache8(1, 1, capacity, d, 64, device=dev)
    k = torch.full((1, 1, capacity, d), 13.0, dtype=BF, device=dev)
    v = torch.randn((1, 1, capacity, d), generator=torch.Generator().manual_seed(1)).to(BF).to(dev)
    sa.store8(cache, k, v)
    q = torch.full((1, 2, d), 5.1, device=dev)
    for pos in (0, 40, 250, 700, 2999):
        o, lse = sa.decode8(q, cache, torch.tensor([pos], dtype=torch.int32, device=dev), 1, 0, S, MG, softmax_scale=1.0)
        torch.cuda.synchronize()
        values = (ref.VALUES[cache.v.view(torch.uint8).cpu().numpy()]
                  * to64(cache.v_scale)[:, :, np.arange(capacity) // 64, None])[0, 0, :pos + 1]
        lim = (pos + 1 + 5) * 2.0 ** -24 * np.abs(values).mean(axis=0)
        assert np.all(np.abs(to64(o) - values.mean(axis=0)) <= lim), pos


def test_layouts_outputs_and_workspace():
    """Keys and values apart in wide rows, query and output views, a caller's workspace: the bits of the plain call."""
    dev, d, l, c = device(), 64, 32, 8
    at = [299, 150]
    cache, _ = make_cache(2, 3, 300, d, 16, 2, at)
    positions = torch.tensor(at, dtype=torch.int32, device=dev)
    q = torch.randn((2, 6, d), generator=torch.Generator().manual_seed(1)).to(BF).to(dev)
    want = sa.decode8(q, cache, positions, l, c, F, MG)
    room = [torch.full((2, 300, 3, d + 32), 0x7F, dtype=torch.uint8, device=dev) for _ in range(2)]
    apart = sa.Cache8(room[0][..., :d].transpose(1, 2), room[1][..., :d].transpose(1, 2), cache.k_scale, cache.v_scale, 16)
    apart.k.copy_(cache.k.view(torch.uint8))
    apart.v.copy_(cache.v.view(torch.uint8))
    wide = torch.zeros(2, 6, 3 * d, dtype=BF, device=dev)
    wide[..., d:2 * d] = q
    out = torch.full((2, 6, 4 * d), 5.0, dtype=BF, device=dev)  # other strides than q's
    lse = torch.empty(2, 6, device=dev)
    need = sa.sparse_attn_decode8_workspace_size(299, l, c, F, MG, 2, 6, 3, d, sa.SA_BF16)
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device=dev)
    sa.decode8(wide[..., d:2 * d], apart, positions, l, c, F, MG, out=out[..., d:2 * d], lse=lse, workspace=ws[:max(need, 16)])
    assert torch.equal(out[..., d:2 * d], want[0]) and torch.equal(lse, want[1])
    same = q[:1].expand(2, 6, d)  # one query for both sequences, a cache that both share: rows of each are read in place
    shared = sa.Cache8(cache.k[:1].expand_as(cache.k), cache.v[:1].expand_as(cache.v), *(
        t[:1].expand_as(t).contiguous() for t in (cache.k_scale, cache.v_scale)), 16)
    got = sa.decode8(same, shared, torch.tensor([at[0]] * 2, dtype=torch.int32, device=dev), l, c, F, MG)
    assert torch.equal(got[0], want[0][:1].expand_as(got[0])) and torch.equal(got[1], want[1][:1].expand_as(got[1]))
    assert torch.all(out[..., :d] == 5) and torch.all(out[..., 2 * d:] == 5) and torch.all(ws[max(need, 16):] == 255)


@pytest.mark.parametrize("exponent", [-100, -7, 0, 3, 100])
def test_every_code(exponent):
    """One key alone: the output is its value, code times scale, to the bit (fp32: the weight is 1), for every finite code;
    with one-hot queries the log-sum-exp is the key's element times the softmax scale, to 2^-20 (two changes of base)."""
    dev, d = device(), 128
    codes = torch.arange(256, dtype=torch.uint8)
    codes[(codes & 127) == 127] = 3  # NaN
    cache = sa.build_cache8(2, 1, 1, d, 16, device=dev)
    for t in (cache.k, cache.v):
        t.copy_(codes.reshape(2, 1, 1, d).view(torch.float8_e4m3fn))
    cache.k_scale.fill_(2.0 ** exponent)
    cache.v_scale.fill_(2.0 ** exponent)
    want = ref.VALUES[codes.numpy()].reshape(2, 1, d) * 2.0 ** exponent
    q = torch.eye(d).expand(2, d, d)
    for dtype in (FP, BF):
        o, lse = sa.decode8(q.to(dtype).to(dev), cache, torch.zeros(2, dtype=torch.int32, device=dev), 1, 0, S, MG,
                            softmax_scale=0.5)
        torch.cuda.synchronize()
        assert np.array_equal(to64(o), np.broadcast_to(want, (2, d, d)))  # four bits: exact in bf16 as well
        assert np.all(np.abs(to64(lse) - 0.5 * want[:, 0]) <= 2.0 ** -20 * np.abs(0.5 * want[:, 0]))


def test_positions_of_any_value():
    """The ends of int32 and the neighbours of the bound, in a batch whose other rows stay as they are."""
    dev, d = device(), 64
    cache, values = make_cache(6, 1, 300, d, 32, 7, [299] * 6)
    q = torch.randn((6, 2, d), generator=torch.Generator().manual_seed(4)).to(BF).to(dev)
    at = [299, -2 ** 31, 280, 281, 2 ** 31 - 1, 0]
    o, lse = sa.decode8(q, cache, torch.tensor(at, dtype=torch.int32, device=dev), 30, 0, S, MG, max_pos=280)
    torch.cuda.synchronize()
    above = torch.tensor([p > 280 for p in at])
    assert torch.isnan(o[above]).all() and torch.isnan(lse[above]).all()
    keep = [i for i, p in enumerate(at) if p <= 280]
    check(o[keep], lse[keep], q[keep], [v[keep] for v in values], [max(at[i], -1) for i in keep], 30, 0, S, MG, d ** -0.5)


def test_offsets_past_32_bits():
    """Positions behind 2^31 and 2^32 bytes of one sequence's cache."""
    dev, d, block, capacity, l = device(), 128, 128, 20_000_000, 70_001
    cache = sa.build_cache8(1, 1, capacity, d, block, device=dev)
    x = torch.randn((1, 1, block, d), generator=torch.Generator().manual_seed(1)).to(BF).to(dev)
    q = torch.randn((1, 2, d), generator=torch.Generator().manual_seed(2)).to(BF).to(dev)
    for pos in (capacity - 1, 2 ** 32 // 256 + 5, 2 ** 31 // 256 + 5):
        keys = np.sort(np.arange(pos, -1, -l))
        for i, j in enumerate(keys):
            sa.store8(cache, x[:, :, i % block:i % block + 1], x[:, :, (7 * i) % block:(7 * i) % block + 1],
                      torch.tensor([j // block * block], dtype=torch.int32, device=dev))
            cache.k[:, :, j], cache.v[:, :, j] = cache.k[:, :, j // block * block], cache.v[:, :, j // block * block]
        o, lse = sa.decode8(q, cache, torch.tensor([pos], dtype=torch.int32, device=dev), l, 0, S, A2)
        torch.cuda.synchronize()
        idx = torch.from_numpy(keys).to(dev)
        values = [ref.VALUES[t[:, :, idx].view(torch.uint8).cpu().numpy()] * to64(s[:, :, idx // block])[..., None]
                  for t, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale))]
        check(o, lse, q, values, [len(keys) - 1], 1, 0, S, A2, d ** -0.5)  # the same keys side by side
