"""Scores below fp32's range: a key with one has the weight 0, wherever it lies and whatever shares the call."""
import numpy as np
import pytest
import torch

import operator_refs
import paged_refs as ref
from paper_1904_10509_amd import sparse_attn as sa

from gpu_util import device, to64
import test_gpu_packed as packed
import test_gpu_paged_decode as paged

pytestmark = pytest.mark.gpu
S, F = sa.SA_STRIDED, sa.SA_FIXED
A1, A2, MG = sa.SA_MODE_A1, sa.SA_MODE_A2, sa.SA_MODE_MERGED
BF, FP = torch.bfloat16, torch.float32
FAR, AT = 1e30, 9  # element AT of a query, and negated of a lost key: a product of -1e60, beyond fp32
# positions of the lost keys, by sequence: none; those that every wave meets first; all; every other one; all but the last
LOST = [lambda p, n: False, lambda p, n: p < 300, lambda p, n: True, lambda p, n: p % 2 == 0, lambda p, n: p < n - 1]


def check_row(o, lse, q, k, v, keys, dtype, piece):
    """One row in 64 bits over the keys that are left of its set (bounds: paged_refs.bounds, of these keys)."""
    if not len(keys):
        assert lse == -np.inf and np.all(o == 0), (lse, o)
        return
    d = len(q)
    k, v = k[keys], v[keys]
    s = k @ q * d ** -0.5
    want = s.max() + np.log(np.exp(s - s.max()).sum())
    p = np.exp(s - want)
    qk = np.array((np.abs(k) @ np.abs(q)).max() * d ** -0.5)
    o_lim, lse_lim = ref.bounds(p @ v, np.array(want), p @ np.abs(v), qk, np.array(len(keys)), d, paged.LAST[dtype], piece)
    assert abs(lse - want) <= lse_lim, (lse, want)
    assert np.all(np.abs(o - p @ v) <= o_lim), float(np.abs(o - p @ v).max())


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("pattern,mode,l,c", [(S, A1, 1000, 0), (S, MG, 32, 0), (F, MG, 64, 16), (S, A2, 3, 0)])
def test_lost_keys_of_a_step(pattern, mode, l, c, dtype):
    at = [640, 699, 350, 500, 600]
    cache, table, _ = paged.make(at, 2, 700, 64, dtype, 16, l)
    where = table.cpu().numpy()
    q = torch.randn((5, 4, 64), generator=torch.Generator().manual_seed(l)).to(dtype)
    q[..., AT] = FAR
    for b, pos in enumerate(at):
        for p in range(pos + 1):
            cache.k[where[b, p // 16], :, p % 16, AT] = -FAR if LOST[b](p, pos + 1) else 0.0
    k, v = (ref.gather(to64(x), where, 700, 16) for x in (cache.k, cache.v))
    q, positions = q.to(device()), torch.tensor(at, dtype=torch.int32, device=device())
    together = sa.paged_decode(q, cache, table, positions, l, c, pattern, mode)
    alone = [sa.paged_decode(q[b:b + 1], cache, table[b:b + 1], positions[b:b + 1], l, c, pattern, mode) for b in range(5)]
    torch.cuda.synchronize()
    for o, lse in (together, [torch.cat(x) for x in zip(*alone)]):
        o, lse = to64(o), to64(lse)
        for b, pos in enumerate(at):
            for h in range(4):
                keys = operator_refs.attended(pattern, mode, l, c, h, pos)
                keys = keys[[not LOST[b](j, pos + 1) for j in keys]]
                check_row(o[b, h], lse[b, h], to64(q)[b, h], k[b, h // 2], v[b, h // 2], keys, dtype, paged.PIECE[dtype])


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("pattern,mode,l,c", [(S, A1, 1000, 0), (S, MG, 32, 0), (F, MG, 64, 16), (S, A2, 3, 0)])
def test_lost_keys_of_prompts(pattern, mode, l, c, dtype):
    lengths = [100, 330, 90, 130, 70]
    q, k, v, starts = packed.make(lengths, 4, 2, 64, dtype, l)
    at = starts.tolist()
    q[..., AT] = FAR
    for b, n in enumerate(lengths):
        lost = torch.tensor([LOST[b](p, n) for p in range(n)])
        k[at[b]:at[b + 1], :, AT] = torch.where(lost, -FAR, 0.0).to(dtype).to(device())[:, None]
    o, lse = sa.packed_forward(q, k, v, starts, l, c, pattern, mode)
    torch.cuda.synchronize()
    o, lse, q, k, v = (to64(x) for x in (o, lse, q, k, v))
    for b, n in enumerate(lengths):
        rows = slice(at[b], at[b + 1])
        for i in sorted({0, 1, l - 1, l, n // 2, n - 2, n - 1} & set(range(n))):
            for h in range(4):
                keys = operator_refs.attended(pattern, mode, l, c, h, i)
                keys = keys[[not LOST[b](j, n) for j in keys]]
                check_row(o[at[b] + i, h], lse[h, at[b] + i], q[at[b] + i, h], k[rows, h // 2], v[rows, h // 2], keys, dtype,
                          packed.PIECE[dtype])
