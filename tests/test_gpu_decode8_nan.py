"""NaN codes among the attended keys and values (the store keeps a NaN or an infinity as one) and NaN in a query: what the
formula gives.  A NaN score is in the sum of its row, so o and lse are NaN there (-inf is left to rows without a key); a NaN
value reaches its own element of o and no lse; every other row keeps its bits."""
import pytest
import torch

from paper_1904_10509_amd import sparse_attn as sa

from gpu_util import device

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float32
NAN = float("nan")
B, KV, GROUP = 3, 2, 3


def setup(dtype, d, capacity):
    g = torch.Generator().manual_seed(d)
    k, v = (torch.randn((B, KV, capacity, d), generator=g).to(dtype).to(device()) for _ in range(2))
    q = torch.randn((B, KV * GROUP, d), generator=g).to(dtype).to(device())
    return q, k, v


def run(q, k, v, positions):
    cache = sa.build_cache8(B, KV, k.shape[2], k.shape[3], 32, device=device())
    sa.store8(cache, k, v)
    at = torch.tensor(positions, dtype=torch.int32, device=device())
    o, lse = sa.decode8(q, cache, at, k.shape[2] + 1, 0, sa.SA_STRIDED, sa.SA_MODE_A1)
    torch.cuda.synchronize()
    return o, lse


def same_elsewhere(got, want, hit):
    for g, w in zip(got, want):
        assert torch.equal(g[~hit], w[~hit])


# one range of a set, a few, and many; one chunk that is all NaN, the first and the last key of a set
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d,capacity,keys", [(64, 200, [0]), (32, 200, [199]), (128, 40, [39]), (64, 1, [0]),
                                             (64, 1000, [640]), (128, 3000, [2999]), (32, 3000, range(256, 320)),
                                             (64, 300, range(300)), (128, 900, range(900))])
def test_nan_key(dtype, d, capacity, keys):
    q, k, v = setup(dtype, d, capacity)
    at = [capacity - 1] * B
    want = run(q, k, v, at)
    bad = k.clone()
    bad[1, 0, list(keys), 3] = NAN
    o, lse = run(q, bad, v, at)
    hit = torch.zeros(B, KV * GROUP, dtype=torch.bool, device=q.device)
    hit[1, :GROUP] = True  # the heads that read the cache head
    assert torch.isnan(o[hit]).all() and torch.isnan(lse[hit]).all()
    # the block's scale is the largest of the others': the same unless the NaN took the place of the largest
    if len(keys) == 1:
        same_elsewhere((o, lse), want, hit)
    # an infinity is stored as NaN
    bad[1, 0, list(keys), 3] = float("inf")
    o, lse = run(q, bad, v, at)
    assert torch.isnan(o[hit]).all() and torch.isnan(lse[hit]).all()
    # behind the positions nothing reads it
    if keys[0] > 0:
        before = [capacity - 1, keys[0] - 1, capacity - 1]
        o, lse = run(q, bad, v, before)
        assert torch.isfinite(o).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d,capacity,key", [(64, 200, 0), (128, 200, 199), (32, 3000, 1234)])
def test_nan_value(dtype, d, capacity, key):
    q, k, v = setup(dtype, d, capacity)
    at = [capacity - 1] * B
    want = run(q, k, v, at)
    bad = v.clone()
    bad[2, 1, key, 5] = NAN
    o, lse = run(q, k, bad, at)
    hit = torch.zeros_like(o, dtype=torch.bool)
    hit[2, GROUP:, 5] = True
    assert torch.isnan(o[hit]).all() and torch.equal(lse, want[1])
    assert torch.equal(o[~hit], want[0][~hit])


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d,capacity", [(64, 200), (128, 3000)])
def test_nan_query(dtype, d, capacity):
    q, k, v = setup(dtype, d, capacity)
    at = [capacity - 1, -1, 20]
    want = run(q, k, v, at)
    bad = q.clone()
    bad[0, 4, 7] = NAN
    bad[1, 0, 0] = NAN  # a sequence without a query: not read
    got = run(bad, k, v, at)
    hit = torch.zeros(B, KV * GROUP, dtype=torch.bool, device=q.device)
    hit[0, 4] = True
    assert torch.isnan(got[0][hit]).all() and torch.isnan(got[1][hit]).all()
    same_elsewhere(got, want, hit)
    assert torch.all(got[0][1] == 0) and torch.isneginf(got[1][1]).all()
