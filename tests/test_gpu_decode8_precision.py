"""What the step over an 8-bit cache loses below the result's type."""
import math

import numpy as np
import pytest
import torch

from paper_1904_10509_amd import sparse_attn as sa

from gpu_util import device, to64

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float32


def test_small_pieces_of_a_large_score():
    """Two keys whose fp32 scores are both 4,096 + 2^-11, a number of 24 bits: the first key's in two terms, the second's
    as 4,096 and twice 2^-12 from elements (1 + 2^-12) - 1.  Every sum is exact unless halves of the last place are added to
    4,096 one at a time, where each is rounded away; so the weights are equal, and values of 1 and -1 cancel."""
    dev, d = device(), 128
    q = torch.zeros(1, 1, d)
    q[..., 0], q[..., 1] = 4096, 2.0 ** -11
    k = torch.zeros(1, 1, 2, d)
    k[..., 0, 0] = k[..., 0, 1] = k[..., 1, 0] = 1
    for e in (8, 64):
        q[..., e], q[..., e + 1] = 1 + 2.0 ** -12, -1
        k[..., 1, e] = k[..., 1, e + 1] = 1
    v = torch.ones(1, 1, 2, d)
    v[..., 1, :] = -1
    cache = sa.build_cache8(1, 1, 2, d, 16, device=dev)
    sa.store8(cache, k.to(dev), v.to(dev))
    o, lse = sa.decode8(q.to(dev), cache, torch.ones(1, dtype=torch.int32, device=dev), 1, 0, sa.SA_STRIDED, sa.SA_MODE_MERGED,
                        softmax_scale=1.0)
    torch.cuda.synchronize()
    assert torch.all(o == 0)
    # the logarithm is off by 2^-22 of its size (two changes of base)
    assert abs(float(lse) - (4096 + 2.0 ** -11 + math.log(2))) <= 2.0 ** -22 * 4097


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_pieces_of_a_weight(dtype, d):
    """Rows of two keys of weights 1 and w, 1/2 <= w <= 1, whose values nearly cancel in some elements: o = (v - w) / (1 + w), v in
    sixteenths, so that a weight's own rounding is not hidden by the result's.  The scores are one exact product each.  In
    2^-24 of the weight: the exponent's argument, below 1 in size, is rounded three times (log2 e, the scale, the product), 3 ln 2;
    its power is a unit in the last place off, 2; the sums, the reciprocal and the product with it 1 each, 4: 8.1 in
    all.  Weights go in as pieces of bf16 that sum to them, two of them (2^-16) for bf16 results and three (2^-24) for
    fp32; each of that times the sum of p |v|.  The result itself is off by half a step."""
    dev, heads = device(), 96
    g = torch.Generator().manual_seed(d)
    q = torch.zeros(1, heads, d)
    q[0, :, 0] = -torch.rand(heads, generator=g) * math.log(2)
    q = q.to(dtype)
    k, v = torch.zeros(1, 1, 2, d), torch.zeros(1, 1, 2, d)
    k[..., 1, 0] = 1
    v[..., 0, :] = (8 + torch.arange(d) % 8) / 16
    v[..., 1, :] = -1
    cache = sa.build_cache8(1, 1, 2, d, 16, device=dev)
    sa.store8(cache, k.to(dev), v.to(dev))
    o, lse = sa.decode8(q.to(dev), cache, torch.ones(1, dtype=torch.int32, device=dev), 1, 0, sa.SA_STRIDED, sa.SA_MODE_MERGED,
                        softmax_scale=1.0)
    torch.cuda.synchronize()
    w = np.exp(to64(q)[0, :, :1])
    v0 = v[0, 0, 0].double().numpy()[None]
    want, size = (v0 - w) / (1 + w), (v0 + w) / (1 + w)
    piece, last = (2.0 ** -16, 2.0 ** -8) if dtype == BF else (2.0 ** -24, 2.0 ** -24)
    off = np.abs(to64(o)[0] - want)
    assert np.all(off <= (8.1 * 2.0 ** -24 + piece) * size + last * np.abs(want)), float((off / size).max())
    assert np.all(np.abs(to64(lse)[0] - np.log(1 + w[:, 0])) <= 2.0 ** -21)
