"""What the step over an 8-bit cache loses below the result's type."""
import math

import pytest
import torch

from paper_1904_10509_amd import sparse_attn as sa

from gpu_util import device

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
