"""Keys and values of different layouts into the 8-bit cache: keys packed by rotary, values a slice of the projection."""
import pytest
import torch

from paper_1904_10509_amd import sparse_attn as sa

from gpu_util import device
from test_gpu_cache8 import state

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n", [1, 37, 300])
@pytest.mark.parametrize("named", [False, True])
def test_rotated_keys_and_sliced_values(dtype, n, named):
    dev, b, h, d = device(), 3, 2, 64
    qkv = torch.randn((b, n, 3, h, d), generator=torch.Generator().manual_seed(n)).to(dtype).to(dev)
    q, k, v = (qkv[:, :, i].transpose(1, 2) for i in range(3))
    grid = sa.grid_positions((n,), device=dev)
    start = torch.tensor([0, 5, 70], dtype=torch.int32, device=dev)
    caches = [sa.build_cache8(b, h, 400, d, 32, device=dev) for _ in range(3)]
    for c in caches:
        for t in (c.k, c.v):
            t.copy_(torch.zeros(t.shape, dtype=torch.uint8).view(torch.float8_e4m3fn))
    stream = torch.cuda.Stream(device=dev) if named else None
    torch.cuda.synchronize()
    _, packed = sa.rotary(q, k, grid, (d,), out=(torch.empty_like(q).contiguous(), torch.empty(k.shape, dtype=dtype, device=dev)),
                          stream=stream)
    sa.store8(caches[0], packed, v, start, stream=stream)
    torch.cuda.synchronize()
    sa.store8(caches[1], packed, v.contiguous(), start)
    sa.store8(caches[2], v, packed, start, stream=stream)  # either of them
    torch.cuda.synchronize()
    got, want, turned = (state(c) for c in caches)
    for x, y in zip(got, want):
        assert (x == y).all()
    for x, y in zip(turned, (want[1], want[0], want[3], want[2])):
        assert (x == y).all()
    assert want[2].max() > 0
