"""The precision that rotary's angles, sines and cosines are stated to have, element by element.

Of a pair (1, 0) the result is (cos, sin) itself, of (0, 1) (-sin, cos).  fp32: the angle is off by 2^-28 turns (an eighth of a turn
as a float), 2^-32 (its place in the 64 bits) and |p| times 8.4 units of 2^-64 turns (the frequency), e in all; the sine and
the cosine of it by a unit in the last place, 2^-24 for results below 1: 2 pi e + 2^-24.  Of any pair, S = |x0| + |x1|
times that, and a product and a sum of 2^-24 S each.  bf16: 2^-22 of S, the same two, and half a step of the result, 2^-8."""
from decimal import Decimal, getcontext

import numpy as np
import pytest
import torch

import operator_refs as ref
from paper_1904_10509_amd import sparse_attn as sa

from gpu_util import device, to64

pytestmark = pytest.mark.gpu
ADJ, HALF = sa.SA_ROTARY_ADJACENT, sa.SA_ROTARY_HALVES


def turns(places, dims, base):
    """Turns of every pair, in [-1/2, 1/2), from integers of 128 bits: [tokens, pairs]."""
    getcontext().prec = 60
    out = []
    for a, s in enumerate(dims):
        p = places[:, a].numpy().astype(object)
        for t in range(s // 2):
            unit = int(Decimal(base) ** (Decimal(-2 * t) / Decimal(s)) / (2 * ref.PI) * 2 ** 128)
            fraction = (p * unit) % 2 ** 128 // 2 ** 75  # 53 bits
            out.append(((fraction + 2 ** 52) % 2 ** 53 - 2 ** 52).astype(np.float64) / 2 ** 53)
    return np.stack(out, axis=1)


def some_places(kind, n, axes):
    g = torch.Generator().manual_seed(n)
    ends = {"near": (-5000, 5000), "any": (-2 ** 31, 2 ** 31)}[kind]
    p = torch.randint(*ends, (n, axes), generator=g)
    p[:4, 0] = torch.tensor([0, 1, ends[0], ends[1] - 1])
    return p.to(torch.int32)


CASES = [((128,), 128, 10000.0), ((64,), 64, 1.0001), ((32, 16, 16), 64, 500000.0), ((40, 88), 128, 1.5), ((2,), 32, 10000.0)]


@pytest.mark.parametrize("kind", ["near", "any"])
@pytest.mark.parametrize("pairing", [ADJ, HALF])
@pytest.mark.parametrize("dims,d,base", CASES)
def test_sines_and_cosines(dims, d, base, pairing, kind):
    places = some_places(kind, 1500, len(dims))
    angle = turns(places, dims, base)
    first, second = ref.pair_elements(dims, pairing == HALF)
    x = torch.zeros(1, 2, len(places), d)
    x[:, 0, :, first] = 1
    x[:, 1, :, second] = 1
    far = np.concatenate([np.repeat(np.abs(places[:, a].numpy().astype(np.float64))[:, None], s // 2, 1)
                          for a, s in enumerate(dims)], axis=1)
    lim = 2 * np.pi * (2.0 ** -28 + 2.0 ** -32 + far * 8.4 * 2.0 ** -64) + 2.0 ** -24
    c, s = np.cos(2 * np.pi * angle), np.sin(2 * np.pi * angle)
    for inverse in (False, True):
        y, _ = sa.rotary(x.to(device()), None, places.to(device()), dims, base=base, pairing=pairing, inverse=inverse)
        got, sign = to64(y)[0], -1 if inverse else 1
        for value, want in ((got[0][:, first], c), (got[0][:, second], sign * s), (got[1][:, first], -sign * s),
                            (got[1][:, second], c)):
            off = np.abs(value - want)
            assert np.all(off <= lim), (float(off.max()), float(lim.min()))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pairing", [ADJ, HALF])
@pytest.mark.parametrize("dims,d,base", CASES)
def test_any_pairs(dims, d, base, pairing, dtype):
    places = some_places("near", 700, len(dims))
    x = torch.randn((1, 3, len(places), d), generator=torch.Generator().manual_seed(2)).to(dtype).to(device())
    y, _ = sa.rotary(x, None, places.to(device()), dims, base=base, pairing=pairing)
    want, size = ref.rotary(to64(x), turns(places, dims, base)[None], dims, pairing == HALF)
    if dtype == torch.float32:
        lim = (2 * np.pi * (2.0 ** -28 + 2.0 ** -32 + 2.0 ** -40) + 3 * 2.0 ** -24) * size
    else:
        lim = (2.0 ** -22 + 2 * 2.0 ** -24) * size + 2.0 ** -8 * (np.abs(want) + 2.0 ** -21 * size)
    assert np.all(np.abs(to64(y) - want) <= lim)
