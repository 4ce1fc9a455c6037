"""Rotary positions of several axes against 64 bits.

Bounds, per element with its pair's |x0| + |x1| = S.  The angle is off by 2^-29 turns, becomes a float (half a step of
2^-25 below half a turn) and its sine and cosine are off by 2^-22 each at most: 2 pi (2^-29 + 2^-26) + 2^-22 = 3.5e-7,
times S; two products and a sum round by 2^-24 of S each, 1.8e-7 S.  6e-7 S in fp32.  For bf16 outputs the sines and
cosines may be off by 2^-14, which S carries into y below the rounding of y itself: 2^-14 S + 2^-8 |y|."""
import numpy as np
import pytest
import torch

import operator_refs as ref
from paper_1904_10509_amd import sparse_attn as sa

from gpu_util import device, to64

pytestmark = pytest.mark.gpu
ADJ, HALF = sa.SA_ROTARY_ADJACENT, sa.SA_ROTARY_HALVES


def bound(y, size, dtype):
    return 6e-7 * size if dtype == torch.float32 else 2.0 ** -14 * size + 2.0 ** -8 * np.abs(y)


def check(got, x, turns, dims, halves, inverse=False):
    y, size = ref.rotary(to64(x), turns, dims, halves, inverse)
    d = np.abs(to64(got) - y) - bound(y, size, got.dtype)
    assert np.all(d <= 0), float(d.max())
    rest = sum(dims)
    assert torch.equal(got[..., rest:], x[..., rest:])


def make(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).to(device())


# (batch, n, heads, k heads, d, axis dims, dtype): W of 8 to 1 pairs a thread, tokens that pass a workgroup's end, all,
# some and few of the elements turned, shared key heads, more key heads than query heads, one token
CASES = [
    (1, 1, 1, 1, 64, (64,), torch.bfloat16), (2, 37, 3, 1, 64, (32, 16, 16), torch.bfloat16),
    (1, 129, 4, 2, 128, (32, 48, 48), torch.bfloat16), (3, 65, 2, 5, 32, (10, 6), torch.bfloat16),
    (2, 50, 8, 8, 64, (28, 28, 8), torch.bfloat16), (1, 300, 2, 2, 128, (2,), torch.bfloat16),
    (2, 33, 3, 3, 64, (20, 20, 20, 4), torch.float32), (1, 70, 16, 2, 128, (64, 64), torch.float32),
    (2, 1, 5, 5, 32, (8, 8, 16), torch.float32), (1, 257, 2, 1, 32, (6, 2, 4), torch.float32),
    (4, 19, 33, 31, 128, (16, 56, 56), torch.bfloat16),
]


@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("batch,n,heads,kv_heads,d,dims,dtype", CASES)
def test_rotary_matches_64_bits(batch, n, heads, kv_heads, d, dims, dtype, halves):
    q, k = make((batch, heads, n, d), dtype, n), make((batch, kv_heads, n, d), dtype, n + 1)
    places = torch.randint(-4000, 4000, (batch, n, len(dims)), generator=torch.Generator().manual_seed(n + 2),
                           dtype=torch.int32)
    turns = np.stack([ref.turn_table(places[b].numpy(), dims, 10000) for b in range(batch)])
    for inverse in (False, True):
        got = sa.rotary(q, k, places.to(q.device), dims, pairing=HALF if halves else ADJ, inverse=inverse)
        for g, x in zip(got, (q, k)):
            check(g, x, turns, dims, halves, inverse)
    # places that the batch shares; q alone
    got, none = sa.rotary(q, None, places[0].to(q.device), dims, pairing=HALF if halves else ADJ)
    assert none is None
    check(got, q, turns[:1], dims, halves)
    again, _ = sa.rotary(q, None, places[:1].to(q.device), dims, pairing=HALF if halves else ADJ)  # [1, n, axes]
    assert torch.equal(again, got)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_far_places_and_other_bases(dtype):
    """The furthest places of int32, both ends: the angle is as exact as at the first ones (reference in 50 digits)."""
    dims = (32, 16, 16)
    places = torch.tensor([[0, 1, -1], [2 ** 31 - 1, -2 ** 31, 1048575], [10 ** 9 + 7, -123456789, 65535]],
                          dtype=torch.int32)
    x = make((2, 2, 3, 64), dtype, 5)
    for base in (10000.0, 500000.0, 1.5):
        got, _ = sa.rotary(x, None, places.to(x.device), dims, base=base)
        check(got, x, ref.turn_table(places.numpy(), dims, base)[None], dims, False)
    got, _ = sa.rotary(x, None, torch.zeros_like(places).to(x.device), dims)
    assert torch.equal(got, x)


@pytest.mark.parametrize("halves", [False, True])
def test_views_in_place_and_single_tokens(halves):
    """q and k cut out of one projection, written into slices of a larger buffer, or over themselves; [b, h, d]; places
    with strides of their own.  All give the bits of the plain call, and nothing beside the outputs changes."""
    dev, pairing, dims = device(), HALF if halves else ADJ, (16, 24)
    qkv = make((2, 21, 3, 4, 64), torch.bfloat16, 9)  # [b, n, qkv, h, d]
    q, k = qkv[:, :, 0].transpose(1, 2), qkv[:, :, 1].transpose(1, 2)
    wide = torch.randint(0, 900, (2, 21, 7), dtype=torch.int32, device=dev)
    places = wide[..., 3:5]
    want = sa.rotary(q.contiguous(), k.contiguous(), places.contiguous(), dims, pairing=pairing)
    for g, w in zip(sa.rotary(q, k, places, dims, pairing=pairing), want):
        assert torch.equal(g, w)
    buf = torch.full((2, 4, 30, 3, 64), 7.0, dtype=torch.bfloat16, device=dev)
    sa.rotary(q, k, places, dims, pairing=pairing, out=(buf[:, :, 2:23, 0], buf[:, :, 2:23, 2]))
    assert torch.equal(buf[:, :, 2:23, 0], want[0]) and torch.equal(buf[:, :, 2:23, 2], want[1])
    assert torch.all(buf[:, :, :, 1] == 7) and torch.all(buf[:, :, :2] == 7) and torch.all(buf[:, :, 23:] == 7)
    own = qkv.clone()
    oq, ok = own[:, :, 0].transpose(1, 2), own[:, :, 1].transpose(1, 2)
    sa.rotary(oq, ok, places, dims, pairing=pairing, out=(oq, ok))
    assert torch.equal(oq, want[0]) and torch.equal(ok, want[1]) and torch.equal(own[:, :, 2], qkv[:, :, 2])
    one = sa.rotary(q[:, :, 5], k[:, :, 5], places[:, 5], dims, pairing=pairing)
    assert torch.equal(one[0], want[0][:, :, 5]) and torch.equal(one[1], want[1][:, :, 5])


def test_nan_and_infinity_stay_in_their_pair():
    dims, x = (16, 16), make((1, 1, 4, 64), torch.float32, 3)
    x[0, 0, 1, 4], x[0, 0, 2, 40] = float("nan"), float("inf")  # a turned pair; an element behind the axes
    places = torch.tensor([[3, 4]] * 4, dtype=torch.int32, device=x.device)
    got = sa.rotary(x, None, places, dims)[0]
    clean = sa.rotary(torch.nan_to_num(x, nan=0.0, posinf=0.0), None, places, dims)[0]
    assert torch.isnan(got[0, 0, 1, 4:6]).all() and got[0, 0, 2, 40] == float("inf")
    same = torch.ones_like(x, dtype=torch.bool)
    same[0, 0, 1, 4:6] = same[0, 0, 2, 40] = False
    assert torch.equal(got[same], clean[same])


@pytest.mark.parametrize("halves", [False, True])
def test_gradients_against_formula_and_differences(halves):
    """dL/dx of L = sum w y: the inverse rotation of w.  y is linear in x, so a difference quotient of any step h is off by
    the roundings of y alone: with |x| <= 1, h = 1 and |w| <= 1 over 64 elements each rounding 6e-7 * 2: 2 * 64 * 1.2e-6."""
    dims, pairing = (16, 24, 8), HALF if halves else ADJ
    q, k = make((2, 3, 5, 64), torch.float32, 1), make((2, 1, 5, 64), torch.float32, 2)
    q, k = q.clamp(-1, 1).requires_grad_(), k.clamp(-1, 1).requires_grad_()
    places = torch.randint(0, 5000, (5, 3), dtype=torch.int32, device=q.device)
    w = [make(q.shape, torch.float32, 3).clamp(-1, 1), make(k.shape, torch.float32, 4).clamp(-1, 1)]
    yq, yk = sa.Rotary.apply(q, k, places, dims, 10000.0, pairing)
    dq, dk = torch.autograd.grad((yq, yk), (q, k), w)
    turns = ref.turn_table(places.cpu().numpy(), dims, 10000)[None]
    check(dq, w[0], turns, dims, halves, inverse=True)
    check(dk, w[1], turns, dims, halves, inverse=True)
    for at in ((0, 2, 1, 0), (1, 0, 4, 17), (1, 1, 2, 47), (0, 0, 0, 60)):
        step = torch.zeros_like(q)
        step[at] = 1.0
        with torch.no_grad():
            up, down = (sa.rotary(q + s * step, k, places, dims, pairing=pairing)[0] for s in (0.5, -0.5))
        slope = float((w[0].double() * (up.double() - down.double())).sum())
        assert abs(slope - float(dq[at])) <= 2 * 64 * 1.2e-6
    # one output unused; a gradient that comes expanded; both unused leaves nothing to do
    yq, yk = sa.Rotary.apply(q, k, places, dims, 10000.0, pairing)
    (dk_alone,) = torch.autograd.grad(yk, (k,), w[1], retain_graph=True)
    assert torch.equal(dk_alone, dk)
    (dq_alone,) = torch.autograd.grad(yq, (q,), w[0], retain_graph=True)
    assert torch.equal(dq_alone, dq)
    (ones,) = torch.autograd.grad(yq.sum(), (q,), retain_graph=True)
    check(ones, torch.ones_like(q), turns, dims, halves, inverse=True)
    # gradients at an odd address, and permuted
    yq, yk = sa.Rotary.apply(q, k, places, dims, 10000.0, pairing)
    odd = [torch.empty(t.numel() + 1, device=t.device)[1:].view(t.shape).copy_(t) for t in w]
    got = torch.autograd.grad((yq, yk), (q, k), odd, retain_graph=True)
    assert torch.equal(got[0], dq) and torch.equal(got[1], dk)
    turned = [t.transpose(1, 2).contiguous().transpose(1, 2) for t in w]
    got = torch.autograd.grad((yq, yk), (q, k), turned, retain_graph=True)
    assert torch.equal(got[0], dq) and torch.equal(got[1], dk)
    # the gradient is linear in w: its own gradient is the rotation
    leaf = w[0].clone().requires_grad_()
    (dq,) = torch.autograd.grad(yq, (q,), leaf, create_graph=True)
    (again,) = torch.autograd.grad(dq, (leaf,), q.detach())
    assert torch.equal(again, yq)


def test_long_sequences_by_slices():
    """Nine million tokens of 128 in pieces of one pair each (2.3 GB a tensor, more workgroups than one grid row holds):
    slices around the borders give the bits of calls of their own."""
    dev, n, d, dims = device(), 9_000_000, 128, (2,)
    x = torch.randn((1, 1, n, d), generator=torch.Generator(device=dev).manual_seed(1), device=dev, dtype=torch.bfloat16)
    places = torch.arange(n, dtype=torch.int32, device=dev)[:, None]
    y, _ = sa.rotary(x, None, places, dims, pairing=HALF)
    for at in (0, 4_194_304 - 50, 8_388_608 - 50, 2 ** 30 // 128 - 50, n - 100):
        part, _ = sa.rotary(x[:, :, at:at + 100].contiguous(), None, places[at:at + 100], dims, pairing=HALF)
        assert torch.equal(y[:, :, at:at + 100], part), at
    assert torch.equal(y[..., 2:], x[..., 2:])
