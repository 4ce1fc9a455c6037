"""Packed attention in tiles of 128 rows, and with keys and values of different layouts (bounds as in test_gpu_packed)."""
import numpy as np
import pytest
import torch

import paged_refs as ref
from paper_1904_10509_amd import sparse_attn as sa

from gpu_util import device
from test_gpu_packed import LAST, check, make

pytestmark = pytest.mark.gpu
S, F, P = sa.SA_STRIDED, sa.SA_FIXED, sa.SA_FIXED_PER_HEAD
A1, A2, MG, IL = sa.SA_MODE_A1, sa.SA_MODE_A2, sa.SA_MODE_MERGED, sa.SA_MODE_INTERLEAVED
BF, FP = torch.bfloat16, torch.float32
SETS = [(S, A1, 5000, 0), (S, A1, 33, 0), (S, A2, 8, 0), (S, MG, 16, 0), (F, MG, 48, 8), (F, A2, 48, 8), (F, A1, 20, 4),
        (P, IL, 64, 16)]


def lengths_of(seed):
    """140 sequences, three long ones among them: with 8 heads, more places of 128 rows than 1,024."""
    rng = np.random.RandomState(seed)
    lengths = rng.randint(0, 40, 140)
    lengths[[3, 80, 139]] = 300, 129, 257
    return lengths.tolist()


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("pattern,mode,l,c", SETS)
def test_wide_tiles_match_64_bits(pattern, mode, l, c, d):
    q, k, v, starts = make(lengths_of(d + l), 8, 2, d, BF, d + l + c, first=1, behind=3)
    o, lse = sa.packed_forward(q, k, v, starts, l, c, pattern, mode)
    torch.cuda.synchronize()
    check(o, lse, q, k, v, starts, l, c, pattern, mode)


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("pattern,mode,l,c", SETS)
def test_nan_reaches_every_row_that_attends_it_and_no_other(pattern, mode, l, c, d):
    """In tiles of 128 rows: NaN among keys and values of the first key head, infinities among its values."""
    lengths = lengths_of(d + l)
    q, k, v, starts = make(lengths, 8, 2, d, BF, d + l + c)
    clean, clean_lse = sa.packed_forward(q, k, v, starts, l, c, pattern, mode)
    torch.cuda.synchronize()
    at = starts.tolist()
    hit = {at[3] + 17: ("k", float("nan")), at[3] + 140: ("v", float("inf")), at[80] + 47: ("v", float("nan")),
           at[139]: ("v", float("nan")), at[139] + 250: ("k", float("nan"))}
    for row, (what, x) in hit.items():
        (k if what == "k" else v)[row, 0, 5] = x
    o, lse = sa.packed_forward(q, k, v, starts, l, c, pattern, mode)
    torch.cuda.synchronize()
    assert torch.equal(o[:, 4:], clean[:, 4:]) and torch.equal(lse[4:], clean_lse[4:])  # the other key head
    bad_o, bad_lse = np.zeros((at[-1], 4, d), bool), np.zeros((4, at[-1]), bool)
    for a, b in zip(at[:-1], at[1:]):
        for h in range(4):
            keep = ref.set_mask(pattern, mode, l, c, h, b - a)
            for row, (what, x) in hit.items():
                if a <= row < b and what == "k":  # the score, and with it everything
                    bad_o[a:b, h] |= keep[:, row - a, None]
                    bad_lse[h, a:b] |= keep[:, row - a]
                elif a <= row < b:
                    bad_o[a:b, h, 5] |= keep[:, row - a]
    bad_o, bad_lse = (torch.tensor(x, device=o.device) for x in (bad_o, bad_lse))
    assert torch.equal(~torch.isfinite(o[:, :4]), bad_o)
    assert torch.equal(torch.isnan(lse[:4]), bad_lse)
    assert torch.equal(lse[:4][~bad_lse], clean_lse[:4][~bad_lse])
    # sums that were formed a second time may add in another order: within twice the rounding of the first
    a, b = o[:, :4][~bad_o].double(), clean[:, :4][~bad_o].double()
    assert torch.all((a - b).abs() <= 2 * LAST[BF] * b.abs() + 64 * 2.0 ** -22)


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("pattern,mode,l,c", [(S, A1, 5000, 0), (S, A1, 200, 0), (S, A2, 3, 0), (S, MG, 5, 0), (F, MG, 128, 32),
                                              (F, MG, 40, 7), (P, A2, 64, 16)])
def test_keys_and_values_of_different_layouts(pattern, mode, l, c, dtype, d):
    """Keys in a tensor of their own, values between the heads of a larger one: steps that take every row's address."""
    q, k, v, starts = make([700, 65, 0, 130], 4, 2, d, dtype, d + l)
    wide = torch.full((v.shape[0], 7, d + 16), float("nan"), dtype=dtype, device=v.device)
    values = wide[:, 3:5, 8:8 + d]
    values.copy_(v)
    o, lse = sa.packed_forward(q, k, values, starts, l, c, pattern, mode)
    torch.cuda.synchronize()
    check(o, lse, q, k, v, starts, l, c, pattern, mode)


@pytest.mark.parametrize("pattern,mode,l,c,n,stride", [
    (S, A2, 256, 0, 256 * 130 + 7, 65536),     # rows of a class 2^24 elements apart
    (S, MG, 256, 0, 256 * 67, 65536),
    (F, MG, 8192, 32, 3 * 8192 + 300, 65536),  # summary columns as far; near keys are not
    (S, A1, 300, 0, 1000, 2 ** 24),            # neighbours
])
def test_rows_that_lie_far_apart(pattern, mode, l, c, n, stride):
    """Rows whose distances pass 32 bits are addressed one by one: the bits of the same call on rows side by side."""
    dev = device()
    g = torch.Generator().manual_seed(l)
    q, k, v = (torch.randn((n, 1, 64), generator=g).to(BF).to(dev) for _ in range(3))
    starts = torch.tensor([0, n], dtype=torch.int32, device=dev)
    want = sa.packed_forward(q, k, v, starts, l, c, pattern, mode)
    far = torch.empty(n * stride, dtype=BF, device=dev)
    fk, fv = far.as_strided((n, 1, 64), (stride, 64, 1)), far.as_strided((n, 1, 64), (stride, 64, 1), 64)
    fk.copy_(k)
    fv.copy_(v)
    o, lse = sa.packed_forward(q, fk, fv, starts, l, c, pattern, mode)
    torch.cuda.synchronize()
    assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
