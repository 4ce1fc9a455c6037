"""Packed sequences in large numbers: every tile finds the sequence that it belongs to (bounds as in test_gpu_packed)."""
import numpy as np
import pytest
import torch

from paper_1904_10509_amd import sparse_attn as sa

from gpu_util import device, to64
from test_gpu_packed import check, make

pytestmark = pytest.mark.gpu
S, F = sa.SA_STRIDED, sa.SA_FIXED
A1, A2, MG = sa.SA_MODE_A1, sa.SA_MODE_A2, sa.SA_MODE_MERGED
BF, FP = torch.bfloat16, torch.float32
SETS = [(S, A1, 1000, 0), (S, MG, 4, 0), (S, A2, 3, 0), (S, A2, 500, 0), (F, MG, 8, 2)]


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("pattern,mode,l,c", SETS)
def test_thousands_of_short_prompts(pattern, mode, l, c, dtype):
    rng = np.random.RandomState(l)
    lengths = rng.randint(0, 6, 5000)
    lengths[[0, 70, 2500, 4999]] = 0, 150, 90, 40
    q, k, v, starts = make(lengths.tolist(), 2, 1, 32, dtype, l, first=2, behind=7)
    o, lse = sa.packed_forward(q, k, v, starts, l, c, pattern, mode)
    torch.cuda.synchronize()
    check(o, lse, q, k, v, starts, l, c, pattern, mode)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("sequences", [1, 63, 64, 65, 127, 128, 129, 4095, 4096, 4097, 8200, 2 ** 20])
def test_prompts_of_one_token(sequences, dtype):
    """Sequences of one token and of none, in no order: a row is its own key alone, so o = v bit for bit (its weight is 1 to
    within 2^-22, which moves no value to a neighbour) and lse its score."""
    dev, rng = device(), np.random.RandomState(sequences)
    lengths = (rng.rand(sequences) < 0.7).astype(np.int64)
    lengths[sequences // 2] = 1
    print(f"one token: {sequences} {dtype}", flush=True)
    starts = torch.tensor(np.concatenate([[0], np.cumsum(lengths)]), dtype=torch.int32, device=dev)
    n = int(lengths.sum())
    g = torch.Generator().manual_seed(sequences)
    q, k, v = (torch.randn((n, 1, 32), generator=g).to(dtype).to(dev) for _ in range(3))
    score = (to64(q) * to64(k)).sum(axis=2).T * 32 ** -0.5
    size = (np.abs(to64(q)) * np.abs(to64(k))).sum(axis=2).T * 32 ** -0.5
    for pattern, mode, l, c in SETS:
        o, lse = sa.packed_forward(q, k, v, starts, l, c, pattern, mode)
        torch.cuda.synchronize()
        if dtype == BF:
            assert torch.equal(o, v)
        else:
            assert torch.all((o - v).abs() <= 2.0 ** -22 * v.abs())
        assert np.all(np.abs(to64(lse) - score) <= (32 + 8) * 2.0 ** -24 * size + 2.0 ** -22 * (np.abs(score) + 1) + 2.0 ** -24)
