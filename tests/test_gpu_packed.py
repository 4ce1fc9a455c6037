"""Attention over packed sequences against 64 bits (bounds: paged_refs.bounds; weights rounded once to bf16, 2^-8)."""
import numpy as np
import pytest
import torch

import paged_refs as ref
from paper_1904_10509_amd import sparse_attn as sa

from gpu_util import device, to64

pytestmark = pytest.mark.gpu
S, F, P = sa.SA_STRIDED, sa.SA_FIXED, sa.SA_FIXED_PER_HEAD
A1, A2, MG, IL = sa.SA_MODE_A1, sa.SA_MODE_A2, sa.SA_MODE_MERGED, sa.SA_MODE_INTERLEAVED
BF, FP = torch.bfloat16, torch.float32
LAST = {BF: 2.0 ** -8, FP: 2.0 ** -24}
PIECE = {BF: 2.0 ** -8, FP: 0.0}


def make(lengths, heads, kv_heads, d, dtype, seed, first=0, behind=0, fused=False):
    """q, k, v with `first` rows in front of the sequences and `behind` after them, which hold NaN; starts."""
    dev, g = device(), torch.Generator().manual_seed(seed)
    n = first + sum(lengths) + behind
    x = torch.randn((n, heads + 2 * kv_heads, d), generator=g)
    x[:first] = float("nan")
    x[n - behind:] = float("nan")
    x = x.to(dtype).to(dev)
    parts = [x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:]]
    if not fused:
        parts = [t.contiguous() for t in parts]
    return (*parts, torch.tensor(np.concatenate([[0], np.cumsum(lengths)]) + first, dtype=torch.int32, device=dev))


def check(o, lse, q, k, v, starts, l, c, pattern, mode, scale=None):
    d = q.shape[2]
    at = starts.tolist()
    want, want_lse, pv, qk, count = ref.packed(*(np.nan_to_num(to64(t)) for t in (q, k, v)), at, l, c, pattern, mode,
                                               d ** -0.5 if scale is None else scale)
    o_lim, lse_lim = ref.bounds(want, want_lse.T, pv, qk, count, d, LAST[q.dtype], PIECE[q.dtype])
    lse_lim = lse_lim.T
    o, ls = to64(o), to64(lse)
    rows = slice(at[0], at[-1])
    o, ls, want, want_lse = o[rows], ls[:, rows], want[rows], want_lse[:, rows]
    none = np.isneginf(want_lse)
    assert np.array_equal(np.isneginf(ls), none)
    assert np.all(o[none.T] == 0) and np.all(np.isfinite(o))
    off = np.abs(ls[~none] - want_lse[~none]) - lse_lim[:, rows][~none]
    assert np.all(off <= 0), float(off.max())
    off = np.abs(o - want) - o_lim[rows]
    assert np.all(off <= 0), (float(off.max()), np.argwhere(off > 0)[:4].tolist(), int((off > 0).sum()))


# (pattern, mode, l, c, d, dtype, heads, kv_heads, lengths)
CASES = [
    (S, A1, 5000, 0, 64, BF, 2, 2, [300]),                       # dense causal
    (S, A1, 5000, 0, 128, BF, 8, 1, [1, 63, 64, 65, 0, 200]),
    (S, A1, 5000, 0, 32, FP, 6, 2, [129, 1, 31, 32, 33, 0, 0, 77]),
    (S, A1, 40, 0, 64, BF, 3, 1, [200, 41, 40, 39, 1]),
    (S, A1, 128, 0, 128, FP, 2, 2, [400, 130, 7]),
    (S, A2, 16, 0, 64, BF, 4, 2, [300, 15, 16, 17, 1, 0, 100]),
    (S, A2, 7, 0, 32, BF, 1, 1, [1000]),                         # classes longer than a tile
    (S, A2, 1, 0, 64, FP, 2, 1, [150, 3]),                       # every position
    (S, A2, 3, 0, 128, FP, 4, 4, [260, 2, 1]),
    (S, MG, 16, 0, 64, BF, 4, 4, [300, 31, 32, 33, 34, 0, 1, 100]),
    (S, MG, 5, 0, 32, BF, 8, 4, [700, 9, 10, 11]),
    (S, MG, 1, 0, 64, BF, 2, 2, [200, 2, 3]),
    (S, MG, 31, 0, 128, BF, 6, 2, [500, 1, 62, 63]),
    (S, MG, 20, 0, 64, FP, 3, 3, [333, 40, 41]),
    (S, MG, 200, 0, 64, BF, 2, 2, [390, 20]),                    # no sequence of three strides
    (S, IL, 24, 0, 64, BF, 5, 5, [300, 1, 23, 25]),
    (S, IL, 24, 0, 32, FP, 4, 1, [200, 49]),
    (S, IL, 24, 0, 64, BF, 1, 1, [100]),                         # one head: A1 alone
    (F, A1, 32, 8, 64, BF, 2, 1, [200, 31, 32, 33]),
    (F, A1, 100, 8, 128, FP, 2, 2, [320, 5]),
    (F, A2, 64, 16, 64, BF, 4, 4, [400, 47, 48, 49, 63, 1]),     # rows before the first summary column are empty
    (F, A2, 20, 20, 32, BF, 2, 2, [100, 19]),
    (F, A2, 48, 1, 64, FP, 2, 2, [200, 47]),
    (F, MG, 64, 16, 64, BF, 8, 2, [500, 1, 63, 65, 0, 130]),
    (F, MG, 100, 33, 128, BF, 4, 4, [600, 99, 101]),
    (F, MG, 5, 2, 32, BF, 2, 2, [300, 4, 6]),                    # l-blocks smaller than a tile
    (F, MG, 1, 1, 64, BF, 2, 2, [150]),
    (F, MG, 128, 32, 64, FP, 4, 2, [400, 127, 129]),
    (F, MG, 17, 3, 128, FP, 3, 1, [210]),
    (F, IL, 64, 24, 64, BF, 6, 3, [300, 40]),
    (F, IL, 30, 7, 32, FP, 2, 2, [170, 31]),
    (P, MG, 64, 16, 64, BF, 8, 2, [400, 50, 1]),
    (P, A2, 60, 13, 128, BF, 5, 5, [300, 59]),
    (P, IL, 48, 12, 64, FP, 8, 4, [250, 47]),
    (P, MG, 20, 6, 32, BF, 12, 3, [200, 19, 21]),
    (P, A1, 20, 6, 64, BF, 4, 4, [90]),
]


@pytest.mark.parametrize("pattern,mode,l,c,d,dtype,heads,kv_heads,lengths", CASES)
def test_packed_matches_64_bits(pattern, mode, l, c, d, dtype, heads, kv_heads, lengths):
    fused = (l + d) % 2 == 0
    q, k, v, starts = make(lengths, heads, kv_heads, d, dtype, l + d + c, first=3 * (c % 2), behind=5, fused=fused)
    print(f"packed {pattern} {mode} l={l} c={c} d={d} {dtype} {heads}/{kv_heads} {lengths}", flush=True)
    o, lse = sa.packed_forward(q, k, v, starts, l, c, pattern, mode)
    torch.cuda.synchronize()
    check(o, lse, q, k, v, starts, l, c, pattern, mode)
    again = sa.packed_forward(q, k, v, starts, l, c, pattern, mode)
    at = slice(int(starts[0]), int(starts[-1]))
    assert torch.equal(again[0][at], o[at]) and torch.equal(again[1][:, at], lse[:, at])


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("pattern,mode,l,c", [(S, A1, 10000, 0), (S, MG, 64, 0), (S, A2, 64, 0), (F, MG, 128, 32), (F, A2, 128, 32)])
def test_many_sequences(pattern, mode, l, c, dtype):
    """More sequences than a wave has lanes, and enough tiles for tiles of 128 rows."""
    rng = np.random.RandomState(l)
    lengths = (np.exp(rng.uniform(0, np.log(400), 300)) * (rng.rand(300) < 0.9)).astype(int).tolist()
    q, k, v, starts = make(lengths, 8, 4, 64, dtype, l, behind=9)
    o, lse = sa.packed_forward(q, k, v, starts, l, c, pattern, mode)
    torch.cuda.synchronize()
    check(o, lse, q, k, v, starts, l, c, pattern, mode)


def test_rows_outside_are_left_alone():
    dev = device()
    for mode, l in ((A1, 5000), (MG, 16), (A2, 16)):
        q, k, v, starts = make([70, 0, 200], 2, 1, 64, BF, 3, first=11, behind=40)
        o = torch.full(q.shape, 7.0, dtype=BF, device=dev)
        lse = torch.full((2, q.shape[0]), 9.0, device=dev)
        versions = o._version, lse._version
        got = sa.packed_forward(q, k, v, starts, l, 0, S, mode, out=o, lse=lse)
        torch.cuda.synchronize()
        assert got[0] is o and got[1] is lse and (o._version, lse._version) > versions
        for t in (o[:11], o[281:]):
            assert torch.all(t == 7.0)
        for t in (lse[:, :11], lse[:, 281:]):
            assert torch.all(t == 9.0)
        check(o, lse, q, k, v, starts, l, 0, S, mode)


def test_starts_beyond_the_rows():
    """Values outside 0 .. tokens are the nearest of both; nothing outside the tensors is touched."""
    q, k, v, starts = make([100, 60], 2, 2, 64, BF, 4)
    wide = starts.clone()
    wide[0], wide[2] = -50, 10 ** 9
    for mode, l in ((A1, 5000), (MG, 16)):
        a = sa.packed_forward(q, k, v, starts, l, 0, S, mode)
        b = sa.packed_forward(q, k, v, wide, l, 0, S, mode)
        torch.cuda.synchronize()
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("pattern,mode,l,c", [(S, A1, 5000, 0), (S, A1, 33, 0), (S, A2, 8, 0), (S, MG, 16, 0), (F, MG, 48, 8),
                                              (F, A2, 48, 8), (F, A1, 20, 4)])
def test_infinities_and_nan_reach_what_attends_them_alone(pattern, mode, l, c, dtype):
    lengths = [150, 1, 90]
    q, k, v, starts = make(lengths, 2, 2, 64, dtype, l + c)
    clean = sa.packed_forward(q, k, v, starts, l, c, pattern, mode)
    torch.cuda.synchronize()
    hit = {17: ("k", float("nan")), 60: ("v", float("inf")), 149: ("v", float("nan")), 151 + 80: ("k", float("inf")),
           151 + 3: ("v", float("-inf"))}
    for row, (what, x) in hit.items():
        (k if what == "k" else v)[row, 0, 5] = x
    o, lse = sa.packed_forward(q, k, v, starts, l, c, pattern, mode)
    torch.cuda.synchronize()
    touched = np.zeros(sum(lengths), bool)
    for a, b in zip(starts.tolist()[:-1], starts.tolist()[1:]):
        keep = ref.set_mask(pattern, mode, l, c, 0, b - a)
        for row in hit:
            if a <= row < b:
                touched[a:b] |= keep[:, row - a]
    rest = torch.tensor(~touched, device=o.device)
    # sums that were formed a second time may add in another order: within twice the rounding of the first
    assert torch.isfinite(o[rest]).all()
    assert torch.equal(lse[:, rest], clean[1][:, rest]) and torch.equal(o[:, 1], clean[0][:, 1])
    a, b = o[rest].double(), clean[0][rest].double()
    assert torch.all((a - b).abs() <= 2 * LAST[dtype] * b.abs() + 64 * 2.0 ** -22)
    for row, (what, x) in hit.items():  # the row itself attends its own key in A1 and strided sets
        if what == "k" and np.isinf(x):
            continue  # (an infinite key may score -inf: a weight of 0)
        if pattern == S or mode != A2:
            assert not torch.isfinite(o[row, 0]).all(), row


def test_large_scores():
    """Scores in the hundreds: weights from differences."""
    for dtype in (BF, FP):
        q, k, v, starts = make([300, 50], 2, 2, 64, dtype, 8)
        q = q * 8
        for mode, l in ((A1, 5000), (MG, 16)):
            o, lse = sa.packed_forward(q, k, v, starts, l, 0, S, mode, softmax_scale=1.0)
            torch.cuda.synchronize()
            check(o, lse, q, k, v, starts, l, 0, S, mode, scale=1.0)


def test_streams_workspace_and_graph():
    """A captured call replayed with other inputs and other lengths, a stream of the caller's, a workspace of its own."""
    dev = device()
    q, k, v, starts = make([200, 50, 150], 4, 2, 64, BF, 21)
    need = sa.sparse_attn_packed_workspace_size(400, 16, 0, S, MG, 4, 2, 64, sa.SA_BF16)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device=dev)
    with pytest.raises(sa.SparseAttnError):
        sa.packed_forward(q, k, v, starts, 16, 0, S, MG, workspace=ws[:need - 16])
    want = sa.packed_forward(q, k, v, starts, 16, 0, S, MG)
    side = torch.cuda.Stream(device=dev)
    side.wait_stream(torch.cuda.current_stream(dev))
    o, lse = sa.packed_forward(q, k, v, starts, 16, 0, S, MG, workspace=ws, stream=side)
    torch.cuda.current_stream(dev).wait_stream(side)
    torch.cuda.synchronize()
    assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sa.packed_forward(q, k, v, starts, 16, 0, S, MG, out=o, lse=lse, workspace=ws)
    for rep, cut in enumerate(([0, 200, 250, 400], [0, 0, 399, 400], [0, 100, 100, 400], [0, 1, 2, 400])):
        starts.copy_(torch.tensor(cut, dtype=torch.int32))
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=torch.Generator().manual_seed(rep)).to(BF))
        ws.fill_(0xFF)
        o.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = sa.packed_forward(q, k, v, starts, 16, 0, S, MG)
        torch.cuda.synchronize()
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1]), rep


@pytest.mark.parametrize("pattern,mode,l,c", [(S, MG, 128, 0), (F, MG, 128, 32), (F, A2, 128, 32)])
def test_agrees_with_the_layout_path(pattern, mode, l, c):
    """One sequence of whole blocks: the attention over a layout, within twice the parity bound of each."""
    dev, n = device(), 1024
    q, k, v, starts = make([n], 4, 4, 64, BF, 31)
    layout = sa.build_layout(n, 64, l, c, pattern, mode, device=dev)
    o, lse = sa.forward(*(t.transpose(0, 1)[None].contiguous() for t in (q, k, v)), layout)
    got = sa.packed_forward(q, k, v, starts, l, c, pattern, mode)
    torch.cuda.synchronize()
    assert torch.all((got[0].transpose(0, 1).double() - o[0].double()).abs() <= 4e-2 + 2 * LAST[BF] * o[0].double().abs())
    fine = torch.isfinite(lse[0])
    assert torch.equal(fine, torch.isfinite(got[1])) and torch.all((got[1] - lse[0])[fine].abs() <= 2e-3)
