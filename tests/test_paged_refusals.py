"""What the page tables, the paged store, the paged step and the packed attention refuse, before anything is enqueued (no
GPU needed: the pointers are never dereferenced)."""
import ctypes
import os

import pytest

from paper_1904_10509_amd import sparse_attn as sa

FAKE = 0x100000
INV, UNS, SMALL = sa.SA_ERR_INVALID, sa.SA_ERR_UNSUPPORTED, sa.SA_ERR_BUFFER_TOO_SMALL


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(sa.LIB_PATH):
        from paper_1904_10509_amd import build
        build.build()
    return sa.lib()


def longs(*v):
    return (ctypes.c_int64 * len(v))(*v)


TABLES = dict(sequences=4, held=FAKE, fresh=FAKE, page=64, max_pages=10, table=FAKE, table_stride=10, free=FAKE,
              free_count=100, tokens=50, starts=FAKE, positions=FAKE, slots=FAKE, last=FAKE, taken=FAKE, stream=None)


@pytest.mark.parametrize("over,expect", [
    (dict(sequences=0), INV), (dict(sequences=8001), UNS), (dict(held=None), INV), (dict(fresh=None), INV),
    (dict(held=FAKE + 2), INV), (dict(page=48), INV), (dict(page=512), INV), (dict(page=0), INV), (dict(max_pages=0), INV),
    (dict(max_pages=2 ** 26, table_stride=2 ** 26), UNS), (dict(table=None), INV), (dict(table=FAKE + 1), INV),
    (dict(table_stride=9), INV), (dict(table_stride=-10), INV), (dict(free=None), INV), (dict(free_count=-1), INV),
    (dict(free_count=2 ** 31), INV), (dict(tokens=0), INV), (dict(tokens=2 ** 31), INV), (dict(starts=None), INV),
    (dict(positions=None), INV), (dict(slots=FAKE + 3), INV), (dict(last=None), INV), (dict(taken=None), INV),
])
def test_page_tables_refusals(L, over, expect):
    assert L.sparse_attn_page_tables(*dict(TABLES, **over).values()) == expect


STORE = dict(tokens=50, heads=4, d=64, dtype=sa.SA_BF16, k=FAKE, ks=longs(256, 64), v=FAKE, vs=longs(512, 64), slots=FAKE,
             kp=FAKE, vp=FAKE + 128, ps=longs(32768, 8192, 128), pages=10, page=64, stream=None)


@pytest.mark.parametrize("over,expect", [
    (dict(tokens=0), INV), (dict(tokens=2 ** 31), INV), (dict(heads=0), INV), (dict(heads=65536, ps=longs(2 ** 33, 8192, 128)), UNS),
    (dict(d=48), UNS), (dict(dtype=2), INV), (dict(k=None), INV), (dict(v=FAKE + 8), INV), (dict(ks=None), INV),
    (dict(ks=longs(260, 64)), INV), (dict(vs=longs(512, -64)), INV), (dict(slots=None), INV), (dict(slots=FAKE + 2), INV),
    (dict(kp=None), INV), (dict(vp=FAKE + 4), INV), (dict(ps=None), INV), (dict(ps=longs(32768, 8192, 32)), INV),
    (dict(ps=longs(32768, 8192, 132)), INV), (dict(ps=longs(32768, 0, 128)), INV), (dict(ps=longs(0, 8192, 128)), INV),
    (dict(pages=0), INV), (dict(pages=2 ** 31), INV), (dict(pages=2 ** 25), UNS), (dict(page=8), INV),
])
def test_paged_store_refusals(L, over, expect):
    assert L.sparse_attn_paged_store(*dict(STORE, **over).values()) == expect


DECODE = dict(positions=FAKE, max_pos=6000, l=128, c=32, pattern=sa.SA_FIXED, mode=sa.SA_MODE_MERGED, batch=2, heads=8, kv=4,
              d=64, dtype=sa.SA_BF16, q=FAKE, qs=longs(512, 64), kp=FAKE, vp=FAKE + 128, ps=longs(32768, 8192, 128), pages=30,
              page=64, table=FAKE, ts=100, max_pages=100, scale=0.125, o=FAKE, os=longs(512, 64), lse=FAKE, ws=FAKE,
              nbytes=1 << 30, stream=None)


@pytest.mark.parametrize("over,expect", [
    (dict(positions=None), INV), (dict(positions=FAKE + 1), INV), (dict(max_pos=-1), INV), (dict(max_pos=6400), INV),
    (dict(max_pos=2 ** 31), INV), (dict(l=0), INV), (dict(c=0), INV), (dict(c=129), INV), (dict(pattern=3), INV),
    (dict(mode=4), INV), (dict(pattern=sa.SA_FIXED_PER_HEAD, c=1), UNS), (dict(batch=0), INV), (dict(heads=0), INV),
    (dict(kv=3), INV), (dict(kv=0), INV), (dict(batch=2 ** 20), UNS), (dict(d=96), UNS), (dict(dtype=5), INV),
    (dict(q=None), INV), (dict(q=FAKE + 2), INV), (dict(qs=longs(512, 60)), INV), (dict(kp=None), INV), (dict(ps=None), INV),
    (dict(ps=longs(32768, 8192, 32)), INV), (dict(pages=0), INV), (dict(pages=2 ** 30), UNS), (dict(page=24), INV),
    (dict(table=None), INV), (dict(table=FAKE + 2), INV), (dict(ts=99), INV), (dict(ts=-1), INV), (dict(max_pages=0), INV),
    (dict(scale=0.0), INV), (dict(scale=float("nan")), INV), (dict(scale=float("inf")), INV), (dict(o=None), INV),
    (dict(os=longs(512, 0)), INV), (dict(os=longs(0, 64)), INV), (dict(lse=None), INV), (dict(lse=FAKE + 2), INV),
    (dict(ws=None), INV), (dict(ws=FAKE + 8), INV), (dict(nbytes=0), SMALL),
])
def test_paged_decode_refusals(L, over, expect):
    assert L.sparse_attn_paged_decode(*dict(DECODE, **over).values()) == expect


def test_paged_decode_workspace(L):
    args = dict(max_pos=6000, l=128, c=32, pattern=sa.SA_FIXED, mode=sa.SA_MODE_MERGED, batch=2, heads=8, kv=4, d=64,
                dtype=sa.SA_BF16)
    need = sa.sparse_attn_paged_decode_workspace_size(*args.values())
    assert need > 0 and (need - 2 * 8 * 8) % (8 * 66 * 4) == 0  # a state of each head for every range
    assert sa.sparse_attn_paged_decode_workspace_size(*dict(args, max_pos=255).values()) == 0  # one range a sequence
    out = ctypes.c_size_t()
    for over, expect in ((dict(kv=5), INV), (dict(max_pos=-1), INV), (dict(d=16), UNS), (dict(batch=2 ** 20), UNS),
                         (dict(dtype=9), INV)):
        assert L.sparse_attn_paged_decode_workspace_size(*dict(args, **over).values(), ctypes.byref(out)) == expect
    assert L.sparse_attn_paged_decode_workspace_size(*args.values(), None) == INV


PACKED = dict(sequences=3, starts=FAKE, tokens=1000, l=128, c=0, pattern=sa.SA_STRIDED, mode=sa.SA_MODE_MERGED, heads=8, kv=2,
              d=64, dtype=sa.SA_BF16, q=FAKE, qs=longs(768, 64), k=FAKE, ks=longs(768, 64), v=FAKE, vs=longs(768, 64),
              scale=0.125, o=FAKE, os=longs(512, 64), lse=FAKE, ws=FAKE, nbytes=1 << 40, stream=None)


@pytest.mark.parametrize("over,expect", [
    (dict(sequences=0), INV), (dict(sequences=2 ** 20 + 1), UNS), (dict(starts=None), INV), (dict(starts=FAKE + 2), INV),
    (dict(tokens=0), INV), (dict(tokens=2 ** 31 - 1024), UNS), (dict(l=0), INV), (dict(c=8), INV),
    (dict(pattern=sa.SA_FIXED), INV), (dict(pattern=7), INV), (dict(mode=-1), INV),
    (dict(pattern=sa.SA_FIXED_PER_HEAD, c=1), UNS), (dict(heads=0), INV), (dict(heads=65537, kv=1), UNS), (dict(kv=3), INV),
    (dict(kv=0), INV), (dict(d=80), UNS), (dict(dtype=-1), INV), (dict(q=None), INV), (dict(k=None), INV), (dict(v=None), INV),
    (dict(q=FAKE + 8), INV), (dict(k=FAKE + 2), INV), (dict(v=FAKE + 4), INV), (dict(qs=None), INV),
    (dict(ks=longs(764, 64)), INV), (dict(vs=longs(-768, 64)), INV), (dict(o=None), INV), (dict(o=FAKE + 8), INV),
    (dict(os=longs(0, 64)), INV), (dict(os=longs(512, 0)), INV), (dict(os=longs(512, 60)), INV), (dict(lse=None), INV),
    (dict(lse=FAKE + 1), INV), (dict(scale=0.0), INV), (dict(scale=-1.0), INV), (dict(scale=float("nan")), INV),
    (dict(ws=None), INV), (dict(ws=FAKE + 4), INV), (dict(nbytes=100), SMALL),
])
def test_packed_refusals(L, over, expect):
    assert L.sparse_attn_packed_fwd(*dict(PACKED, **over).values()) == expect


def test_packed_workspace(L):
    def need(**over):
        args = dict(tokens=1000, l=128, c=0, pattern=sa.SA_STRIDED, mode=sa.SA_MODE_MERGED, heads=8, kv=2, d=64,
                    dtype=sa.SA_BF16)
        return sa.sparse_attn_packed_workspace_size(*dict(args, **over).values())
    assert need() == 1000 * 8 * 66 * 4
    assert need(l=500) == 0 and need(l=499) > 0  # no sequence has keys beyond the band
    assert need(mode=sa.SA_MODE_A1) == need(mode=sa.SA_MODE_A2) == need(mode=sa.SA_MODE_INTERLEAVED) == 0
    assert need(pattern=sa.SA_FIXED, c=32) == 0
    with pytest.raises(sa.SparseAttnError):
        need(kv=3)


# arguments of a call on 4 sequences of 10 entries 16 apart, 50 rows and a list of 100, each at an address of its own
SPACED = dict(TABLES, held=0x100000, fresh=0x110000, table=0x120000, table_stride=16, free=0x130000, starts=0x140000,
              positions=0x150000, slots=0x160000, last=0x170000, taken=0x180000)


@pytest.mark.parametrize("name,at", [
    ("last", "held"), ("last", "fresh"), ("starts", "held"), ("positions", "fresh"), ("taken", "free"), ("slots", "free"),
    ("positions", "slots"), ("last", "starts"), ("taken", "last"), ("starts", "table"), ("table", "held"), ("table", "free"),
    ("fresh", "table"), ("taken", "positions"),
])
@pytest.mark.parametrize("by", [0, 4, -4])
def test_page_tables_that_overlap(L, name, at, by):
    """An output in an input or in another output, whole or by an element at either end, would be read by one workgroup
    while another writes it."""
    size = dict(held=4, fresh=4, table=3 * 16 + 10, free=100, starts=5, positions=50, slots=50, last=4, taken=1)
    places = {SPACED[at] + by if by >= 0 else SPACED[at] - 4 * (size[name] - 1),  # its start, or its last element there
              SPACED[at] + 4 * (size[at] - 1)}                                    # its first element on the other's last
    for place in places:
        if by == 4 and size[at] == 1:
            continue
        assert L.sparse_attn_page_tables(*dict(SPACED, **{name: place}).values()) == INV, hex(place)


@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("mode", [sa.SA_MODE_MERGED, sa.SA_MODE_A1])
def test_packed_output_in_an_input(L, which, mode):
    args = dict(PACKED, mode=mode, q=0x300000, k=0x400000, v=0x500000, o=0x200000)
    assert L.sparse_attn_packed_fwd(*dict(args, **{which: args["o"]}).values()) == INV
