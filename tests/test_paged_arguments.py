"""What the binding takes and refuses around packed sequences and the cache in pages, without a GPU: the launches are recorded in
place of being made."""
import contextlib

import pytest
import torch

from paper_1904_10509_amd import sparse_attn as sa
from test_operator_arguments import OnGpu, gpu

PAGES, KV, PAGE, D, B, H, N = 12, 2, 16, 64, 3, 4, 20


class Library:
    """Records the calls by name; workspaces are of 4,096 bytes."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            if name.endswith("workspace_size"):
                args[-1]._obj.value = 4096
            else:
                self.calls.append((name, args))
            return sa.SA_OK
        return call


@pytest.fixture
def library(monkeypatch):
    got = Library()
    monkeypatch.setattr(sa, "lib", lambda: got)
    monkeypatch.setattr(sa, "_here", lambda device, stream: contextlib.nullcontext())
    monkeypatch.setattr(sa, "_stream", lambda stream, device: 0)
    return got


def ints(*shape):
    return gpu(*shape, dtype=torch.int32)


def cache(dtype=torch.bfloat16):
    c = sa.build_paged_cache(PAGES, KV, PAGE, D, dtype, device="cpu")
    return sa.PagedCache(*(t.as_subclass(OnGpu) for t in (c.k, c.v)))


def tables(**over):
    args = dict(table=ints(B, 4), held=ints(B), fresh=ints(B), free=ints(9), page=PAGE, tokens=N)
    args.update(over)
    return sa.page_tables(**args)


def packed(**over):
    args = dict(q=gpu(N, H, D), k=gpu(N, KV, D), v=gpu(N, KV, D), starts=ints(B + 1), stride_l=16, summary_c=0,
                pattern=sa.SA_STRIDED, head_mode=sa.SA_MODE_MERGED)
    args.update(over)
    return sa.packed_forward(**args)


def decode(**over):
    args = dict(q=gpu(B, H, D), cache=cache(), table=ints(B, 4), positions=ints(B), stride_l=16, summary_c=0,
                pattern=sa.SA_STRIDED, head_mode=sa.SA_MODE_MERGED)
    args.update(over)
    return sa.paged_decode(**args)


def store(**over):
    args = dict(cache=cache(), k=gpu(N, KV, D), v=gpu(N, KV, D), slots=ints(N))
    args.update(over)
    return sa.paged_store(**args)


def test_calls_as_documented(library):
    m = tables()
    assert (m.starts.shape, m.positions.shape, m.slots.shape, m.last.shape, m.taken.shape) == ((B + 1,), (N,), (N,), (B,), (1,))
    o, lse = packed()
    assert o.shape == (N, H, D) and lse.shape == (H, N) and lse.dtype == torch.float32
    o, lse = decode()
    assert o.shape == (B, H, D) and lse.shape == (B, H)
    store()
    assert [name for name, _ in library.calls] == ["sparse_attn_page_tables", "sparse_attn_packed_fwd",
                                                   "sparse_attn_paged_decode", "sparse_attn_paged_store"]
    # the bound of a step is the table's last position
    assert library.calls[2][1][1] == 4 * PAGE - 1


def test_dimensions_of_one_element_have_any_stride(library):
    """A single token or head is never stepped over: what torch says of its stride does not matter."""
    x = torch.zeros(1, H, D, dtype=torch.bfloat16).as_strided((1, H, D), (3, D, 1)).as_subclass(OnGpu)
    y = torch.zeros(1, 1, D, dtype=torch.bfloat16).as_strided((1, 1, D), (1, 7, 1)).as_subclass(OnGpu)
    packed(q=x, k=y, v=y, starts=ints(2))
    args = library.calls[-1][1]
    for strides in (args[12], args[14], args[16]):
        assert all(s % 8 == 0 for s in strides)


def test_written_tensors_are_reported(library):
    table, out, lse = ints(B, 4), gpu(N, H, D), gpu(H, N, dtype=torch.float32)
    c = cache()
    before = [t._version for t in (table, out, lse, c.k, c.v)]
    tables(table=table)
    packed(out=out, lse=lse)
    store(cache=c)
    assert all(t._version > v for t, v in zip((table, out, lse, c.k, c.v), before))


@pytest.mark.parametrize("call,over", [
    (tables, dict(table=ints(B, 4).t())), (tables, dict(table=gpu(B, 4, dtype=torch.int64))), (tables, dict(held=ints(B + 1))),
    (tables, dict(fresh=gpu(B, dtype=torch.int64))), (tables, dict(free=ints(3, 3))), (tables, dict(held=ints(2 * B)[::2])),
    (tables, dict(table=torch.zeros(B, 4, dtype=torch.int32))),
    (packed, dict(q=gpu(N, 3, D))), (packed, dict(k=gpu(N + 1, KV, D))), (packed, dict(v=gpu(N, KV + 1, D))),
    (packed, dict(k=gpu(N, KV, D, dtype=torch.float32))), (packed, dict(q=gpu(N, H, D, dtype=torch.float16))),
    (packed, dict(q=gpu(N, D, H).transpose(1, 2))), (packed, dict(starts=ints(1))), (packed, dict(starts=gpu(B, dtype=torch.int64))),
    (packed, dict(out=gpu(N, H, D, dtype=torch.float32))), (packed, dict(lse=gpu(N, H, dtype=torch.float32))),
    (packed, dict(workspace=gpu(64, 2, dtype=torch.uint8).t())), (packed, dict(k=gpu(N, 0, D), v=gpu(N, 0, D))),
    (decode, dict(q=gpu(B, 3, D))), (decode, dict(table=ints(B + 1, 4))), (decode, dict(positions=ints(B + 1))),
    (decode, dict(cache=cache(torch.float32))), (decode, dict(q=gpu(B, H, 32))), (decode, dict(out=gpu(B, H, 32))),
    (decode, dict(lse=gpu(H, B, dtype=torch.float32))), (decode, dict(q=gpu(B, H, D, dtype=torch.float16))),
    (store, dict(k=gpu(N, KV + 1, D), v=gpu(N, KV + 1, D))), (store, dict(v=gpu(N, KV, D, dtype=torch.float32))),
    (store, dict(slots=ints(N + 1))), (store, dict(cache=cache(torch.float32))), (store, dict(k=gpu(N, D), v=gpu(N, D))),
])
def test_refusals(library, call, over):
    with pytest.raises(ValueError):
        call(**over)
    assert not library.calls


def test_every_written_tensor_is_reported(library):
    """Each of a call's given outputs by itself: a graph that saved one of them has to know."""
    table, out, lse = ints(B, 4), gpu(N, H, D), gpu(H, N, dtype=torch.float32)
    m = sa.PageMap(ints(B + 1), ints(N), ints(N), ints(B), ints(1))
    step_out, step_lse = gpu(B, H, D), gpu(B, H, dtype=torch.float32)
    written = [table, m.starts, m.positions, m.slots, m.last, m.taken, out, lse, step_out, step_lse]
    before = [t._version for t in written]
    assert tables(table=table, out=m) is m
    packed(out=out, lse=lse)
    decode(out=step_out, lse=step_lse)
    for i, (t, version) in enumerate(zip(written, before)):
        assert t._version > version, i
