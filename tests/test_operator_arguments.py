"""What the binding takes and refuses around the 8-bit cache, without a GPU: the launches are recorded in place of being made."""
import contextlib
import ctypes

import pytest
import torch

from paper_1904_10509_amd import sparse_attn as sa

GPU = torch.device("cuda", 0)
B, KV, CAP, D, T = 2, 4, 100, 64, 32


class OnGpu(torch.Tensor):
    """A tensor in host memory that the binding takes for one on the GPU."""

    @property
    def device(self):
        return GPU


class Library:
    """Records the calls by name; a decoding step asks for a workspace of 4,096 bytes."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            if name == "sparse_attn_decode8_workspace_size":
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


def gpu(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)


def cache(dtype=torch.float8_e4m3fn):
    c = sa.build_cache8(B, KV, CAP, D, T, device="cpu")
    return sa.Cache8(*(t.as_subclass(OnGpu) for t in (c.k.view(dtype), c.v.view(dtype), c.k_scale, c.v_scale)), T)


def decode(c, **over):
    args = dict(q=gpu(B, KV, D), cache=c, positions=gpu(B, dtype=torch.int32), stride_l=16, summary_c=0,
                pattern=sa.SA_STRIDED, head_mode=sa.SA_MODE_MERGED)
    args.update(over)
    return sa.decode8(**args)


@pytest.mark.parametrize("dtype", [torch.float8_e4m3fn, torch.uint8])
def test_cache_types(library, dtype):
    sa.store8(cache(dtype), gpu(B, KV, 5, D), gpu(B, KV, 5, D))
    decode(cache(dtype))
    assert [name for name, _ in library.calls] == ["sparse_attn_cache8_store", "sparse_attn_decode8"]


@pytest.mark.parametrize("dtype", [torch.float8_e5m2, torch.float8_e4m3fnuz, torch.float8_e5m2fnuz, torch.int8])
def test_other_types_of_eight_bits_are_refused(library, dtype):
    """Their values are not those of the codes that the cache holds."""
    with pytest.raises(ValueError, match="float8_e4m3fn or uint8"):
        sa.store8(cache(dtype), gpu(B, KV, 5, D), gpu(B, KV, 5, D))
    with pytest.raises(ValueError, match="float8_e4m3fn or uint8"):
        decode(cache(dtype))
    assert not library.calls


def test_workspace_in_pieces_is_refused(library):
    """The library writes as many bytes as the workspace has elements, one behind the other."""
    room = torch.zeros(16, dtype=torch.uint8).as_subclass(OnGpu)
    for bad in (room[:1].expand(8192), gpu(16384, dtype=torch.uint8)[::2], gpu(64, 128, dtype=torch.uint8).t()):
        with pytest.raises(ValueError, match="contiguous"):
            decode(cache(), workspace=bad)
    assert not library.calls
    decode(cache(), workspace=gpu(64, 128, dtype=torch.uint8))
    assert library.calls[0][1][-2] == 8192


def test_writes_in_place_are_told_to_autograd(library):
    """A graph that saved what a call writes over raises, as behind torch's own operations, and nothing else does."""
    leaf = gpu(B, KV, 8, D).requires_grad_()
    places = gpu(8, 2, dtype=torch.int32)

    def saved():
        x = leaf * 2
        return x, (x * x).sum()

    x, y = saved()
    with torch.no_grad():
        sa.rotary(x, None, places, (32, 32), out=(x, None))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    (q, y), (k, z) = saved(), saved()
    with torch.no_grad():
        sa.rotary(q, k, places, (32, 32), out=(gpu(B, KV, 8, D), k))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        z.backward()
    y.backward()  # q was read alone
    c = cache()
    before = [t._version for t in (c.k, c.v, c.k_scale, c.v_scale)]
    x = gpu(B, KV, 5, D)
    sa.store8(c, x, x)
    assert all(t._version > old for t, old in zip((c.k, c.v, c.k_scale, c.v_scale), before)) and x._version == 0
    q, out, lse = gpu(B, KV, D), gpu(B, KV, D), gpu(B, KV, dtype=torch.float32)
    before = [t._version for t in (c.k, c.v, c.k_scale, c.v_scale)]
    decode(c, q=q, out=out, lse=lse)
    assert out._version > 0 and lse._version > 0 and q._version == 0
    assert [t._version for t in (c.k, c.v, c.k_scale, c.v_scale)] == before
    with torch.inference_mode():  # where tensors have no version
        x = gpu(B, KV, 5, D)
        sa.rotary(x, None, gpu(5, 1, dtype=torch.int32), (64,), out=(x, None))
        sa.store8(cache(), x, x)
        decode(cache(), out=gpu(B, KV, D), lse=gpu(B, KV, dtype=torch.float32))


def test_rotary_outputs_over_each_other_are_refused(library):
    """Workgroups turn q and k at once, in any order: an output may be its own input, not the other's, nor may both be one."""
    q, k, places = gpu(B, KV, 8, D), gpu(B, KV, 8, D), gpu(8, 1, dtype=torch.int32)
    other = gpu(B, KV, 8, D)
    for out in ((k, q), (k, other), (other, q), (other, other), (q, q)):
        with pytest.raises(ValueError, match="out"):
            sa.rotary(q, k, places, (64,), out=out)
    with pytest.raises(ValueError, match="out"):
        sa.rotary(q, q, places, (64,), out=(q, q))
    assert not library.calls
    for out in ((q, k), (other, k), (q, other)):
        sa.rotary(q, k, places, (64,), out=out)
    sa.rotary(q, q, places, (64,), out=(other, k))  # read alone
    sa.rotary(q, None, places, (64,), out=(q, None))
    assert len(library.calls) == 5


def handed_over(call):
    """Of a recorded store: the strides that the library steps over, and the addresses of k and v."""
    return tuple(call[1][7]), call[1][5], call[1][6]


def test_store_of_rotated_keys_and_values_from_a_projection(library):
    """k comes out of rotary packed, v is a slice of the projection: where the strides that are stepped over are one set
    neither is copied, else both reach the library packed.  The same for one token a sequence."""
    c = cache()
    for n in (7, 1):
        qkv = torch.randn(B, n, 3, KV, D).to(torch.bfloat16).as_subclass(OnGpu)
        k, v = (qkv[:, :, i].transpose(1, 2) for i in (1, 2))
        sa.store8(c, k, v)  # of one layout: in place
        assert handed_over(library.calls[-1])[1:] == (k.data_ptr(), v.data_ptr())
        packed = k.contiguous()
        sa.store8(c, packed, v)
        strides, at_k, at_v = handed_over(library.calls[-1])
        assert strides == (KV * n * D, n * D, D) and at_k == packed.data_ptr() and at_v != v.data_ptr()
        if n == 1:
            sa.store8(c, packed[:, :, 0], v[:, :, 0])
            strides, at_k, at_v = handed_over(library.calls[-1])
            assert strides == (KV * D, D, D) and at_k == packed.data_ptr()
    # a dimension of one element is not stepped over: its stride does not tell layouts apart
    one = cache()
    one = sa.Cache8(one.k[:1], one.v[:1], one.k_scale[:1], one.v_scale[:1], T)
    row = torch.randn(1, KV, 1, D).to(torch.bfloat16)
    k, v = row.as_subclass(OnGpu), row.as_strided(row.shape, (7 * D, D, 9 * D, 1)).as_subclass(OnGpu)
    assert k.stride() != v.stride()
    sa.store8(one, k, v)
    assert handed_over(library.calls[-1]) == ((0, D, D), k.data_ptr(), v.data_ptr())
    with pytest.raises(ValueError):
        sa.store8(c, gpu(B, KV, 5, D), gpu(B, KV, 6, D))
    with pytest.raises(ValueError):
        sa.store8(c, gpu(B, KV, 5, D), gpu(B, KV, 5, 2 * D)[..., ::2])


def test_entry_points_marshal_alone(library):
    """The functions named like the C entry points take tensors, addresses or None and hand them on."""
    t = gpu(B, KV, 8, D)
    strides, two = (ctypes.c_int64 * 3)(1, 2, 3), (ctypes.c_int64 * 2)(4, 5)
    at = t.data_ptr()
    sa.sparse_attn_rotary(B, 8, KV, 0, D, sa.SA_BF16, t, strides, t, strides, None, None, None, None, t, two, 1,
                          (ctypes.c_int32 * 1)(D), 10000.0, 0, 0)
    sa.sparse_attn_cache8_store(B, KV, 8, D, sa.SA_BF16, t, t, strides, None, t, CAP, T, t, t, strides, t, t)
    sa.sparse_attn_decode8(t, 9, 16, 0, sa.SA_STRIDED, sa.SA_MODE_MERGED, B, KV, KV, D, sa.SA_BF16, t, two, t, t, strides, t, t,
                           CAP, T, 0.125, t, two, t, t, 64)
    assert [name for name, _ in library.calls] == ["sparse_attn_rotary", "sparse_attn_cache8_store", "sparse_attn_decode8"]
    assert library.calls[0][1][6] == at and library.calls[0][1][10] is None
    assert library.calls[1][1][5] == at and library.calls[1][1][8] is None
    assert library.calls[2][1][0] == at
