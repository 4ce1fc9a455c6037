"""Which memory rotary's gradient reads its positions from, without a GPU: the tensor that autograd hands back, whatever a
saved-tensor hook made of it, and not the one that the forward saw, which may be gone.  The launch is recorded in place of
being made, so no address is followed."""
import contextlib

import pytest
import torch
from torch.utils.checkpoint import checkpoint

from paper_1904_10509_amd import sparse_attn as sa

GPU = torch.device("cuda", 0)
B, H, N, D, DIMS = 2, 3, 8, 64, (32, 16, 16)


class OnGpu(torch.Tensor):
    """A tensor in host memory that the binding takes for one on the GPU."""

    @property
    def device(self):
        return GPU


class Library:
    """Records each rotary call's inverse, address of the positions and their strides."""

    def __init__(self):
        self.calls = []

    def sparse_attn_rotary(self, *args):
        self.calls.append((args[-2], args[14], tuple(args[15])))
        return sa.SA_OK


@pytest.fixture
def library(monkeypatch):
    got = Library()
    monkeypatch.setattr(sa, "lib", lambda: got)
    monkeypatch.setattr(sa, "_here", lambda device, stream: contextlib.nullcontext())
    monkeypatch.setattr(sa, "_stream", lambda stream, device: 0)
    return got


def host(*shape):
    return torch.randn(*shape).as_subclass(OnGpu)


def places(shared=True):
    t = torch.zeros((N, 3) if shared else (B, N, 3), dtype=torch.int32)
    return t.as_subclass(OnGpu)


def gradients(q, k, out):
    return torch.autograd.grad(out, (q, k), (host(*q.shape), host(*k.shape)))


def leaves():
    return host(B, H, N, D).requires_grad_(), host(B, 1, N, D).requires_grad_()


@pytest.mark.parametrize("shared", [True, False])
def test_without_hooks_the_positions_themselves(library, shared):
    (q, k), at = leaves(), places(shared)
    gradients(q, k, sa.Rotary.apply(q, k, at, DIMS))
    want = (at.data_ptr(), (0 if shared else 3 * N, 3))
    assert library.calls == [(0, *want), (1, *want)]


def test_a_hook_that_copies(library):
    """What the hook unpacks may lie elsewhere and have another layout."""
    (q, k), wide = leaves(), torch.zeros(N, 7, dtype=torch.int32).as_subclass(OnGpu)
    alive = []

    def unpack(t):
        alive.append(t)
        return t

    with torch.autograd.graph.saved_tensors_hooks(lambda t: t.clone(memory_format=torch.contiguous_format), unpack):
        out = sa.Rotary.apply(q, k, wide[:, 2:5], DIMS)
    gradients(q, k, out)
    assert library.calls[0] == (0, wide[:, 2:5].data_ptr(), (0, 7))
    assert library.calls[1] == (1, alive[-1].data_ptr(), (0, 3)) and alive[-1].data_ptr() != wide[:, 2:5].data_ptr()


def test_recomputed_positions(library):
    """Checkpointing: the gradient turns by the positions of the second forward; the first one's are gone."""
    q, k = leaves()
    made = []

    def layer(q, k):
        at = places()
        made.append(at)
        return sa.Rotary.apply(q, k, at, DIMS)

    gradients(q, k, checkpoint(layer, q, k, use_reentrant=False))
    assert len(made) == 2 and [c[0] for c in library.calls] == [0, 0, 1]
    assert [c[1] for c in library.calls] == [made[0].data_ptr(), made[1].data_ptr(), made[1].data_ptr()]


def test_unpacked_positions_are_checked(library):
    """A hook that hands back another type or shape is refused like a call with it."""
    for pack in (lambda t: t.long() if t.dtype == torch.int32 else t, lambda t: t[:4] if t.dtype == torch.int32 else t):
        q, k = leaves()
        with torch.autograd.graph.saved_tensors_hooks(pack, lambda t: t):
            out = sa.Rotary.apply(q, k, places(), DIMS)
        with pytest.raises(ValueError, match="positions must be"):
            gradients(q, k, out)
    assert [c[0] for c in library.calls] == [0, 0]
