"""What the rotary, 8-bit store and 8-bit decoding entry points refuse, before anything is enqueued (no GPU needed:
the pointers are never dereferenced), and the arithmetic that their host code does."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

import operator_refs as ref
from paper_1904_10509_amd import sparse_attn as sa

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
SAN = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
       "-Xarch_host", "-fno-sanitize-recover=undefined"]
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


def ints(*v):
    return (ctypes.c_int32 * len(v))(*v)


ROTARY = dict(batch=2, n=8, qh=4, kh=2, d=64, dtype=sa.SA_BF16, q=FAKE, qs=longs(2048, 512, 64), qo=FAKE,
              qos=longs(2048, 512, 64), k=FAKE, ks=longs(1024, 512, 64), ko=FAKE, kos=longs(1024, 512, 64), pos=FAKE,
              ps=longs(0, 2), axes=2, dims=ints(32, 32), base=10000.0, pairing=0, inverse=0, stream=None)


@pytest.mark.parametrize("over,expect", [
    (dict(batch=0), INV), (dict(n=0), INV), (dict(n=2 ** 31), INV), (dict(qh=-1), INV), (dict(qh=0, kh=0), INV),
    (dict(d=48), UNS), (dict(dtype=2), INV), (dict(q=None), INV), (dict(q=FAKE + 8), INV), (dict(qo=FAKE + 2), INV),
    (dict(qs=longs(2048, 512, 32)), INV), (dict(qs=longs(2048, 516, 64)), INV), (dict(qos=longs(-8, 512, 64)), INV),
    (dict(qs=longs(4096, 512, 64)), INV),  # its own output with other strides
    (dict(qos=longs(2048, 0, 64)), INV), (dict(qos=longs(0, 512, 64)), INV),  # rows that two heads would write
    (dict(k=None), INV), (dict(ko=None), INV), (dict(kos=None), INV), (dict(ks=longs(1024, 512, 68)), INV),
    (dict(pos=None), INV), (dict(pos=FAKE + 2), INV), (dict(ps=None), INV), (dict(ps=longs(-1, 2)), INV),
    (dict(axes=0), INV), (dict(axes=5), INV), (dict(dims=ints(31, 32)), INV), (dict(dims=ints(0, 32)), INV),
    (dict(dims=ints(34, 32)), INV), (dict(dims=None), INV), (dict(base=1.0), INV), (dict(base=float("nan")), INV),
    (dict(base=float("inf")), INV), (dict(pairing=2), INV), (dict(inverse=2), INV),
    (dict(batch=2 ** 30, n=2 ** 10), UNS), (dict(qh=65536), UNS), (dict(kh=2 ** 31 - 1), UNS),
])
def test_rotary_refusals(L, over, expect):
    assert L.sparse_attn_rotary(*dict(ROTARY, **over).values()) == expect


STORE = dict(batch=2, kvh=4, n=8, d=64, dtype=sa.SA_BF16, k=FAKE, v=FAKE, ks=longs(2048, 512, 64), start=FAKE, counts=FAKE,
             capacity=100, block=64, kc=FAKE, vc=FAKE + 64, cs=longs(51200, 12800, 128), ksc=FAKE, vsc=FAKE, stream=None)


@pytest.mark.parametrize("over,expect", [
    (dict(batch=0), INV), (dict(kvh=0), INV), (dict(n=0), INV), (dict(n=2 ** 31), INV), (dict(d=40), UNS),
    (dict(dtype=3), INV), (dict(k=None), INV), (dict(v=FAKE + 8), INV), (dict(ks=None), INV),
    (dict(ks=longs(2048, 512, 56)), INV), (dict(ks=longs(2048, 510, 64)), INV), (dict(start=FAKE + 1), INV),
    (dict(counts=FAKE + 2), INV), (dict(capacity=0), INV), (dict(capacity=2 ** 31), INV), (dict(block=48), INV),
    (dict(block=256), INV), (dict(kc=None), INV), (dict(vc=FAKE + 8), INV), (dict(cs=None), INV),
    (dict(cs=longs(51200, 12800, 48)), INV), (dict(cs=longs(51200, 12808, 128)), INV), (dict(ksc=None), INV),
    (dict(cs=longs(0, 12800, 128)), INV), (dict(cs=longs(51200, 0, 128)), INV),  # rows that two would write
    (dict(vsc=FAKE + 2), INV), (dict(batch=2 ** 20, n=2 ** 20), UNS),
])
def test_store_refusals(L, over, expect):
    assert L.sparse_attn_cache8_store(*dict(STORE, **over).values()) == expect


DECODE = dict(pos=FAKE, max_pos=99, l=16, c=0, pattern=sa.SA_STRIDED, mode=sa.SA_MODE_MERGED, batch=2, heads=4, kvh=2, d=64,
              dtype=sa.SA_BF16, q=FAKE, qs=longs(256, 64), kc=FAKE, vc=FAKE, cs=longs(12800, 6400, 64), ksc=FAKE, vsc=FAKE,
              capacity=100, block=16, scale=0.125, o=FAKE, os=longs(256, 64), lse=FAKE, ws=FAKE, wsb=1 << 30, stream=None)


@pytest.mark.parametrize("over,expect", [
    (dict(pos=None), INV), (dict(pos=FAKE + 2), INV), (dict(max_pos=-1), INV), (dict(max_pos=100), INV),
    (dict(max_pos=2 ** 31), INV), (dict(l=0), INV), (dict(c=3), INV), (dict(pattern=3), INV), (dict(mode=4), INV),
    (dict(pattern=sa.SA_FIXED_PER_HEAD, l=130, c=2), UNS), (dict(batch=0), INV), (dict(heads=3), INV), (dict(kvh=0), INV),
    (dict(d=16), UNS), (dict(dtype=-1), INV), (dict(q=FAKE + 4), INV), (dict(qs=longs(256, 60)), INV), (dict(qs=None), INV),
    (dict(kc=None), INV), (dict(vc=FAKE + 4), INV), (dict(cs=longs(12800, 6400, 32)), INV), (dict(ksc=None), INV),
    (dict(capacity=0), INV), (dict(block=8), INV), (dict(scale=0.0), INV), (dict(scale=float("nan")), INV),
    (dict(o=None), INV), (dict(os=None), INV), (dict(os=longs(0, 64)), INV), (dict(os=longs(256, 56)), INV),
    (dict(os=longs(256, 68)), INV), (dict(lse=None), INV), (dict(lse=FAKE + 2), INV), (dict(ws=None), INV), (dict(ws=FAKE + 8), INV),
    (dict(wsb=0), SMALL), (dict(batch=2 ** 20, heads=8), UNS), (dict(capacity=2 ** 31 - 1), UNS),
    (dict(cs=longs(0, 0, 2 ** 62)), UNS),
])
def test_decode8_refusals(L, over, expect):
    assert L.sparse_attn_decode8(*dict(DECODE, **over).values()) == expect


def test_decode8_workspace(L):
    def size(*a):
        return sa.sparse_attn_decode8_workspace_size(*a)
    some = size(65535, 256, 32, sa.SA_FIXED, sa.SA_MODE_MERGED, 1, 8, 8, 64, sa.SA_BF16)
    assert 0 < some == size(65535, 256, 32, sa.SA_FIXED, sa.SA_MODE_MERGED, 1, 8, 8, 64, sa.SA_F32)
    # a launch's ranges are bounded, and so is its workspace: 4,096 workgroups, or one a row
    most = size(2 ** 31 - 1, 2 ** 31 - 1, 0, sa.SA_STRIDED, sa.SA_MODE_A1, 64, 8, 8, 128, sa.SA_BF16)
    assert most <= 4096 * 16 * 130 * 4
    out = ctypes.c_size_t(0)
    assert L.sparse_attn_decode8_workspace_size(10, 16, 0, 0, 2, 1, 3, 2, 64, 1, ctypes.byref(out)) == INV
    assert L.sparse_attn_decode8_workspace_size(10, 16, 0, 0, 2, 1, 2, 2, 64, 1, None) == INV
    assert L.sparse_attn_decode8_workspace_size(10, 16, 0, 0, 2, 1, 2, 2, 24, 1, ctypes.byref(out)) == UNS


def cpu(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype)


def test_binding_refuses_what_the_library_cannot_see(L):
    """Shapes, types and devices, before anything reaches the library (here: tensors that are on no GPU)."""
    q, places = cpu(1, 2, 8, 64), cpu(8, 1, dtype=torch.int32)
    for bad in (dict(q=cpu(8, 64)), dict(k=cpu(1, 2, 9, 64)), dict(k=cpu(1, 2, 8, 32)), dict(k=cpu(2, 8, 64))):
        args = dict(q=q, k=q)
        args.update(bad)
        with pytest.raises(ValueError, match="batch, heads"):
            sa.rotary(args["q"], args["k"], places, (64,))
    with pytest.raises(ValueError, match="share type and GPU"):
        sa.rotary(q, q, places, (64,))
    cache = sa.build_cache8(1, 2, 100, 64, 32, device="cpu")
    assert cache.k.stride() == (25600, 12800, 128, 1) and cache.v.data_ptr() - cache.k.data_ptr() == 64
    assert cache.k_scale.shape == (1, 2, 4)
    with pytest.raises(ValueError):
        sa.store8(cache, q, q)
    with pytest.raises(ValueError, match="on the GPU"):
        sa.decode8(q[:, :, 0], cache, cpu(1, dtype=torch.int32), 16, 0, 0, 2)
    with pytest.raises(ValueError, match="one layout"):
        sa.Cache8(cache.k, cache.v[:, :, :50], cache.k_scale, cache.v_scale, 32)._args(64, cache.k.device)
    with pytest.raises(ValueError, match="scales"):
        sa.Cache8(cache.k, cache.v, cache.k_scale, cache.v_scale, 64)._args(64, cache.k.device)
    with pytest.raises(ValueError, match="d of the tensors"):
        cache._args(32, cache.k.device)


def test_grid_positions():
    got = sa.grid_positions((2, 3, 2), device="cpu")
    assert got.dtype == torch.int32 and got.shape == (12, 3)
    assert got.tolist() == [[a, b, c] for a in range(2) for b in range(3) for c in range(2)]


def test_reference_codes_match_torch():
    """The tests' own e4m3 against torch's: every code's value, and the nearest code of values around every border."""
    codes = torch.arange(256, dtype=torch.uint8)
    values = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(values, ref.VALUES, equal_nan=True)
    fine = np.sort(ref.VALUES[np.isfinite(ref.VALUES)])
    mid = (fine[1:] + fine[:-1]) / 2
    x = np.concatenate([fine, mid, mid * (1 + 2.0 ** -20), mid * (1 - 2.0 ** -20)])
    want = torch.from_numpy(x).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    got = ref.e4m3_encode(x)
    assert np.array_equal(ref.VALUES[got], ref.VALUES[want])


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")
@pytest.mark.parametrize("program", ["check_scale", "check_key_set"])
def test_host_arithmetic(tmp_path, program):
    """The scales' exponents (csrc/sa_e4m3.h) and the step's index space (KeySet, csrc/sa_pattern.h) against their
    definitions, around every border."""
    exe = tmp_path / program
    subprocess.run([HIPCC, "-O2", "-std=c++17", *SAN, "-I", os.path.join(ROOT, "paper_1904_10509_amd", "csrc"),
                    os.path.join(ROOT, "tests", "host", program + ".cpp"), "-o", str(exe)], check=True, capture_output=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300,
                         env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
    assert out.returncode == 0 and out.stdout.startswith("ok"), out.stdout + out.stderr
