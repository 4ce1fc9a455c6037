"""The rotary frequencies that the host hands to the kernel (csrc/sa_turns.h) against 60 digits, for bases from next to 1 to
the largest, within the bound that the angle's own is made of."""
import os
import subprocess
from decimal import Decimal, getcontext

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
SAN = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
       "-Xarch_host", "-fno-sanitize-recover=undefined"]
PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459")


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")
def test_frequencies(tmp_path):
    exe = tmp_path / "turns"
    subprocess.run([HIPCC, "-O2", "-std=c++17", *SAN, "-I", os.path.join(ROOT, "paper_1904_10509_amd", "csrc"),
                    os.path.join(ROOT, "tests", "host", "check_turns.cpp"), "-o", str(exe)], check=True, capture_output=True)
    cases = [(base, size) for base in (1.0000000001, 1.0001, 1.1, 1.5, 3.0, 10000.0, 500000.0, 1e30, 1.7e308)
             for size in (2, 4, 10, 48, 64, 96, 126, 128)]
    out = subprocess.run([str(exe), *(str(x) for c in cases for x in map(repr, c))], capture_output=True, text=True,
                         timeout=60, check=True, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0")).stdout.splitlines()
    getcontext().prec = 60
    bound = Decimal(float(out[0]))
    for (base, size), line in zip(cases, out[1:]):
        got = [Decimal(x) for x in line.split()]
        assert len(got) == size // 2
        for t, x in enumerate(got):
            want = Decimal(base) ** (Decimal(-2 * t) / Decimal(size)) / (2 * PI) * Decimal(2) ** 64
            assert abs(x - want) <= bound, (base, size, t, x - want)
