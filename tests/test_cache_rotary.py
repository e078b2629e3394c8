"""Rotary positions without a GPU: frequencies, turns, refusals, and the C
struct against the binding's."""
import ctypes
import math
import os
import shutil
import subprocess
from decimal import Decimal, getcontext

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if not os.path.exists(os.path.join(ROOT, "paper_2410_18234_gb300", "_lib", "libmds.so")):
    from paper_2410_18234_gb300 import build
    build.build()

from paper_2410_18234_gb300 import cache  # noqa: E402

getcontext().prec = 60
TWO_PI = 2 * Decimal("3.14159265358979323846264338327950288419716939937510582097494459")


@pytest.mark.parametrize("kw", [dict(), dict(base=500000.0, factor=8.0, original=8192), dict(factor=4.0),
                                dict(freqs=[math.pi, -math.pi, -1.0, 1e-9, -1e-300, 0.0] + [0.1 * i for i in range(26)])])
def test_turns_are_off_by_less_than_a_unit(kw):
    r = cache.Rotary(64, **kw)
    for f, t in zip(r.freqs, r.struct.turns):
        units = int((Decimal(f) / TWO_PI * 2 ** 64 * 1024).to_integral_value()) - t * 1024
        units %= 2 ** 74
        assert min(units, 2 ** 74 - units) <= 1024


def test_frequencies():
    r = cache.Rotary(48)
    assert r.freqs == [10000.0 ** (-2 * i / 48) for i in range(24)]
    near = cache.Rotary(48, factor=4.0)
    assert near.freqs == [f / 4.0 for f in r.freqs]
    # with a length: pairs that turn often stay, the slowest are divided
    part = cache.Rotary(48, factor=4.0, original=4096)
    assert part.freqs[0] == r.freqs[0] and part.freqs[-1] == r.freqs[-1] / 4.0
    assert all(a / 4.0 <= b <= a for a, b in zip(r.freqs, part.freqs))


@pytest.mark.parametrize("code,kw", [("S", dict(dim=0)), ("S", dict(dim=8)), ("S", dict(dim=24)), ("S", dict(dim=144)),
                                     ("S", dict(dim=1 << 33)), ("S", dict(dim=64, freqs=[1.0] * 31)),
                                     ("E", dict(dim=64, freqs=[3.2] * 32)), ("E", dict(dim=64, freqs=[float("nan")] * 32)),
                                     ("E", dict(dim=64, base=0.5)), ("E", dict(dim=64, base=float("inf"))),
                                     ("E", dict(dim=64, factor=0.0)), ("E", dict(dim=64, factor=0.1)),
                                     ("E", dict(dim=64, original=-1)), ("E", dict(dim=64, slow=4.0, fast=4.0)),
                                     ("E", dict(dim=64, magnitude=0.0)), ("E", dict(dim=64, magnitude=float("nan"))),
                                     ("E", dict(dim=64, magnitude=-1.0)), ("E", dict(dim=64, magnitude=2.0 ** 21))])
def test_refusals(code, kw):
    with pytest.raises(cache.MdsError) as e:
        cache.Rotary(**kw)
    assert e.value.code == {"S": cache.MDS_ESHAPE, "E": cache.MDS_EINVAL}[code]


def test_null_arguments():
    lib, one = cache._lib, cache.RotaryStruct()
    freqs = (ctypes.c_double * 64)()
    assert lib.mds_cache_rotary_init(None, freqs, 64, 0, 1.0) == cache.MDS_EINVAL
    assert lib.mds_cache_rotary_init(ctypes.byref(one), None, 64, 0, 1.0) == cache.MDS_EINVAL
    assert lib.mds_cache_rotary_init(ctypes.byref(one), freqs, 64, 2, 1.0) == cache.MDS_EINVAL
    assert lib.mds_cache_rotate(None, None, None, ctypes.byref(one), None, None, None, 1, 1, 1, 1, None) == cache.MDS_EINVAL
    assert lib.mds_cache_append_rotated(None, 0, None, None, ctypes.byref(one), None, None, None, None, None, None, None,
                                        0, 1, 1, 1, None) == cache.MDS_EINVAL


def test_struct_mirrors_the_header(tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    src = tmp_path / "size.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "mds_cache.h"\n'
                   'int main(void) { printf("%zu %zu %zu %zu\\n", sizeof(mds_cache_rotary), offsetof(mds_cache_rotary, interleaved), '
                   'offsetof(mds_cache_rotary, magnitude), offsetof(mds_cache_rotary, turns)); return 0; }\n')
    exe = tmp_path / "size"
    subprocess.run([gcc, "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)],
                   check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    R = cache.RotaryStruct
    assert got == [ctypes.sizeof(R), R.interleaved.offset, R.magnitude.offset, R.turns.offset]
