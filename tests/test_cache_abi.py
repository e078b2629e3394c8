"""The cache's C ABI without a GPU: the header against the binding, sizes, and
refusals before any device work."""
import ctypes
import os
import re
import shutil
import subprocess

import numpy as np
import pytest

from cache_model import Model, quantise, visible

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "mds_cache.h")


@pytest.fixture(scope="module")
def cache():
    if not os.path.exists(os.path.join(ROOT, "paper_2410_18234_gb300", "_lib", "libmds.so")):
        from paper_2410_18234_gb300 import build
        build.build()
    from paper_2410_18234_gb300 import cache as c
    return c


def test_binding_mirrors_the_header(cache):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(mds_cache_[a-z_]+)\s*\(", text))
    assert names == set(cache.EXPORTS)
    for name in names:
        assert hasattr(cache._lib, name)
    fields = re.findall(r"\b(\w+)\s*;", re.search(r"typedef struct \{(.*?)\} mds_cache_config;", text, flags=re.S).group(1))
    assert [f[0] for f in cache.CacheConfig._fields_] == fields
    value = {k: v for k, v in re.findall(r"#define (MDS_\w+) (.+)", text)}
    for name, own in (("MDS_ST_NOPAGES", cache.MDS_ST_NOPAGES), ("MDS_ST_BADSEQ", cache.MDS_ST_BADSEQ)):
        assert int(value[name].strip().rstrip("u")) == own
    for name, own in (("BLOCK", cache.BLOCK), ("MAX_BATCH", cache.MAX_BATCH), ("MAX_TOKENS", cache.MAX_TOKENS),
                      ("MAX_NODES", cache.MAX_NODES), ("MAX_GROUP", cache.MAX_GROUP)):
        assert eval(value["MDS_CACHE_" + name]) == own


def test_header_compiles_as_c(cache, tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    src = tmp_path / "size.c"
    src.write_text('#include <stdio.h>\n#include "mds_cache.h"\n'
                   'int main(void) { printf("%zu\\n", sizeof(mds_cache_config)); return 0; }\n')
    exe = tmp_path / "size"
    subprocess.run([gcc, "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)],
                   check=True)
    assert int(subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout) == ctypes.sizeof(cache.CacheConfig)


def test_sizes(cache):
    one = cache.cache_bytes(1, 100, 8, 128, 4, 50)
    two = cache.cache_bytes(2, 100, 8, 128, 4, 50)
    pool = 100 * 2 * 8 * 64 * 128
    assert two - one == pool + 100 * 2 * 8 * 4 * 4       # a layer's bytes and scales
    for bad in (dict(layers=0), dict(pages=0), dict(pages=(1 << 24) + 1), dict(kv_heads=0), dict(head_dim=96),
                dict(page_tokens=48), dict(max_seqs=0), dict(max_pages=0), dict(max_pages=1 << 15), dict(dtype=5)):
        kw = dict(layers=1, pages=10, kv_heads=2, head_dim=64, max_seqs=2, max_pages=4, page_tokens=64)
        kw.update(bad)
        with pytest.raises(cache.MdsError) as e:
            cache.cache_bytes(**kw)
        assert e.value.code == cache.MDS_ESHAPE


def test_null_arguments_are_refused(cache):
    lib, n = cache._lib, None
    st = (ctypes.c_int64 * 3)(0, 0, 0)
    assert lib.mds_cache_create(n, n, 0, n, n) == cache.MDS_EINVAL
    h = ctypes.c_void_p()
    cfg = cache.CacheConfig(1, 10, 64, 2, 64, 2, 4, 1)
    assert lib.mds_cache_create(ctypes.byref(h), ctypes.byref(cfg), 0, n, n) == cache.MDS_EINVAL    # no memory
    assert lib.mds_cache_create(ctypes.byref(h), ctypes.byref(cfg), 0, 1536, n) == cache.MDS_EINVAL  # not aligned
    assert not h
    assert lib.mds_cache_state(n, n, n) == cache.MDS_EINVAL
    assert lib.mds_cache_reserve(n, n, n, 1, 1, n) == cache.MDS_EINVAL
    assert lib.mds_cache_append(n, 0, n, n, n, st, n, st, 1, 1, n) == cache.MDS_EINVAL
    assert lib.mds_cache_attend(n, 0, n, n, n, st, n, 1, 1, 1, 0, 0, 1.0, 1, n) == cache.MDS_EINVAL
    assert lib.mds_cache_commit(n, n, n, n, n, 1, 0, 1, n) == cache.MDS_EINVAL
    assert lib.mds_cache_fork(n, n, n, 1, n) == cache.MDS_EINVAL
    assert lib.mds_cache_truncate(n, n, n, 1, n) == cache.MDS_EINVAL
    assert lib.mds_cache_free(n, n, 1, n) == cache.MDS_EINVAL
    assert lib.mds_cache_read(n, 0, n, n, n, n, n, 1, 1, n) == cache.MDS_EINVAL
    assert lib.mds_cache_status(n, n) == cache.MDS_EINVAL
    lib.mds_cache_destroy(n)


# ------------------------------------------- what the tests' model stands on


def test_model_quantiser():
    """Every e4m3 number stands for itself, midpoints go to even mantissas,
    quantising values again changes nothing, the scale holds the maximum."""
    grid = sorted({m * 2.0 ** (e - 3) for e in range(-6, 9) for m in range(8, 16) if m * 2.0 ** (e - 3) <= 448}
                  | {m * 2.0 ** -9 for m in range(8)})
    x = np.zeros((16, 16))
    x.flat[:len(grid)] = grid
    np.testing.assert_array_equal(quantise(x), x)
    y = np.full((16, 2), 448.0)
    y[0] = 17.0, 19.0                       # between 16, 18 and 20
    np.testing.assert_array_equal(quantise(y)[0], [16.0, 20.0])
    rng = np.random.default_rng(0)
    for _ in range(200):
        z = rng.standard_normal((16, 8)) * 2.0 ** rng.integers(-60, 60) * np.exp2(rng.integers(-20, 1, (16, 1)))
        q = quantise(z)
        np.testing.assert_array_equal(quantise(q), q)
        assert np.abs(q - z).max() <= 2.0 ** -4 * np.abs(z).max()


def test_model_tree():
    """Visibility on a tree of 2 branches of 2 behind 3 tokens, by hand."""
    see = visible(5, 2, 3)
    want = ["11110000", "11111000", "11111100", "11110010", "11110011"]
    assert ["".join("01"[int(x)] for x in r) for r in see] == want
    see = visible(5, 2, 3, window=2, sinks=1)
    want = ["10110000", "10011000", "10001100", "10010010", "10000011"]
    assert ["".join("01"[int(x)] for x in r) for r in see] == want


def test_model_pages():
    m = Model(1, 6, 1, 4, 3, 6, 16)
    assert m.reserve([1, 0], [20, 1]) == []
    assert m.rows == [[2], [0, 1], []]
    m.commit([1], [19])
    m.fork([1], [2])
    assert m.reserve([1, 2], [3, 3]) == [] and m.rows[1:] == [[0, 3], [0, 4]] and m.ref == [2, 0, 1, 1, 1, 0]
    m.free([1, 2])
    assert m.ref == [0, 0, 1, 0, 0, 0]
