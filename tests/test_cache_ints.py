"""Sizes that do not fit the C interface's integers are refused, not cut to 32 bits."""
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if not os.path.exists(os.path.join(ROOT, "paper_2410_18234_gb300", "_lib", "libmds.so")):
    from paper_2410_18234_gb300 import build
    build.build()

import torch  # noqa: E402

from paper_2410_18234_gb300 import cache  # noqa: E402

WIDE = 1 << 32


@pytest.mark.parametrize("name", ["layers", "pages", "kv_heads", "head_dim", "max_seqs", "max_pages", "page_tokens", "dtype"])
def test_configurations(name):
    kw = dict(layers=1, pages=10, kv_heads=2, head_dim=64, max_seqs=2, max_pages=4, page_tokens=64, dtype=1)
    assert cache.cache_bytes(**kw) > 0
    for far in (WIDE, -WIDE):
        with pytest.raises(cache.MdsError) as e:
            cache.cache_bytes(**{**kw, name: kw[name] + far})
        assert e.value.code == cache.MDS_ESHAPE


@pytest.mark.gpu
def test_calls():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    c = cache.Cache(1, 20, 2, 64, 2, 10, page_tokens=16)
    seqs = torch.tensor([0], device="cuda", dtype=torch.int32)
    x = torch.zeros(1, 5, 2, 64, device="cuda", dtype=torch.bfloat16)
    c.reserve(seqs, 5)

    def refused(fn, *a, **kw):
        with pytest.raises(cache.MdsError) as e:
            fn(*a, **kw)
        assert e.value.code == cache.MDS_ESHAPE

    refused(c.reserve, seqs, WIDE + 1)
    refused(c.append, WIDE, seqs, x, x)
    refused(c.attend, WIDE, seqs, x)
    refused(c.attend, 0, seqs, x, branches=WIDE + 2)
    refused(c.attend, 0, seqs, x, window=WIDE + 2)
    refused(c.attend, 0, seqs, x, window=4, sinks=WIDE)
    refused(c.commit, seqs, seqs, branches=WIDE + 1)
    refused(c.read, WIDE, seqs, None, 5)
    refused(c.read, -WIDE, seqs, None, 5)
    assert c.status() == (0, "ok")
    with pytest.raises(cache.MdsError):
        cache.Cache(1, 20, 2, 64, 2 + WIDE, 10)


@pytest.mark.gpu
def test_read_of_no_layer():
    """-1 means every layer at the C entry only: the binding's outputs are
    one layer's, and the call is refused before anything is written."""
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    c = cache.Cache(3, 20, 2, 64, 2, 10, page_tokens=16)
    seqs = torch.tensor([0], device="cuda", dtype=torch.int32)
    out = tuple(torch.full((3, 1, 5, 2, 64), 7.0, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    with pytest.raises(cache.MdsError) as e:
        c.read(-1, seqs, None, 5, out=(out[0][0], out[1][0]))
    assert e.value.code == cache.MDS_ESHAPE
    assert all((x == 7.0).all() for x in out)
    c.read(None, seqs, None, 5, out=out)
    assert not any(x.any() for x in out)
    assert c.status() == (0, "ok")
