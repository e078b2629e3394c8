"""Batch, node and head axes that run backwards in memory: strides below 0 with
the base at the first row, which the C interface takes."""
import ctypes

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

from paper_2410_18234_gb300 import cache  # noqa: E402
from test_gpu_cache_shared import DEV, both, fork, grow, ints, tokens  # noqa: E402

BACK = [(0,), (1,), (2,), (0, 1), (0, 1, 2)]
# members of a group, branches, length, query heads on one: rows of a group and
# of a sequence for each of the kernels
ROWS = [(2, 1, 0, 4), (6, 1, 0, 4), (6, 1, 2, 4), (6, 2, 4, 4), (3, 3, 3, 1)]


def backwards(x, axes):
    """Address and strides of x's values in memory whose `axes` run backwards."""
    y = x.flip(axes).contiguous()
    at = tuple(y.shape[i] - 1 if i in axes else 0 for i in range(3))
    strides = (ctypes.c_int64 * 3)(*(y.stride(i) * (-1 if i in axes else 1) for i in range(3)))
    return y, y[at].data_ptr(), strides


def stream():
    return torch.cuda.current_stream().cuda_stream


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G,K,L,g", ROWS)
def test_attention(G, K, L, g, dtype):
    """The same numbers by the same kernels: bit for bit."""
    rng = np.random.default_rng(G + L)
    B, H, D, n = 6, 2, 64, 1 + K * L
    c, m = both(120, H, D, B, 16, 64, dtype)
    grow(c, m, rng, [0], [333], dtype)
    fork(c, m, [0] * 5, [1, 2, 3, 4, 5])
    grow(c, m, rng, list(range(B)), [9, 40, 70, 0, 1, 130], dtype)
    grow(c, m, rng, list(range(B)), [n] * B, dtype, keep=False)
    seqs, q = ints(range(B)), tokens(rng, B, n, H * g, D, dtype=dtype)
    alone, shared = c.attend(0, seqs, q, branches=K), c.attend_shared(0, seqs, q, G, branches=K, least_saved=0)
    # the workspace holds another call's sums
    c.attend_shared(0, seqs, 3 * q, G, branches=K, least_saved=0)
    for axes in BACK:
        kept, at, strides = backwards(q, axes)
        out = torch.full_like(q, 7.0)
        assert cache._lib.mds_cache_attend(c.ctx, 0, seqs.data_ptr(), None, at, strides, out.data_ptr(), H * g, n, K, 0,
                                           0, D ** -0.5, B, stream()) == 0
        assert torch.equal(out, alone), axes
        out.fill_(7.0)
        assert cache._lib.mds_cache_attend_shared(c.ctx, 0, seqs.data_ptr(), None, at, strides, out.data_ptr(), H * g, n,
                                                  K, G, D ** -0.5, 0, B, stream()) == 0
        assert torch.equal(out, shared), axes
    assert c.status() == (0, "ok")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rotation_and_append(dtype):
    rng = np.random.default_rng(3)
    B, H, D, n = 3, 2, 64, 5
    c, m = both(40, H, D, B, 8, 16, dtype)
    grow(c, m, rng, list(range(B)), [9, 16, 30], dtype)
    r, seqs = cache.Rotary(48, magnitude=1.25), ints(range(B))
    q, k, v = tokens(rng, B, n, 6, D, dtype=dtype), *(tokens(rng, B, n, H, D, dtype=dtype) for _ in range(2))
    c.reserve(seqs, n)
    want = c.append_rotated(0, seqs, k, v, r, branches=2, q=q)
    stored = c.read(0, seqs, None, 35)
    for axes in BACK:
        (kq, aq, sq), (kk, ak, sk), (kv, av, sv) = (backwards(x, axes) for x in (q, k, v))
        c.append(0, seqs, 0 * k, 0 * v)
        out = torch.full_like(q, 7.0)
        assert cache._lib.mds_cache_append_rotated(c.ctx, 0, seqs.data_ptr(), None, ctypes.byref(r.struct), ak, sk, av, sv,
                                                   aq, sq, out.data_ptr(), 6, n, 2, B, stream()) == 0
        assert torch.equal(out, want), axes
        for a, b in zip(c.read(0, seqs, None, 35), stored):
            assert torch.equal(a, b), axes
        out.fill_(7.0)
        assert cache._lib.mds_cache_rotate(c.ctx, seqs.data_ptr(), None, ctypes.byref(r.struct), aq, sq, out.data_ptr(), 6,
                                           n, 2, B, stream()) == 0
        assert torch.equal(out, want), axes
    assert c.status() == (0, "ok")
