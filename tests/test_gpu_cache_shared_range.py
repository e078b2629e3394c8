"""Shared prefixes of which rows see scores beyond the floats' range."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

from paper_2410_18234_gb300 import cache  # noqa: E402
from test_gpu_cache_shared import DEV, ints  # noqa: E402


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [2, 6, 16])
@pytest.mark.parametrize("K,L", [(1, 0), (2, 4)])
def test_tiles_without_a_finite_score(G, K, L, D):
    """The prefix's first tile has scores below every float for every row, the
    rest scores of -800: the outputs are the rest's values' mean.  The weights
    are 1, so only the sums and the output round."""
    rng = np.random.default_rng(G)
    n = 1 + K * L
    c = cache.Cache(1, 8 + 2 * G, 1, D, G, 8, page_tokens=64)
    k = torch.full((1, 300, 1, D), -1e30 * 0.125, device=DEV)
    k[:, 128:] = -1e-28 * 0.78125
    v = torch.tensor(rng.standard_normal((1, 300, 1, D)), device=DEV)
    v[:, :128] = 1000.0
    c.reserve(ints([0]), 300)
    c.append(0, ints([0]), k.bfloat16(), v.bfloat16())
    c.commit(ints([0]), ints([299]), length=299)
    c.fork(ints([0] * (G - 1)), ints(range(1, G)))
    seqs = ints(range(G))
    c.reserve(seqs, n)
    own = torch.tensor(rng.standard_normal((G, n, 1, D)), device=DEV).bfloat16()
    c.append(0, seqs, k[:, 128:129].expand(G, n, 1, D).bfloat16(), own)
    q = torch.full((G, n, 4, D), 1e30, device=DEV, dtype=torch.bfloat16)
    values = c.read(0, seqs, None, 300 + n)[1].double()[:, :, 0]
    alone, shared = c.attend(0, seqs, q, branches=K), c.attend_shared(0, seqs, q, G, branches=K, least_saved=0)
    for b in range(G):
        for i in range(n):
            first = 1 + (i - 1) // max(L, 1) * L
            seen = list(range(128, 301)) + ([300 + j for j in range(first, i + 1)] if i else [])
            want = values[b, seen].mean(0)
            # 32-bit sums of values below 5, then half a step of the output
            tol = 2.0 ** -8 * want.abs() + len(seen) * 2.0 ** -24 * 8
            for o in (alone, shared):
                assert ((o[b, i].double() - want).abs() <= tol).all(), (b, i)
    assert c.status() == (0, "ok")
