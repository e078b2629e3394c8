"""Attention at the ends of its scores' range, in the kernel for many rows and
in the one for few, against 64 bits on what the cache stores."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

from cache_model import attend, visible  # noqa: E402
from test_gpu_cache import DEV, DT, both, bound, grow, ints, tokens, wide  # noqa: E402

# branches, length, query heads on one: 17, 72 and 132 rows, and 9 (the kernel for few)
ROWS = [(1, 16, 1), (2, 4, 8), (8, 4, 4), (2, 4, 1)]


def prompt(c, m, k, v):
    """Store k and v [n][D] as sequence 0's first tokens, one head."""
    n = k.shape[0]
    k, v = (torch.as_tensor(x, device=DEV)[None, :, None].to(c.dtype) for x in (k, v))
    m.reserve([0], [n])
    c.reserve(ints([0]), n)
    m.append(0, [0], [n], wide(k), wide(v))
    c.append(0, ints([0]), k, v)
    m.commit([0], [n - 1])
    c.commit(ints([0]), ints([n - 1]), length=n - 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [20, 31, 40, 60])
@pytest.mark.parametrize("K,L,group", ROWS)
def test_large_scores_pick_their_token(K, L, group, size, dtype):
    """Scores of about 2^size: a row's output is the value of the token that
    dominates it, whose score grows from tile to tile.  Queries look along one
    direction or against it, at sizes that differ by row."""
    rng = np.random.default_rng(size)
    D, n, T = 128, 1 + K * L, 700
    c, m = both(kv_heads=1, head_dim=D, max_pages=60, page_tokens=16, dtype=dtype)
    u = rng.choice([-1.0, 1.0], D)
    k = rng.choice([-0.125, 0.125], (T, D))
    for i, at in enumerate(range(60, T, 128)):          # one larger pair of keys a tile
        k[at], k[at + 7] = u * 2.0 ** (i / 2 - 3), -u * 2.0 ** (i / 2 - 3)
    k *= 2.0 ** (size // 2)
    prompt(c, m, k, rng.standard_normal((T, D)))
    grow(c, m, rng, [0], [n], dtype, keep=False)
    sign = rng.choice([-1.0, 1.0], (1, n, group, 1)) * np.exp2(rng.integers(-2, 3, (1, n, group, 1)))
    q = torch.tensor(u * sign * 2.0 ** (size - size // 2), device=DEV).to(DT[dtype])
    o = c.attend(0, ints([0]), q, branches=K)
    kk, vv = m.get(0, 0, 0, T + n)
    want, _, big = attend(wide(q[0]), kk, vv, visible(n, K, T), D ** -0.5)
    assert big.min() > 2.0 ** (size - 2)
    # one weight is 1 and the others are below 2^-1000: the value itself
    np.testing.assert_array_equal(wide(o[0]), want)
    assert c.status() == (0, "ok")


@pytest.mark.parametrize("size", [100.0, 2e4, 3e4, 1e6, 1e12])
@pytest.mark.parametrize("K,L,group", ROWS)
def test_outputs_stay_between_the_values(K, L, group, size):
    """Queries and keys of one large magnitude in every dimension: weights
    that no rounding of the scores makes more than 1, so that an output lies
    between the least and the largest value of its dimension."""
    rng = np.random.default_rng(int(size))
    D, n, T = 128, 1 + K * L, 300
    c, m = both(kv_heads=1, head_dim=D, max_pages=30, page_tokens=16)
    prompt(c, m, rng.standard_normal((T, D)) * size, rng.standard_normal((T, D)))
    grow(c, m, rng, [0], [n], keep=False)
    q = torch.tensor(rng.standard_normal((1, n, group, D)) * size, device=DEV).bfloat16()
    o = wide(c.attend(0, ints([0]), q, branches=K))
    v = m.get(0, 0, 0, T + n)[1][:, 0]
    assert np.isfinite(o).all()
    # the normaliser's and the output's roundings: 2^-8 of a value
    room = 2.0 ** -8 * np.abs(v).max(0)
    assert (o <= v.max(0) + room).all() and (o >= v.min(0) - room).all()
    assert c.status() == (0, "ok")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K,L,group", ROWS)
def test_negative_scale(K, L, group, dtype):
    """A negative scale is the positive one on negated queries, bit for bit."""
    rng = np.random.default_rng(21)
    c, m = both(pages=40, kv_heads=1, head_dim=64, max_pages=40, page_tokens=16, dtype=dtype)
    grow(c, m, rng, [0], [333], dtype)
    grow(c, m, rng, [0], [1 + K * L], dtype, keep=False)
    q = tokens(rng, 1, 1 + K * L, group, 64, dtype=dtype)
    for window in (0, 100):
        a = c.attend(0, ints([0]), q, branches=K, window=window, scale=-0.25)
        assert torch.equal(a, c.attend(0, ints([0]), -q, branches=K, window=window, scale=0.25))
        n = 1 + K * L
        k, v = m.get(0, 0, 0, 333 + n)
        want, mag, big = attend(-wide(q[0]), k, v, visible(n, K, 333, window), 0.25)
        assert (np.abs(wide(a[0]) - want) <= bound(mag, big, want, 333 + n, 64, dtype)).all()


@pytest.mark.parametrize("K,L,group", ROWS)
def test_a_row_of_tiny_queries_changes_no_other(K, L, group):
    """Keys of 2^-14 and queries of 2^18, with and without a node whose
    queries are 2^-90: the other nodes' outputs are right either way."""
    rng = np.random.default_rng(22)
    D, n, T = 128, 1 + K * L, 200
    c, m = both(kv_heads=1, head_dim=D, max_pages=20, page_tokens=16)
    prompt(c, m, rng.standard_normal((T, D)) * 2.0 ** -14, rng.standard_normal((T, D)))
    grow(c, m, rng, [0], [n], keep=False)
    q = torch.tensor(rng.standard_normal((1, n, group, D)) * 2.0 ** 18, device=DEV).bfloat16()
    first = c.attend(0, ints([0]), q, branches=K, window=100)
    k, v = m.get(0, 0, 0, T + n)
    want, mag, big = attend(wide(q[0]), k, v, visible(n, K, T, 100), D ** -0.5)
    assert (np.abs(wide(first[0]) - want) <= bound(mag, big, want, T + n, D, "bf16")).all()
    q[0, n // 2] *= 2.0 ** -108
    again = c.attend(0, ints([0]), q, branches=K, window=100)
    want, mag, big = attend(wide(q[0]), k, v, visible(n, K, T, 100), D ** -0.5)
    assert (np.abs(wide(again[0]) - want) <= bound(mag, big, want, T + n, D, "bf16")).all()
    assert c.status() == (0, "ok")


@pytest.mark.parametrize("score", [-12, -27, -38])
@pytest.mark.parametrize("K,L,group", ROWS)
def test_small_values_under_low_scores(K, L, group, score):
    """Scores of about `score` (e^-38 is 2^-55) for every token, values of
    2^-98: the weights' size must not push them out of 32 bits."""
    rng = np.random.default_rng(23)
    D, n, T = 64, 1 + K * L, 300
    c, m = both(kv_heads=1, head_dim=D, max_pages=30, page_tokens=16)
    k = 0.1 * rng.standard_normal((T + n, D))
    k[:, 0] = score
    v = rng.standard_normal((T + n, D)) * 2.0 ** -98
    prompt(c, m, k[:T], v[:T])
    kk, vv = (torch.tensor(x[None, T:, None], device=DEV).bfloat16() for x in (k, v))
    m.reserve([0], [n])
    c.reserve(ints([0]), n)
    m.append(0, [0], [n], wide(kk), wide(vv))
    c.append(0, ints([0]), kk, vv)
    q = torch.tensor(0.1 * rng.standard_normal((1, n, group, D)), device=DEV)
    q[..., 0] = 1.0
    q = q.bfloat16()
    o = c.attend(0, ints([0]), q, branches=K, scale=1.0)
    kk, vv = m.get(0, 0, 0, T + n)
    want, mag, big = attend(wide(q[0]), kk, vv, visible(n, K, T), 1.0)
    assert (np.abs(wide(o[0]) - want) <= bound(mag, big, want, T + n, D, "bf16") - 1e-30).all()
    assert c.status() == (0, "ok")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [50, 300])
@pytest.mark.parametrize("K,L,group", ROWS)
def test_scores_far_below_zero(K, L, group, T, dtype):
    """Every score of a row is below -2^100: the largest of them picks its token."""
    rng = np.random.default_rng(24)
    D, n = 64, 1 + K * L
    c, m = both(kv_heads=1, head_dim=D, max_pages=30, page_tokens=16, dtype=dtype)
    u = rng.choice([-1.0, 1.0], D)
    k = -u * 2.0 ** 50 * rng.choice([2.0, 3.0, 4.0], (T + n, 1))
    k[T // 2] = -u * 2.0 ** 50
    v = rng.standard_normal((T + n, D))
    prompt(c, m, k[:T], v[:T])
    kk, vv = (torch.tensor(x[None, T:, None], device=DEV).to(DT[dtype]) for x in (k, v))
    m.reserve([0], [n])
    c.reserve(ints([0]), n)
    m.append(0, [0], [n], wide(kk), wide(vv))
    c.append(0, ints([0]), kk, vv)
    q = torch.tensor(u * np.exp2(rng.integers(50, 54, (1, n, group, 1))), device=DEV).to(DT[dtype])
    o = c.attend(0, ints([0]), q, branches=K)
    want = m.get(0, 0, T // 2, 1)[1][0]
    np.testing.assert_array_equal(wide(o[0]), np.broadcast_to(want, (n, group, D)))
    assert c.status() == (0, "ok")
