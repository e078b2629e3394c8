"""The key/value cache on the GPU against the 64-bit model of
tests/cache_model.py: stored values, lengths and page tables exactly, the
attention within bounds that its roundings give."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

from cache_model import Model, attend, quantise, visible  # noqa: E402
from paper_2410_18234_gb300 import cache, mds  # noqa: E402

DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def wide(t):
    return t.double().cpu().numpy()


def tokens(rng, *shape, dtype="bf16"):
    """Normals with a magnitude per token and an offset per dimension."""
    x = rng.standard_normal(shape) * np.exp(rng.standard_normal((*shape[:-2], 1, 1))) + 2 * rng.standard_normal(shape[-1])
    return torch.tensor(x, device=DEV).to(DT[dtype])


def same_state(c, m):
    assert c.lens.tolist() == m.lens
    np.testing.assert_array_equal(c.table.cpu().numpy(), m.table())


def same_values(c, m, seqs):
    n = max(m.lens[q] for q in seqs)
    if n == 0:
        return
    k, v = c.read(None, ints(seqs), None, n, counts=ints([m.lens[q] for q in seqs]))
    for b, q in enumerate(seqs):
        for layer in range(m.layers):
            want = m.get(q, layer, 0, m.lens[q])
            np.testing.assert_array_equal(wide(k[layer, b, :m.lens[q]]), want[0])
            np.testing.assert_array_equal(wide(v[layer, b, :m.lens[q]]), want[1])
            assert not k[layer, b, m.lens[q]:].any() and not v[layer, b, m.lens[q]:].any()


def both(layers=1, pages=64, kv_heads=2, head_dim=64, max_seqs=6, max_pages=16, page_tokens=16, dtype="bf16"):
    c = cache.Cache(layers, pages, kv_heads, head_dim, max_seqs, max_pages, page_tokens=page_tokens, dtype=dtype)
    return c, Model(layers, pages, kv_heads, head_dim, max_seqs, max_pages, page_tokens)


def grow(c, m, rng, seqs, counts, dtype="bf16", keep=None):
    """Reserve, append random tokens to every layer, commit `keep` (all)."""
    n = max(max(counts), 1)
    assert m.reserve(seqs, counts) == []
    c.reserve(ints(seqs), n, counts=ints(counts))
    for layer in range(m.layers):
        k, v = (tokens(rng, len(seqs), n, m.H, m.D, dtype=dtype) for _ in range(2))
        m.append(layer, seqs, counts, wide(k), wide(v))
        c.append(layer, ints(seqs), k, v, counts=ints(counts))
    if keep is None:
        m.commit(seqs, [x - 1 for x in counts])
        c.commit(ints(seqs), ints([x - 1 for x in counts]), length=n - 1)


# ------------------------------------------------------------ the quantiser


@pytest.mark.parametrize("head_dim", [64, 128])
def test_quantiser_edges(head_dim):
    """Blocks at the scale's boundaries, of tiny and huge numbers, of zeros."""
    rng = np.random.default_rng(0)
    rows = []
    for top in (0.0, 1.0, 448.0, 448.0000305, 447.99, 449.0, 2.0 ** -130, 1.5e-38, 1e-40, 3.4e38, 3.0e38, 2.0 ** -8 * 1.75,
                2.0 ** -8 * 1.7500001):
        x = rng.standard_normal((16, head_dim))
        x = x / np.abs(x).max() * top * np.exp2(-rng.integers(0, 24, (16, 1)))
        x[0, 0] = top
        rows.append(x)
    x = torch.tensor(np.concatenate(rows)[None, :, None], dtype=torch.float32, device=DEV)
    c, _ = both(kv_heads=1, head_dim=head_dim, page_tokens=32, dtype="f32")
    seqs = ints([3])
    c.reserve(seqs, x.shape[1])
    c.append(0, seqs, x, -x)
    c.commit(seqs, ints([x.shape[1] - 1]), length=x.shape[1] - 1)
    k, v = c.read(0, seqs, None, x.shape[1])
    for i in range(len(rows)):
        want = quantise(wide(x[0, 16 * i:16 * i + 16, 0]))
        np.testing.assert_array_equal(wide(k[0, 16 * i:16 * i + 16, 0]), want)
        np.testing.assert_array_equal(wide(v[0, 16 * i:16 * i + 16, 0]), -want)
    assert c.status() == (0, "ok")


def test_non_finite_inputs_are_absorbed_and_reported():
    c, _ = both(dtype="f32")
    x = torch.randn(1, 20, 2, 64, device=DEV)
    x[0, 3, 0, 5], x[0, 4, 0, 6], x[0, 5, 1, 7] = float("nan"), float("inf"), float("-inf")
    seqs = ints([0])
    c.reserve(seqs, 20)
    c.append(0, seqs, x, x)
    k, _ = c.read(0, seqs, None, 20)
    for h in range(2):
        np.testing.assert_array_equal(wide(k[0, :16, h]), quantise(wide(x[0, :16, h])))
    assert torch.isfinite(k).all()
    assert c.status()[0] == cache.MDS_ST_NONFINITE
    assert c.status()[0] == 0


# ------------------------------------------------------------ pages


@pytest.mark.parametrize("page_tokens,head_dim,kv_heads,dtype", [(16, 64, 2, "bf16"), (32, 128, 1, "f32"),
                                                                 (64, 64, 3, "bf16"), (128, 128, 2, "bf16")])
def test_random_steps(page_tokens, head_dim, kv_heads, dtype):
    """A random walk over every operation: lengths, page tables and values."""
    rng = np.random.default_rng(page_tokens)
    c, m = both(layers=2, pages=40, kv_heads=kv_heads, head_dim=head_dim, max_seqs=6, max_pages=12,
                page_tokens=page_tokens, dtype=dtype)
    for step in range(40):
        live = [q for q in range(6) if m.lens[q]]
        empty = [q for q in range(6) if not m.rows[q]]
        kind = rng.choice(["grow", "tree", "tree", "fork", "truncate", "free"])
        if kind == "grow":
            seqs = list(rng.permutation(6)[:3])
            counts = [int(rng.integers(0, 2 * page_tokens)) for _ in seqs]
            used = sum(r > 0 for r in m.ref) + sum(n // page_tokens + 2 for n in counts)
            if used > 40 or any(m.lens[q] + n > 8 * page_tokens for q, n in zip(seqs, counts)):
                continue
            grow(c, m, rng, seqs, counts, dtype)
        elif kind == "tree":
            K, L = [(2, 4), (4, 5), (1, 3), (3, 17), (2, 1)][rng.integers(5)]
            n = 1 + K * L
            seqs = [q for q in range(6) if m.lens[q] + n <= 12 * page_tokens][:4] + [-1]
            used = sum(len(set(r)) for r in m.rows) + len(seqs) * (n // page_tokens + 2)
            if used > 40:
                continue
            grow(c, m, rng, seqs, [n] * len(seqs), dtype, keep=False)
            drafts = rng.integers(0, 3, (len(seqs), K, L))
            accept = rng.integers(-1, L + 1, len(seqs))
            out = np.full((len(seqs), L + 1), 7)
            for b in range(len(seqs)):
                out[b, :max(accept[b], 0)] = drafts[b, rng.integers(K), :max(accept[b], 0)]
            m.commit(seqs, accept.tolist(), K, L, drafts, out)
            c.commit(ints(seqs), ints(accept), branches=K, length=L, draft_tokens=ints(drafts), out_tokens=ints(out))
        elif kind == "fork" and live and empty:
            m.fork(live[:1], empty[:1])
            c.fork(ints(live[:1]), ints(empty[:1]))
        elif kind == "truncate" and live:
            to = [int(rng.integers(0, m.lens[q] + 5)) for q in live]
            m.truncate(live, to)
            c.truncate(ints(live), ints(to))
        elif kind == "free" and len(live) > 3:
            m.free(live[:2])
            c.free(ints(live[:2]))
        same_state(c, m)
    same_values(c, m, list(range(6)))
    assert c.status() == (0, "ok")


def test_fork_copies_on_write():
    """Forks share pages; who writes first gets a copy, and the other's
    tokens stay; two forks that reserve in one call both get one."""
    rng = np.random.default_rng(5)
    c, m = both(layers=3, pages=32, page_tokens=32)
    grow(c, m, rng, [0], [75])
    m.fork([0, 0], [2, 4])
    c.fork(ints([0, 0]), ints([2, 4]))
    same_state(c, m)
    for seqs in ([2, 4], [0]):
        grow(c, m, rng, seqs, [9] * len(seqs))
        same_state(c, m)
        same_values(c, m, [0, 2, 4])
    c.free(ints([0, 4]))
    m.free([0, 4])
    same_state(c, m)
    same_values(c, m, [2])
    # a sequence cut back into a shared page copies it too
    m.fork([2], [1])
    c.fork(ints([2]), ints([1]))
    m.truncate([1], [40])
    c.truncate(ints([1]), ints([40]))
    grow(c, m, rng, [1], [3])
    same_state(c, m)
    same_values(c, m, [1, 2])
    assert c.status() == (0, "ok")


def test_too_few_pages():
    """The list's order decides who gets pages; the others keep what they
    had, and what they append behind it is not stored."""
    rng = np.random.default_rng(6)
    c, m = both(pages=9, page_tokens=16, max_pages=8)
    grow(c, m, rng, [0, 1], [40, 40])                       # three pages each
    assert m.reserve([1, 0, 2], [40, 40, 16]) == [0, 2]     # 2 of 3, then 2 and 1 of 1
    c.reserve(ints([1, 0, 2]), 40, counts=ints([40, 40, 16]))
    assert c.status()[0] == cache.MDS_ST_NOPAGES
    same_state(c, m)
    x = tokens(rng, 1, 40, 2, 64)
    c.append(0, ints([0]), x, x)                            # slots 40..47 exist
    assert c.status()[0] == cache.MDS_ST_BADSEQ
    c.reserve(ints([3]), 129)                               # longer than a page table
    assert c.status()[0] == cache.MDS_ST_NOPAGES
    same_state(c, m)
    c.fork(ints([0]), ints([1]))                            # not empty
    assert c.status()[0] == cache.MDS_ST_BADSEQ
    c.reserve(ints([6]), 1)                                 # no such sequence
    assert c.status()[0] == cache.MDS_ST_BADSEQ
    same_state(c, m)
    c.commit(ints([5]), ints([0]))                          # nothing reserved
    assert c.status()[0] == cache.MDS_ST_BADSEQ
    same_state(c, m)


def test_commit_of_tokens_of_no_branch():
    rng = np.random.default_rng(7)
    c, m = both()
    grow(c, m, rng, [0], [20])
    grow(c, m, rng, [0], [9], keep=False)
    c.commit(ints([0]), ints([2]), branches=2, length=4, draft_tokens=ints([[[1, 2, 3, 4], [5, 6, 7, 8]]]),
             out_tokens=ints([[5, 2, 0, -1, -1]]))
    m.commit([0], [2])
    assert c.status()[0] == cache.MDS_ST_BADTOKEN
    same_state(c, m)
    same_values(c, m, [0])


def test_pools_beyond_32_bit_offsets():
    """The last layer of a pool of more than 2^32 bytes, and its last pages."""
    rng = np.random.default_rng(8)
    c = cache.Cache(9, 4100, 8, 128, 3, 2100, page_tokens=64)
    assert c.memory.numel() > 9 * 4100 * 2 * 8 * 64 * 128 > 2 ** 32
    c.reserve(ints([0, 1]), 64 * 2040)                       # the low pages
    k, v = (tokens(rng, 1, 130, 8, 128) for _ in range(2))
    c.reserve(ints([2]), 130)
    assert int(c.table[2].max()) >= 4080
    c.append(8, ints([2]), k, v)
    got = c.read(8, ints([2]), None, 130)
    q = tokens(rng, 1, 1, 8, 128)
    c.commit(ints([2]), ints([128]), length=129)
    o = c.attend(8, ints([2]), q)
    for x, y in zip((k, v), got):
        for b in range(0, 130, 16):
            np.testing.assert_array_equal(wide(y[0, b:b + 16, 3]), quantise(wide(x[0, b:b + 16, 3])))
    want, mag, _ = attend(wide(q[0]), wide(got[0][0]), wide(got[1][0]), np.ones((1, 130), bool), 128 ** -0.5)
    assert (np.abs(wide(o[0]) - want) <= 2.0 ** -7 * mag).all()
    assert c.status() == (0, "ok")


# ------------------------------------------------------------ attention


def bound(mag, big, o, T, D, dtype):
    """Largest error of an output: roundings of scores (32-bit sums of D exact
    products, their scaling, the exponential's argument), of weights in the
    sum and the normaliser, of the 32-bit sums over T tokens, of the output."""
    u = 2.0 ** -24
    score = (D + 4 + (4 if dtype == "f32" else 0)) * u * big * np.log2(np.e) + 4 * u * big
    weight = 2.0 ** -9 if dtype == "bf16" else 8 * u
    out = 2.0 ** -9 if dtype == "bf16" else u
    return mag * (2 * score + 2 * weight + 2 * (T + 16) * u) + np.abs(o) * out + 1e-30


def check_attend(c, m, rng, seqs, Hq, K, L, dtype, window=0, sinks=0, counts=None, layer=0, scale=None):
    n = 1 + K * L
    grow(c, m, rng, seqs, [n] * len(seqs), dtype, keep=False)
    q = 1.5 * tokens(rng, len(seqs), n, Hq, m.D, dtype=dtype)
    o = c.attend(layer, ints(seqs), q, branches=K, window=window, sinks=sinks, scale=scale,
                 counts=None if counts is None else ints(counts))
    assert o.dtype == DT[dtype] and o.shape == q.shape
    s = m.D ** -0.5 if scale is None else scale
    for b, x in enumerate(seqs):
        live = 0 if x < 0 else n if counts is None else counts[b]
        assert not o[b, live:].any()
        if live == 0:
            continue
        T = m.lens[x] + n
        k, v = m.get(x, layer, 0, T)
        see = visible(n, K, m.lens[x], window, sinks)
        want, mag, big = attend(wide(q[b]), k, v, see, s)
        err = np.abs(wide(o[b]) - want)[:live]
        lim = bound(mag, big, want, T, m.D, dtype)[:live]
        assert (err <= lim).all(), (b, x, float((err / lim).max()))
    m.commit(seqs, [-1] * len(seqs))
    c.commit(ints(seqs), ints([-1] * len(seqs)), branches=K, length=L)
    assert c.status() == (0, "ok")
    return o


SHAPES = [  # head_dim, page_tokens, kv_heads, group
    (64, 16, 2, 1), (128, 64, 2, 4), (128, 32, 1, 16), (64, 128, 3, 5), (128, 16, 1, 64), (64, 64, 1, 8)]
TREES = [(1, 0), (2, 4), (8, 4), (1, 7), (3, 1), (1, 40), (4, 33)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("head_dim,page_tokens,kv_heads,group", SHAPES)
def test_attend(head_dim, page_tokens, kv_heads, group, dtype):
    """Trees, chains and single tokens over empty, short, odd and longer
    sequences in one call."""
    rng = np.random.default_rng(head_dim + page_tokens + group)
    c, m = both(layers=2, pages=3000 // page_tokens + 40, kv_heads=kv_heads, head_dim=head_dim, max_seqs=7,
                max_pages=1024 // page_tokens + 4, page_tokens=page_tokens, dtype=dtype)
    grow(c, m, rng, [0, 1, 2, 3, 4, 5], [1, 15, 129, 0, 700, 256], dtype)
    for K, L in TREES:
        check_attend(c, m, rng, [5, 0, 3, -1, 4, 1, 2], kv_heads * group, K, L, dtype, layer=1)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (3, 0), (16, 4), (100, 3), (128, 128), (130, 17), (500, 0),
                                          (5000, 4), (64, 1000)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_window_and_sinks(window, sinks, dtype):
    """Windows shorter than a branch, than a block, than a tile, longer than
    the cache; sinks inside and outside them."""
    rng = np.random.default_rng(window + sinks)
    c, m = both(pages=200, kv_heads=2, head_dim=64, max_pages=40, page_tokens=32, dtype=dtype)
    grow(c, m, rng, [0, 1, 2, 3], [0, 33, 600, 1023], dtype)
    for K, L in [(1, 0), (2, 4), (3, 6), (1, 150)]:
        check_attend(c, m, rng, [3, 0, 2, 1], 6, K, L, dtype, window, sinks)


def test_live_counts():
    """Rows of tokens that are not live are zeros; so is an unused place."""
    rng = np.random.default_rng(9)
    c, m = both(pages=100, kv_heads=2, head_dim=128, max_pages=12, page_tokens=64)
    grow(c, m, rng, [0, 1, 2, 3], [0, 33, 300, 511])
    check_attend(c, m, rng, [3, 0, 2, -1, 1], 8, 1, 50, "bf16", counts=[51, 1, 17, 51, 0])
    check_attend(c, m, rng, [3, 0, 2, -1, 1], 8, 3, 4, "bf16", counts=[5, 0, 13, 2, 1])


def test_scale_and_outliers():
    """Scores of a few hundred (one token dominates), blocks of values of very
    different magnitude, keys of very different scales."""
    rng = np.random.default_rng(10)
    for dtype in ("bf16", "f32"):
        c, m = both(pages=100, kv_heads=1, head_dim=64, max_pages=20, page_tokens=32, dtype=dtype)
        n = 500
        size = np.exp2(rng.integers(-40, 40, (1, n, 1, 1)).astype(float))
        k = tokens(rng, 1, n, 1, 64, dtype=dtype)
        v = (tokens(rng, 1, n, 1, 64, dtype="f32") * torch.tensor(size, device=DEV)).to(DT[dtype])
        m.reserve([0], [n])
        c.reserve(ints([0]), n)
        m.append(0, [0], [n], wide(k), wide(v))
        c.append(0, ints([0]), k, v)
        m.commit([0], [n - 1])
        c.commit(ints([0]), ints([n - 1]), length=n - 1)
        for scale in (0.0, 0.01, 0.125, 3.0):
            check_attend(c, m, rng, [0], 4, 2, 3, dtype, scale=scale)


def test_split_sequences_join():
    """One long sequence and one head: every SM holds a piece of each row."""
    rng = np.random.default_rng(11)
    c, m = both(pages=700, kv_heads=1, head_dim=128, max_pages=640, page_tokens=64)
    grow(c, m, rng, [0, 1], [40001, 77])
    for K, L in [(1, 0), (8, 4)]:
        a = check_attend(c, m, rng, [1, 0], 4, K, L, "bf16")
        assert a.shape[1] == 1 + K * L


def test_results_do_not_depend_on_the_launch():
    """The same call again and again, bit for bit, and on another stream."""
    rng = np.random.default_rng(12)
    c, m = both(pages=900, kv_heads=2, head_dim=128, max_pages=400, page_tokens=64)
    grow(c, m, rng, [0, 1, 2], [20001, 3, 777])
    seqs, n = ints([2, 0, 1]), 33
    c.reserve(seqs, n)
    k, v = (tokens(rng, 3, n, 2, 128) for _ in range(2))
    c.append(0, seqs, k, v)
    q = tokens(rng, 3, n, 8, 128)
    first = c.attend(0, seqs, q, branches=8)
    side = torch.cuda.Stream()
    for i in range(20):
        if i % 2:
            side.wait_stream(torch.cuda.current_stream())
            again = c.attend(0, seqs, q, branches=8, stream=side)
            torch.cuda.current_stream().wait_stream(side)
        else:
            again = c.attend(0, seqs, q, branches=8)
        assert torch.equal(first, again), i


def test_strided_inputs():
    """Queries, keys and values as slices of one fused projection."""
    rng = np.random.default_rng(13)
    for order in ("token", "head"):
        c, m = both(pages=40, kv_heads=2, head_dim=64, max_pages=16, page_tokens=16)
        grow(c, m, rng, [0, 1], [20, 50])
        B, n, Hq = 2, 9, 6
        if order == "token":
            fused = tokens(rng, B, n, Hq + 4, 64)
        else:   # heads outermost
            fused = tokens(rng, Hq + 4, B, n, 64).permute(1, 2, 0, 3)
        q, k, v = fused[:, :, :Hq], fused[:, :, Hq:Hq + 2], fused[:, :, Hq + 2:]
        assert not q.is_contiguous()
        m.reserve([0, 1], [n, n])
        c.reserve(ints([0, 1]), n)
        c.append(0, ints([0, 1]), k, v)
        got = c.read(0, ints([0, 1]), None, 60)
        a = c.attend(0, ints([0, 1]), q, branches=2)
        c.append(0, ints([0, 1]), k.contiguous(), v.contiguous())
        for x, y in zip(got, c.read(0, ints([0, 1]), None, 60)):
            assert torch.equal(x, y)
        assert torch.equal(a, c.attend(0, ints([0, 1]), q.contiguous(), branches=2))


def test_rows_of_queries_that_are_not_finite():
    """A query with a NaN gives NaN in its own row and no other."""
    rng = np.random.default_rng(14)
    c, m = both(pages=40, kv_heads=2, head_dim=64, max_pages=16, page_tokens=16)
    grow(c, m, rng, [0], [100])
    grow(c, m, rng, [0], [9], keep=False)
    q = tokens(rng, 1, 9, 4, 64)
    want = c.attend(0, ints([0]), q, branches=2)
    q[0, 4, 2, 7] = float("nan")
    got = c.attend(0, ints([0]), q, branches=2)
    assert torch.isnan(got[0, 4, 2]).all()
    got[0, 4, 2] = want[0, 4, 2]
    assert torch.equal(got, want)


def test_step_in_a_graph():
    """reserve, append, attend and commit captured once and replayed."""
    rng = np.random.default_rng(15)
    c, m = both(pages=60, kv_heads=2, head_dim=64, max_pages=16, page_tokens=16)
    grow(c, m, rng, [0, 1], [20, 50])
    K, L, n = 2, 4, 9
    seqs, accept, q = ints([0, 1]), ints([0, 0]), tokens(rng, 2, n, 4, 64)
    k, v = (tokens(rng, 2, n, 2, 64) for _ in range(2))
    drafts, out = ints(np.zeros((2, K, L))), ints(np.zeros((2, L + 1)))
    o = torch.empty_like(q)

    def step():
        c.reserve(seqs, n)
        c.append(0, seqs, k, v)
        c.attend(0, seqs, q, branches=K, out=o)
        c.commit(seqs, accept, branches=K, length=L, draft_tokens=drafts, out_tokens=out)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for i in range(6):
        for x in (k, v, q):
            x.copy_(tokens(rng, *x.shape))
        d = rng.integers(0, 2, (2, K, L))
        a = rng.integers(0, L + 1, 2)
        e = np.full((2, L + 1), 9)
        for b in range(2):
            e[b, :a[b]] = d[b, rng.integers(K), :a[b]]
        accept.copy_(ints(a))
        drafts.copy_(ints(d))
        out.copy_(ints(e))
        graph.replay()
        m.reserve([0, 1], [n, n])
        m.append(0, [0, 1], [n, n], wide(k), wide(v))
        for b in range(2):
            see = visible(n, K, m.lens[b])
            kk, vv = m.get(b, 0, 0, m.lens[b] + n)
            want, mag, big = attend(wide(q[b]), kk, vv, see, 64 ** -0.5)
            assert (np.abs(wide(o[b]) - want) <= bound(mag, big, want, m.lens[b] + n, 64, "bf16")).all()
        m.commit([0, 1], a.tolist(), K, L, d, e)
        same_state(c, m)
    same_values(c, m, [0, 1])


# ------------------------------------------------------------ refusals


def test_refusals():
    c, _ = both(layers=2)
    seqs = ints([0, 1])
    x = torch.zeros(2, 3, 2, 64, dtype=torch.bfloat16, device=DEV)
    q = torch.zeros(2, 3, 4, 64, dtype=torch.bfloat16, device=DEV)

    def refused(code, fn, *a, **kw):
        with pytest.raises(mds.MdsError) as e:
            fn(*a, **kw)
        assert e.value.code == code

    refused(mds.MDS_ESHAPE, c.append, 2, seqs, x, x)                       # no such layer
    refused(mds.MDS_ESHAPE, c.append, -1, seqs, x, x)
    refused(mds.MDS_EINVAL, c.append, 0, seqs, x.float(), x.float())       # another type
    refused(mds.MDS_EINVAL, c.append, 0, seqs, x.cpu(), x.cpu())
    refused(mds.MDS_EINVAL, c.append, 0, seqs.long(), x, x)
    refused(mds.MDS_ESHAPE, c.append, 0, seqs, x[:1], x[:1])
    refused(mds.MDS_ESHAPE, c.append, 0, seqs, x, x[:, :2])
    refused(mds.MDS_ESHAPE, c.append, 0, seqs, x, x, counts=ints([1]))
    refused(mds.MDS_EINVAL, c.append, 0, seqs, x.transpose(2, 3).contiguous().transpose(2, 3), x)
    odd = torch.zeros(2 * 3 * 2 * 64 + 1, dtype=torch.bfloat16, device=DEV)[1:].view(2, 3, 2, 64)
    refused(mds.MDS_EINVAL, c.append, 0, seqs, odd, odd)                   # rows off 16 bytes
    refused(mds.MDS_EINVAL, c.attend, 0, seqs, odd)
    refused(mds.MDS_ESHAPE, c.attend, 0, seqs, q, branches=0)
    refused(mds.MDS_ESHAPE, c.attend, 0, seqs, q[:, :2], branches=2)       # not 1 + 2 L nodes
    refused(mds.MDS_ESHAPE, c.attend, 0, seqs, q[:, :, :3])                # not a multiple of kv_heads
    refused(mds.MDS_EINVAL, c.attend, 0, seqs, q, window=-1)
    refused(mds.MDS_EINVAL, c.attend, 0, seqs, q, scale=float("nan"))
    refused(mds.MDS_EINVAL, c.attend, 0, seqs, q, out=q.float())
    refused(mds.MDS_ESHAPE, c.attend, 0, seqs, q, out=q[:, :2])
    refused(mds.MDS_ESHAPE, c.attend, 0, ints([0] * 1025), q[:1].expand(1025, -1, -1, -1))
    refused(mds.MDS_ESHAPE, c.reserve, seqs, -1)
    refused(mds.MDS_ESHAPE, c.commit, seqs, ints([0]))
    refused(mds.MDS_EINVAL, c.commit, seqs, ints([0, 0]), branches=2, length=2, draft_tokens=ints(np.zeros((2, 2, 2))))
    refused(mds.MDS_ESHAPE, c.fork, seqs, ints([2]))
    refused(mds.MDS_ESHAPE, c.read, 2, seqs, None, 3)
    assert c.status() == (0, "ok")
    for t in (c.reserve(seqs, 0), c.free(ints([]))):                       # nothing to do
        assert t is None
    assert c.attend(0, ints([]), q[:0]).shape == (0, 3, 4, 64)
