"""Attention for sequences that share a prefix, on the GPU against the 64-bit
model of tests/cache_model.py, within bounds that its roundings give."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

from cache_model import Model, attend, visible  # noqa: E402
from paper_2410_18234_gb300 import cache  # noqa: E402

DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def ints(x):
    return torch.tensor([int(i) for i in x], dtype=torch.int32, device=DEV)


def wide(t):
    return t.double().cpu().numpy()


def tokens(rng, *shape, dtype="bf16"):
    x = rng.standard_normal(shape) * np.exp(rng.standard_normal((*shape[:-2], 1, 1))) + 2 * rng.standard_normal(shape[-1])
    return torch.tensor(x, device=DEV).to(DT[dtype])


def both(pages, H, D, seqs, max_pages, page, dtype="bf16"):
    return (cache.Cache(1, pages, H, D, seqs, max_pages, page_tokens=page, dtype=dtype),
            Model(1, pages, H, D, seqs, max_pages, page))


def grow(c, m, rng, seqs, counts, dtype="bf16", keep=True):
    n = max(max(counts), 1)
    assert m.reserve(seqs, counts) == []
    c.reserve(ints(seqs), n, counts=ints(counts))
    k, v = (tokens(rng, len(seqs), n, m.H, m.D, dtype=dtype) for _ in range(2))
    m.append(0, seqs, counts, wide(k), wide(v))
    c.append(0, ints(seqs), k, v, counts=ints(counts))
    if keep:
        m.commit(seqs, [x - 1 for x in counts])
        c.commit(ints(seqs), ints([x - 1 for x in counts]), length=n - 1)


def fork(c, m, src, dst):
    m.fork(src, dst)
    c.fork(ints(src), ints(dst))


def bound(mag, big, o, T, D, dtype):
    """Largest error of an output.  Scores: 32-bit sums of D products, their
    scaling and the exponential's argument (and 22 bits of a 32-bit query).
    Weights: rounded to the query's type in the sum and in the normaliser.
    32-bit sums over T tokens; the two parts' factors and their sum (a few
    roundings more); the output's rounding."""
    u = 2.0 ** -24
    score = (D + 4 + (4 if dtype == "f32" else 0)) * u * big * np.log2(np.e) + 4 * u * big
    weight = 2.0 ** -8 if dtype == "bf16" else 8 * u
    out = 2.0 ** -8 if dtype == "bf16" else u
    return mag * (2 * score + 2 * weight + 2 * (T + 32) * u) * (1 + out) + np.abs(o) * out + 1e-30


def check(c, m, rng, seqs, G, Hq, K, L, dtype="bf16", counts=None, only=None, factor=1.5, scale=None,
          least=0):
    """One call on a new tree of every sequence."""
    n = 1 + K * L
    real = sorted({q for q in seqs if q >= 0})
    if real:
        grow(c, m, rng, real, [n] * len(real), dtype, keep=False)
    x = factor * tokens(rng, len(seqs), n, Hq + 1, m.D, dtype=dtype)
    q = x[:, :, 1:]                       # rows that are not the tensor's own
    out = torch.full((len(seqs), n, Hq, m.D), 7.0, device=DEV, dtype=DT[dtype])
    given = None if counts is None else ints(counts)
    o = c.attend_shared(0, ints(seqs), q, G, branches=K, counts=given, out=out, scale=scale, least_saved=least)
    assert o is out
    for b, s in enumerate(seqs):
        live = 0 if s < 0 else n if counts is None else min(max(counts[b], 0), n)
        assert not o[b, live:].any()
        if live == 0 or (only is not None and b not in only):
            continue
        T = m.lens[s] + n
        k, v = m.get(s, 0, 0, T)
        by = m.D ** -0.5 if scale is None else scale
        want, mag, big = attend(wide(q[b]), k, v, visible(n, K, m.lens[s]), by)
        if by < 0:   # the model's largest |q| |k| scale is one of a scale that is not negative
            big = attend(wide(q[b]), k, v, visible(n, K, m.lens[s]), -by)[2]
        err = np.abs(wide(o[b]) - want)[:live]
        lim = bound(mag, big, want, T, m.D, dtype)[:live]
        assert (err <= lim).all(), (b, s, float((err / lim).max()))
    # the same again, bit for bit, whatever the blocks' order
    assert torch.equal(c.attend_shared(0, ints(seqs), q, G, branches=K, counts=given, scale=scale, least_saved=least), o)
    m.commit(real, [-1] * len(real))
    c.commit(ints(real), ints([-1] * len(real)), branches=K, length=L)
    assert c.status() == (0, "ok")
    return o


TREES = [(1, 0), (2, 4), (8, 4), (1, 3), (1, 40), (4, 33)]
SHAPES = [  # D, page, H, g, dtype
    (64, 16, 2, 1, "bf16"), (128, 64, 2, 4, "bf16"), (128, 128, 1, 16, "bf16"), (64, 32, 3, 5, "bf16"),
    (128, 16, 1, 64, "bf16"), (64, 16, 2, 3, "f32"), (128, 128, 1, 8, "f32")]


@pytest.mark.parametrize("D,page,H,g,dtype", SHAPES)
def test_groups_of_forks(D, page, H, g, dtype):
    """Prefixes of 0, 1, short of, at and past a tile and longer, three
    sequences each, of which some went on and some did not."""
    rng = np.random.default_rng(D + page + g)
    pre = [0, 1, 127, 128, 129, 300, 517]
    c, m = both(4000 // page + 90, H, D, 21, 700 // page + 14, page, dtype)
    roots = list(range(0, 21, 3))
    grow(c, m, rng, roots, pre, dtype)
    held = [r for r, t in zip(roots, pre) if t]
    fork(c, m, held + held, [r + 1 for r in held] + [r + 2 for r in held])
    grow(c, m, rng, list(range(21)), [int(x) for x in rng.choice([0, 1, 17, 40, 150], 21)], dtype)
    order = [3 * i + j for i in (4, 0, 6, 2, 5, 1, 3) for j in (1, 0, 2)]
    for K, L in TREES:
        check(c, m, rng, order, 3, H * g, K, L, dtype)
    # one group of all: nothing is shared by every sequence
    check(c, m, rng, order, 21, H * g, 2, 4, dtype)
    # too little to save
    check(c, m, rng, order, 3, H * g, 2, 4, dtype, least=None)
    check(c, m, rng, order, 3, H * g, 1, 0, dtype, least=1 << 70)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_unused_places_dead_rows_and_strangers(dtype):
    """Groups with unused places in front, between and behind, with one live
    sequence or none, with sequences of no live node, with one that shares
    less or nothing, with nested forks."""
    rng = np.random.default_rng(11)
    c, m = both(300, 2, 64, 12, 50, 32, dtype)
    grow(c, m, rng, [0], [700], dtype)
    fork(c, m, [0, 0, 0], [1, 2, 3])
    grow(c, m, rng, [1], [260], dtype)
    fork(c, m, [1, 1], [4, 5])                       # share 960 tokens, with 0, 2, 3 only 700
    grow(c, m, rng, [0, 2, 4, 5, 6], [3, 40, 1, 200, 500], dtype)
    m.truncate([3], [150])
    c.truncate(ints([3]), ints([150]))
    grow(c, m, rng, [3], [600], dtype)               # shares 128 tokens with the others
    for K, L in [(1, 0), (2, 4), (1, 30)]:
        n = 1 + K * L
        check(c, m, rng, [4, 5, 1, 0, 2, -1], 3, 6, K, L, dtype)
        check(c, m, rng, [-1, 4, -1, 5, 0, -1, -1, -1], 4, 6, K, L, dtype)
        check(c, m, rng, [0, 2, 3, 1], 4, 6, K, L, dtype)
        check(c, m, rng, [6, 0, 2, 5], 2, 6, K, L, dtype)        # 6 shares nothing
        check(c, m, rng, [0, 1, 2, 4, 5, 6], 2, 6, K, L, dtype, counts=[0, n, n, 1, n + 3, -2])
        check(c, m, rng, [-1, -1, -1, -1], 2, 6, K, L, dtype)


def test_many_groups_and_groups_too_large():
    """Rows beyond the workspace: groups in several turns; and one group that
    no turn holds."""
    rng = np.random.default_rng(12)
    B, K, L, Hq = 64, 8, 4, 64
    c, m = both(B * 7 + 40, 8, 128, B, 12, 64)
    roots = list(range(0, B, 4))
    grow(c, m, rng, roots, [260 + 5 * i for i in range(16)])
    for j in (1, 2, 3):
        fork(c, m, roots, [r + j for r in roots])
    grow(c, m, rng, list(range(B)), [int(x) for x in rng.integers(0, 60, B)])
    check(c, m, rng, list(range(B)), 4, Hq, K, L, only=[0, 27, 28, 31, 62])
    check(c, m, rng, list(range(B)), 64, Hq, K, L, only=[0, 63])


def test_least_saved_is_an_exact_border():
    """Two of three sequences' 256 tokens of 2 heads: 2 * 256 * 256 bytes; one
    less and one more give the two ways' roundings."""
    rng = np.random.default_rng(17)
    c, m = both(60, 2, 64, 4, 12, 64)
    grow(c, m, rng, [0], [300])
    fork(c, m, [0, 0], [1, 2])
    grow(c, m, rng, [0, 1, 2], [5, 40, 90])
    saved = 2 * 256 * 2 * 2 * 64
    q = 0.02 * tokens(rng, 4, 1, 8, 64)       # weights that are spread over all tokens, so that the two ways differ
    seqs = ints([0, 1, 2, -1])
    c.reserve(seqs, 1)
    a, b, never, always = (c.attend_shared(0, seqs, q, 4, least_saved=x) for x in (saved, saved + 256, 2 * saved, 0))
    assert torch.equal(a, always) and torch.equal(b, never) and not torch.equal(a, b)
    assert (a.double() - b.double()).abs().max() <= 2.0 ** -7 * b.double().abs().max()


def test_savings_that_no_table_has_room_for():
    """Then, and by default in a small cache, the call is attend's."""
    rng = np.random.default_rng(18)
    c, m = both(60, 2, 64, 4, 12, 64)
    grow(c, m, rng, [0], [300])
    fork(c, m, [0, 0], [1, 2])
    grow(c, m, rng, [0, 1, 2], [5, 40, 90])
    q, seqs = 0.02 * tokens(rng, 4, 1, 8, 64), ints([0, 1, 2, -1])
    c.reserve(seqs, 1)
    room = 3 * 12 * 64 * 2 * 2 * 64           # bytes of three tables of 12 pages
    want = c.attend(0, seqs, q)
    for least in (None, room + 1, 1 << 40, 1 << 80):
        assert torch.equal(c.attend_shared(0, seqs, q, 4, least_saved=least), want)
    o = c.attend_shared(0, seqs, q, 4, least_saved=room)
    assert (o.double() - want.double()).abs().max() <= 2.0 ** -7 * want.double().abs().max()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K,L", [(1, 0), (2, 1), (3, 2), (1, 8)])
def test_the_default_in_long_tables_and_a_sequence_twice(K, L, dtype):
    """Tables with room for any savings, so that the device decides (against
    sharing 256 tokens); the same sequence at several places of a group, and of
    two groups, is attended to at each, shared or not."""
    rng = np.random.default_rng(K + 10 * L)
    c, m = both(60, 2, 128, 8, 4096, 128, dtype)
    grow(c, m, rng, [0], [300], dtype)
    fork(c, m, [0, 0], [1, 2])
    grow(c, m, rng, [0, 1, 2], [5, 40, 90], dtype)
    for least in (None, 0):
        check(c, m, rng, [0, 1, 1, 2, 0, 2, -1, 0], 4, 8, K, L, dtype, least=least)


@pytest.mark.parametrize("G", [2, 17, 100])
def test_wide_groups(G):
    """Row tiles of many members: single tokens and small trees."""
    rng = np.random.default_rng(G)
    c, m = both(G * 3 + 30, 2, 128, G, 20, 64)
    grow(c, m, rng, [0], [900])
    fork(c, m, [0] * (G - 1), list(range(1, G)))
    grow(c, m, rng, list(range(G)), [int(x) for x in rng.integers(0, 70, G)])
    some = sorted(set([0, 1, G // 2, G - 1]))
    for K, L in [(1, 0), (2, 2), (1, 6)]:
        check(c, m, rng, list(range(G)), G, 8, K, L, only=some)


@pytest.mark.parametrize("D,H,Hq", [(128, 2, 8), (64, 5, 5), (64, 1, 7)])
def test_long_rests(D, H, Hq):
    """Rests of one block to thousands of slots: cut within a block of threads,
    between two, and over many."""
    rng = np.random.default_rng(D + H)
    c, m = both(700, H, D, 8, 200, 64)
    grow(c, m, rng, [0, 4], [200, 140])
    fork(c, m, [0, 0, 0, 4, 4, 4], [1, 2, 3, 5, 6, 7])
    grow(c, m, rng, list(range(8)), [9000, 0, 3001, 15, 4000, 1, 700, 64])
    for K, L in [(1, 0), (1, 1), (2, 2)]:
        if (1 + K * L) * (Hq // H) <= 8:
            check(c, m, rng, list(range(8)), 4, Hq, K, L)
    check(c, m, rng, [3, 1, 7, 5], 2, Hq, 1, 0)
    check(c, m, rng, [0, 2], 2, Hq, 1, 0)


@pytest.mark.parametrize("factor,scale", [(1e4, None), (1e-4, None), (1.5, -0.125), (1.5, 0.0), (3e4, -1.0)])
def test_scores_of_any_size(factor, scale):
    """One side may hold all of a row's weight."""
    rng = np.random.default_rng(13)
    c, m = both(60, 1, 64, 4, 12, 64)
    grow(c, m, rng, [0], [400])
    fork(c, m, [0, 0], [1, 2])
    grow(c, m, rng, [0, 1, 2], [5, 0, 130])
    for K, L in [(1, 0), (3, 3)]:
        check(c, m, rng, [0, 1, 2, -1], 4, 4, K, L, factor=factor, scale=scale)


def test_far_apart_halves():
    """Values of the prefix and of a sequence's own tokens that differ by 2^60,
    and a row whose weights lie on one side alone."""
    c = cache.Cache(1, 20, 1, 64, 2, 8, page_tokens=64)
    rng = np.random.default_rng(14)
    k = tokens(rng, 1, 256, 1, 64)
    c.reserve(ints([0]), 256)
    c.append(0, ints([0]), k, torch.full_like(k, 2.0 ** 30))
    c.commit(ints([0]), ints([255]), length=255)
    c.fork(ints([0]), ints([1]))
    c.reserve(ints([0, 1]), 1)
    own = torch.full((2, 1, 1, 64), 100.0, device=DEV, dtype=torch.bfloat16)
    c.append(0, ints([0, 1]), own, torch.full_like(own, 2.0 ** -30))
    for sign, want in ((1, 2.0 ** -30), (-1, 2.0 ** 30)):
        q = sign * torch.full((2, 1, 4, 64), 100.0, device=DEV, dtype=torch.bfloat16)
        o = c.attend_shared(0, ints([0, 1]), q, 2, least_saved=0)
        # scores of 80000 on one side, and below them on the other: one value alone
        assert (o == want).all()
    assert c.status() == (0, "ok")


def test_streams_and_graphs():
    """A captured call finds the prefix again at each replay."""
    rng = np.random.default_rng(15)
    c, m = both(80, 2, 64, 4, 16, 32)
    grow(c, m, rng, [0], [333])
    fork(c, m, [0, 0], [1, 2])
    grow(c, m, rng, [0, 1, 2], [9, 40, 70])
    seqs = ints([0, 1, 2, -1])
    q = tokens(rng, 4, 1, 8, 64)
    c.reserve(seqs, 1)
    want = c.attend_shared(0, seqs, q, 4, least_saved=0)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = c.attend_shared(0, seqs, q, 4, least_saved=0, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    out = torch.zeros_like(q)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.attend_shared(0, seqs, q, 4, least_saved=0, out=out)
    g.replay()
    assert torch.equal(out, want)
    # sequence 2 loses what it shares behind slot 100, and grows again
    c.truncate(ints([2]), ints([100]))
    c.reserve(ints([2]), 200)
    k = tokens(rng, 1, 200, 2, 64)
    c.append(0, ints([2]), k, k)
    c.commit(ints([2]), ints([199]), length=199)
    c.reserve(seqs, 1)
    want = c.attend_shared(0, seqs, q, 4, least_saved=0)
    out.zero_()
    g.replay()
    assert torch.equal(out, want) and (out[2] != 0).any()
    assert c.status() == (0, "ok")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G,K,L", [(2, 1, 0), (3, 1, 0), (6, 1, 0), (6, 2, 4), (3, 1, 30)])
def test_queries_that_are_not_numbers_stay_in_their_rows(G, K, L, dtype):
    """One head of one node is NaN, one infinite: every other row as without, up
    to roundings.  A warp's rows move their references together, so an infinite
    row's moves put the weights of others at other places of their rounding:
    each of the two answers is within its bound of the exact one, 2 * 2^-8 of
    the largest value for weights in the sum and in the normaliser and 2^-8 for
    the output (32-bit queries: 2^-20 covers the few units in 2^-24)."""
    rng = np.random.default_rng(18)
    c, m = both(200, 2, 64, 6, 30, 64, dtype)
    grow(c, m, rng, [0], [700], dtype)
    fork(c, m, [0] * 5, [1, 2, 3, 4, 5])
    grow(c, m, rng, list(range(6)), [5, 40, 90, 0, 33, 200], dtype)
    n = 1 + K * L
    grow(c, m, rng, list(range(6)), [n] * 6, dtype, keep=False)
    q = 0.05 * tokens(rng, 6, n, 10, 64, dtype=dtype)
    want = c.attend_shared(0, ints(range(6)), q, G, branches=K, least_saved=0)
    bad = q.clone()
    bad[1, 0, 3, 7], bad[4, n - 1, 8, 0] = float("nan"), float("inf")
    got = c.attend_shared(0, ints(range(6)), bad, G, branches=K, least_saved=0)
    same = torch.ones(6, n, 10, dtype=torch.bool, device=DEV)
    same[1, 0, 3] = same[4, n - 1, 8] = False
    largest = max(float(np.abs(m.get(s, 0, 0, m.lens[s] + n)[1]).max()) for s in range(6))
    assert torch.isfinite(want).all() and torch.isfinite(got[same]).all()
    assert float((got[same] - want[same]).abs().max()) <= 2 * 3 * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -20) * largest
    assert got[1, 0, 3].isnan().all()
    assert c.status() == (0, "ok")


@pytest.mark.parametrize("D,dtype", [(128, "bf16"), (64, "f32"), (64, "bf16")])
def test_the_largest_batches(D, dtype):
    """1024 sequences in groups of 2, of 32 and all together."""
    rng = np.random.default_rng(19)
    B = 1024
    c = cache.Cache(1, 3 * B + 64, 1, D, B, 8, page_tokens=128, dtype=dtype)
    x = tokens(rng, 1, 300, 1, D, dtype=dtype)
    c.reserve(ints([0]), 300)
    c.append(0, ints([0]), x, x)
    c.commit(ints([0]), ints([299]), length=299)
    c.fork(ints([0] * (B - 1)), ints(range(1, B)))
    seqs = ints(rng.permutation(B))
    c.reserve(seqs, 9)
    y = tokens(rng, B, 9, 1, D, dtype=dtype)
    c.append(0, seqs, y, y)
    for n, K in ((1, 1), (9, 2)):
        q = 0.05 * tokens(rng, B, n, 4, D, dtype=dtype)
        want = c.attend(0, seqs, q, branches=K)
        for G in (2, 32, 1024):
            got = c.attend_shared(0, seqs, q, G, branches=K, least_saved=0)
            # each is within its bound of the exact sum: here at most twice the weights' and the outputs' roundings
            tol = 4 * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -18) * float(torch.maximum(x.abs().max(), y.abs().max()))
            assert float((got - want).abs().max()) <= tol
    assert c.status() == (0, "ok")


def test_tokens_that_are_not_reserved():
    rng = np.random.default_rng(16)
    c, m = both(60, 1, 64, 2, 24, 16)
    grow(c, m, rng, [0], [300])
    fork(c, m, [0], [1])
    c.reserve(ints([0]), 1)
    q = tokens(rng, 2, 3, 4, 64)
    o = c.attend_shared(0, ints([0, 1]), q, 2, least_saved=0)
    assert c.status()[0] == cache.MDS_ST_BADSEQ
    assert o[0, 0].any() and not o[0, 1:].any() and not o[1].any()
    o = c.attend_shared(0, ints([0, 9]), q[:, :1], 2)
    assert c.status()[0] == cache.MDS_ST_BADSEQ and o[0].any() and not o[1].any()


def test_refusals():
    c = cache.Cache(1, 16, 2, 64, 4, 8, page_tokens=16)
    seqs = ints([0, 1, 2, 3])
    q = torch.randn(4, 5, 4, 64, device=DEV, dtype=torch.bfloat16)

    def refused(code, *a, **kw):
        with pytest.raises(cache.MdsError) as e:
            c.attend_shared(*a, **kw)
        assert e.value.code == code

    E, S = cache.MDS_EINVAL, cache.MDS_ESHAPE
    for group in (0, -1, 3, 5, 8, 1 << 32):
        refused(S, 0, seqs, q, group)
    refused(S, 1, seqs, q, 2)
    refused(S, 0, seqs, q, 2, branches=3)
    refused(S, 0, seqs, q[:, :, :3], 2)
    refused(E, 0, seqs, q.float(), 2)
    refused(E, 0, seqs, q, 2, scale=float("nan"))
    refused(S, 0, seqs, q, 2, counts=seqs[:2])
    refused(S, 0, seqs, q, 2, out=q[:2])
    assert c.attend_shared(0, seqs, q[:, :0], 2).shape == (4, 0, 4, 64)
    assert c.attend_shared(0, seqs[:0], q[:0], 2).shape == (0, 5, 4, 64)
    assert c.status() == (0, "ok")
