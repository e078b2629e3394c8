"""Which calls of attend_shared share: the savings of the whole call decide, in
groups of any size, whatever places are unused."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

from paper_2410_18234_gb300 import cache  # noqa: E402
from test_gpu_cache_shared import DEV, both, check, fork, grow, ints, tokens  # noqa: E402


def near(a, b, largest):
    """Each within its bound of the exact answer: 2 * 2^-8 of the largest value
    for the weights in the sum and in the normaliser, 2^-8 for the output."""
    return float((a.double() - b.double()).abs().max()) <= 2 * 3 * 2.0 ** -8 * float(largest)


def forks(rng, B, G, prefix, page=64, H=1, D=64, pages=0, max_pages=12):
    """B / G groups of forks of prefix(group) tokens that went on by 0 to 60 tokens."""
    c, m = both(pages or B * 3 + B // G * 8, H, D, B, max_pages, page)
    roots = list(range(0, B, G))
    grow(c, m, rng, roots, [prefix(i) for i in range(B // G)])
    fork(c, m, [r for r in roots for _ in range(G - 1)], [r + j for r in roots for j in range(1, G)])
    grow(c, m, rng, list(range(B)), [int(x) for x in rng.integers(0, 60, B)])
    return c, m


def test_savings_of_a_call_in_several_turns():
    """4 groups of 64 sequences of 576 rows, of which the workspace holds the
    sums of two groups: what must be saved is compared with what all save."""
    rng = np.random.default_rng(31)
    B, G, n, Hq = 256, 64, 9, 64
    c, m = forks(rng, B, G, lambda i: 300 + 60 * i)                  # 256, 256, 384, 384 shared
    seqs = ints(range(B))
    c.reserve(seqs, n)
    c.append(0, seqs, *(tokens(rng, B, n, 1, 64) for _ in range(2)))
    q = 0.02 * tokens(rng, B, n, Hq, 64)
    largest = c.read(0, seqs, None, 600)[1].abs().max()
    saved = 63 * (256 + 256 + 384 + 384) * 2 * 64                     # bytes
    a, b, always, never = (c.attend_shared(0, seqs, q, G, branches=2, least_saved=x) for x in (saved, saved + 128, 0, 2 * saved))
    assert torch.equal(b, never) and torch.equal(a, always) and not torch.equal(a, b)
    assert near(a, c.attend(0, seqs, q, branches=2), largest)
    assert c.status() == (0, "ok")


@pytest.mark.parametrize("G,parts", [(64, (32, 32)), (53, (27, 26)), (130, (33, 33, 33, 31))])
def test_groups_beyond_the_workspace(G, parts):
    """Sums of 43 sequences of 33 nodes fit: a group is shared in as few parts
    as hold it, each of which reads the prefix once."""
    rng = np.random.default_rng(G)
    n, Hq = 33, 64
    c, m = forks(rng, 2 * G, G, lambda i: 300 + 130 * i)              # 256 and 384 shared
    live = G - 3                                                      # the last places are unused
    order = np.arange(2 * G).reshape(2, G)
    order[:, live:] = -1
    seqs = ints(order.ravel())
    real = ints([x for x in order.ravel() if x >= 0])
    check(c, m, rng, [int(x) for x in order.ravel()], G, Hq, 4, 8, only=[0, parts[0], G - 4, 2 * G - 4])
    c.reserve(real, n)
    c.append(0, real, *(tokens(rng, len(real), n, 1, 64) for _ in range(2)))
    largest = c.read(0, real, None, 600)[1].abs().max()
    q = 0.02 * tokens(rng, 2 * G, n, Hq, 64)
    saved = (live - len(parts)) * (256 + 384) * 2 * 64
    a, b, always, never = (c.attend_shared(0, seqs, q, G, branches=4, least_saved=x) for x in (saved, saved + 128, 0, 2 * saved))
    assert torch.equal(a, always) and torch.equal(b, never) and not torch.equal(a, b)
    alone = c.attend(0, seqs, q, branches=4)
    assert near(a, alone, largest) and near(b, alone, largest)
    assert not a.view(2, G, -1)[:, live:].any()
    # each part as a group of its own, shared in any case: the same launches
    at = 0
    for members in parts:
        ids = seqs.view(2, G)[:, at:at + members]
        for g in range(2):
            one = c.attend_shared(0, ids[g].contiguous(), q.view(2, G, n, Hq, 64)[g, at:at + members], members, branches=4,
                                  least_saved=0)
            assert torch.equal(one, a.view(2, G, n, Hq, 64)[g, at:at + members])
        at += members
    assert at == G and c.status() == (0, "ok")


@pytest.mark.parametrize("least", [None, 0, 200000])
def test_captured_calls_in_turns_and_parts(least):
    """A replay decides again whether it shares: with prefixes of 300 and 430
    tokens and when all but one sequence of each group have lost theirs."""
    rng = np.random.default_rng(8)
    G, n, Hq = 53, 33, 64
    c, m = forks(rng, 2 * G, G, lambda i: 300 + 130 * i)
    seqs = ints(range(2 * G))
    c.reserve(seqs, n)
    c.append(0, seqs, *(tokens(rng, 2 * G, n, 1, 64) for _ in range(2)))
    q = 0.02 * tokens(rng, 2 * G, n, Hq, 64)
    torch.cuda.synchronize()
    graph, out = torch.cuda.CUDAGraph(), torch.zeros_like(q)
    with torch.cuda.graph(graph):
        c.attend_shared(0, seqs, q, G, branches=4, least_saved=least, out=out)
    for step in range(2):
        want = c.attend_shared(0, seqs, q, G, branches=4, least_saved=least)
        shared, alone = (c.attend_shared(0, seqs, q, G, branches=4, least_saved=x) for x in (0, 1 << 30))
        out.fill_(7.0)
        graph.replay()
        assert torch.equal(out, want)
        if step == 0:
            assert torch.equal(alone, c.attend(0, seqs, q, branches=4)) and not torch.equal(shared, alone)
            assert torch.equal(want, shared if least is not None else alone)
            others = ints([x for x in range(2 * G) if x % G])
            c.truncate(others, ints([40] * len(others)))
            c.reserve(others, n)
            c.append(0, others, *(tokens(rng, len(others), n, 1, 64) for _ in range(2)))
        else:   # no tile of 128 tokens is shared any more
            assert torch.equal(want, alone if least is None or least else shared)
            assert near(shared, alone, c.read(0, seqs, None, 600)[1].abs().max())
    assert c.status() == (0, "ok")


def test_unused_places_do_not_count():
    """By default 12 rows a sequence take some 1000 tokens of savings a live
    sequence: 8192 of two are enough, in a list of 16 too."""
    H, D, T = 32, 128, 8192
    c = cache.Cache(1, T // 128 + 4, H, D, 4, 80, page_tokens=128)
    g = torch.Generator(device=DEV).manual_seed(5)

    def new(B, n, heads):
        return torch.randn(B, n, heads, D, generator=g, device=DEV).bfloat16()

    c.reserve(ints([0]), T)
    c.append(0, ints([0]), new(1, T, H), new(1, T, H))
    c.commit(ints([0]), ints([T - 1]), length=T - 1)
    c.fork(ints([0, 0, 0]), ints([1, 2, 3]))
    c.reserve(ints([0, 1]), 3)
    c.append(0, ints([0, 1]), new(2, 3, H), new(2, 3, H))
    q = 0.1 * new(16, 3, 4 * H)
    largest = c.read(0, ints([0]), None, T)[1].abs().max() + 4.5     # new tokens are below that
    for seqs, counts in ((ints([0] + [-1] * 7 + [1] + [-1] * 7), None),
                         (ints([2, 0, 3, 1] + [-1] * 12), ints([0, 3, -1] + [3] * 13))):
        o, always, alone = (c.attend_shared(0, seqs, q, 16, counts=counts, least_saved=x) for x in (None, 0, 2 * 2 * H * D * T))
        assert torch.equal(o, always) and not torch.equal(o, alone) and near(o, alone, largest)
    assert c.status() == (0, "ok")


@pytest.mark.parametrize("D", [64, 128])
def test_groups_at_the_ends_of_tiles(D):
    """Rows of a group about 16, 48, 96 and 144, where one kernel's tiles or
    its variants end, and 256: a sequence each, and a remainder of unused places."""
    rng = np.random.default_rng(D)
    B = 290
    c, m = both(B * 2 + 12, 1, D, B, 12, 64)
    grow(c, m, rng, [0], [333])
    fork(c, m, [0] * (B - 1), list(range(1, B)))
    grow(c, m, rng, list(range(B)), [int(x) for x in rng.integers(0, 40, B)])
    for G in (16, 17, 48, 49, 96, 97, 144, 145, 160, 255, 256, 257, 289):
        check(c, m, rng, list(range(G)), G, 1, 1, 0, only=[0, G // 2, G - 1])
        check(c, m, rng, list(range(G - 1)) + [-1], G, 1, 1, 0, only=[0, G // 2, G - 2])
