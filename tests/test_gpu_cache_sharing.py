"""Which calls of attend_shared share: the savings of the whole call decide,
whatever places are unused."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

from paper_2410_18234_gb300 import cache  # noqa: E402
from test_gpu_cache_shared import DEV, both, fork, grow, ints, tokens  # noqa: E402


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


def test_unused_places_do_not_count():
    """By default 12 rows a sequence take 1200 tokens of savings a sequence:
    8192 of two live ones are enough, in a list of 16 too."""
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
