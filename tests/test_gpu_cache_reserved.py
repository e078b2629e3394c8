"""Only tokens that were reserved are stored, attended to and committed: the
slots that a page holds behind them are not taken for them."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

from cache_model import attend, visible  # noqa: E402
from paper_2410_18234_gb300 import cache  # noqa: E402
from test_gpu_cache import both, bound, grow, ints, same_state, same_values, tokens, wide  # noqa: E402


def refused(c, m, rng, seq, n, values):
    """append, attend and commit of n tokens that were not reserved: nothing
    stored, zeros, nothing kept, and each says so."""
    was = [x.clone() for x in c.read(None, ints([seq]), None, 64)]
    x = tokens(rng, 1, n, m.H, m.D)
    c.append(0, ints([seq]), x, x)
    assert c.status()[0] == cache.MDS_ST_BADSEQ
    for a, b in zip(was, c.read(None, ints([seq]), None, 64)):
        assert torch.equal(a, b)
    for heads in (m.H, 16 * m.H):                       # few rows and many
        o = c.attend(0, ints([seq]), tokens(rng, 1, n, heads, m.D))
        assert not o.any()
        assert c.status()[0] == cache.MDS_ST_BADSEQ
    before = m.lens[seq]
    c.commit(ints([seq]), ints([n - 1]), length=n - 1)
    assert c.status()[0] == cache.MDS_ST_BADSEQ
    m.commit([seq], [-1])
    assert m.lens[seq] == before
    same_state(c, m)
    same_values(c, m, values)


@pytest.mark.parametrize("left", [0, 6])
def test_a_fork_that_got_no_page(left):
    """A fork of a partly filled last page, and no free page to copy it to;
    also where the parent's rejected tokens lie behind the committed ones."""
    rng = np.random.default_rng(30)
    c, m = both(pages=2, page_tokens=16)
    grow(c, m, rng, [0], [19 - left])
    if left:
        grow(c, m, rng, [0], [left + 1], keep=False)
        m.commit([0], [0])
        c.commit(ints([0]), ints([0]), length=left)
    m.fork([0], [1])
    c.fork(ints([0]), ints([1]))
    assert m.reserve([1], [3]) == [1]
    c.reserve(ints([1]), 3)
    assert c.status()[0] == cache.MDS_ST_NOPAGES
    refused(c, m, rng, 1, 3, [0, 1])


def test_a_reserve_that_failed():
    """What a failed call asked for is not there, also where the last page has room."""
    rng = np.random.default_rng(31)
    c, m = both(pages=3, page_tokens=16, max_pages=4)
    grow(c, m, rng, [0], [40])
    for n in (10, 60):                                  # too few pages; a page table too short
        c.reserve(ints([0]), n)
        assert c.status()[0] == cache.MDS_ST_NOPAGES
        refused(c, m, rng, 0, 5, [0])
    grow(c, m, rng, [0], [8])                           # what fits is given
    same_state(c, m)
    same_values(c, m, [0])
    assert c.status() == (0, "ok")


def test_tokens_that_no_one_reserved():
    """Without a reserve, and behind a truncation."""
    rng = np.random.default_rng(32)
    c, m = both(page_tokens=64)
    grow(c, m, rng, [0], [20])
    refused(c, m, rng, 0, 5, [0])
    m.truncate([0], [11])
    c.truncate(ints([0]), ints([11]))
    refused(c, m, rng, 0, 5, [0])
    # more than was reserved: the nodes in front are served, the others are zeros
    grow(c, m, rng, [0], [4], keep=False)
    q = tokens(rng, 1, 6, 4, m.D)
    o = c.attend(0, ints([0]), q)
    assert c.status()[0] == cache.MDS_ST_BADSEQ
    k, v = m.get(0, 0, 0, 15)
    want, mag, big = attend(wide(q[0, :4]), k, v, visible(4, 1, 11), m.D ** -0.5)
    assert (np.abs(wide(o[0, :4]) - want) <= bound(mag, big, want, 15, m.D, "bf16")).all()
    assert not o[0, 4:].any()
    c.commit(ints([0]), ints([4]), length=5)            # five of four
    assert c.status()[0] == cache.MDS_ST_BADSEQ
    m.commit([0], [-1])
    same_state(c, m)
    same_values(c, m, [0])


def test_forks_of_pending_tokens():
    """A fork shares the tokens behind the committed ones: it attends to them
    and keeps them without a copy; once it has reserved, its own are there."""
    rng = np.random.default_rng(33)
    c, m = both(pages=40, page_tokens=16)
    grow(c, m, rng, [0], [20])
    grow(c, m, rng, [0], [30], keep=False)
    m.fork([0, 0], [1, 2])
    c.fork(ints([0, 0]), ints([1, 2]))
    q = tokens(rng, 1, 30, 4, m.D)
    assert torch.equal(c.attend(0, ints([0]), q), c.attend(0, ints([1]), q))
    m.commit([1], [24])
    c.commit(ints([1]), ints([24]), length=29)
    assert c.status() == (0, "ok")
    same_state(c, m)
    same_values(c, m, [0, 1])
    # a copy for 3 tokens: the pages behind it stay shared, their slots are not the fork's own
    assert m.reserve([2], [3]) == []
    c.reserve(ints([2]), 3)
    same_state(c, m)
    o = c.attend(0, ints([2]), q)
    assert c.status()[0] == cache.MDS_ST_BADSEQ
    k, v = m.get(2, 0, 0, 23)
    want, mag, big = attend(wide(q[0, :3]), k, v, visible(3, 1, 20), m.D ** -0.5)
    assert (np.abs(wide(o[0, :3]) - want) <= bound(mag, big, want, 23, m.D, "bf16")).all()
    assert not o[0, 3:].any()
    c.commit(ints([2]), ints([3]), length=29)
    assert c.status()[0] == cache.MDS_ST_BADSEQ
    m.commit([2], [-1])
    same_state(c, m)
    same_values(c, m, [0, 1, 2])
