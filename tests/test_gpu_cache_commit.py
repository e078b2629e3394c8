"""commit on sequences of one call that share pages behind the committed
tokens: what is kept follows from the state before the call, in every layer."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

from paper_2410_18234_gb300 import cache  # noqa: E402
from test_gpu_cache import both, grow, ints, same_state, same_values  # noqa: E402


@pytest.mark.parametrize("order", [[0, 1], [1, 0], [2, 0, 1], [1, 2, 0]])
@pytest.mark.parametrize("head_dim", [64, 128])
def test_forks_commit_together(order, head_dim):
    """Forks of a pending tree: one drops it, the others would move a branch
    into pages that were shared when the call began.  Again and again, with
    enough layers for many blocks of threads a sequence."""
    rng = np.random.default_rng(len(order) + head_dim)
    K, L = 2, 20
    n = 1 + K * L
    c, m = both(layers=8, pages=30, kv_heads=8, head_dim=head_dim, page_tokens=16)
    grow(c, m, rng, [0], [20])
    drafts = rng.integers(0, 3, (len(order), K, L))
    drafts[:, 1] += 3                                   # branch 1 is no other
    accept = [-1 if q == order[0] else L for q in order]
    out = np.concatenate([drafts[:, 1], np.full((len(order), 1), 9)], 1)
    others = [q for q in order if q]
    for turn in range(30):
        grow(c, m, rng, [0], [n], keep=False)
        m.fork([0] * len(others), others)
        c.fork(ints([0] * len(others)), ints(others))
        c.commit(ints(order), ints(accept), branches=K, length=L, draft_tokens=ints(drafts), out_tokens=ints(out))
        m.commit(order, [-1] * len(order))
        assert c.status()[0] == cache.MDS_ST_BADSEQ
        same_state(c, m)
        same_values(c, m, order)
        m.free(others)
        c.free(ints(others))
    grow(c, m, rng, [0], [n], keep=False)
    # alone, the pages are its own: the branch is kept
    c.commit(ints([0]), ints([L]), branches=K, length=L, draft_tokens=ints(drafts[:1]), out_tokens=ints(out[:1]))
    m.commit([0], [L], K, L, drafts[:1], out[:1])
    assert c.status() == (0, "ok")
    same_state(c, m)
    same_values(c, m, [0])


def test_forks_keep_branch_0_together():
    """Nothing moves for branch 0: every fork keeps it, shared pages or not."""
    rng = np.random.default_rng(40)
    K, L = 3, 9
    c, m = both(layers=3, pages=30, page_tokens=16)
    grow(c, m, rng, [0], [21])
    grow(c, m, rng, [0], [1 + K * L], keep=False)
    m.fork([0, 0], [3, 4])
    c.fork(ints([0, 0]), ints([3, 4]))
    drafts = rng.integers(0, 3, (3, K, L))
    accept = [9, 0, 4]
    out = np.concatenate([drafts[:, 0], np.full((3, 1), 9)], 1)
    c.commit(ints([3, 0, 4]), ints(accept), branches=K, length=L, draft_tokens=ints(drafts), out_tokens=ints(out))
    m.commit([3, 0, 4], accept, K, L, drafts, out)
    assert c.status() == (0, "ok")
    same_state(c, m)
    same_values(c, m, [0, 3, 4])
