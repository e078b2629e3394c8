"""The attention on batches of the largest size, of short sequences: every
place of the list, against 64 bits on what the cache stores."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

from paper_2410_18234_gb300 import cache  # noqa: E402


@pytest.mark.parametrize("B,branches,length,group,head_dim", [(1024, 1, 0, 4, 128), (1024, 2, 4, 8, 64), (1000, 8, 4, 4, 128)])
def test_largest_batches(B, branches, length, group, head_dim):
    g = torch.Generator(device="cuda").manual_seed(B + length)
    H, n, most = 1, 1 + branches * length, 40
    c = cache.Cache(1, B * 6, H, head_dim, B, 6, page_tokens=16)
    seqs = torch.randperm(B, generator=g, device="cuda").int()
    lens = torch.randint(0, most + 1, (B,), generator=g, device="cuda", dtype=torch.int32)

    def new(tokens, heads):
        return torch.randn(B, tokens, heads, head_dim, generator=g, device="cuda").bfloat16()

    c.reserve(seqs, most, counts=lens)
    c.append(0, seqs, new(most, H), new(most, H), counts=lens)
    c.commit(seqs, lens - 1, length=most - 1)
    c.reserve(seqs, n)
    c.append(0, seqs, new(n, H), new(n, H))
    q = new(n, H * group)
    o = c.attend(0, seqs, q, branches=branches)
    T = most + n
    k, v = (x[:, :, 0].double() for x in c.read(0, seqs, None, T, counts=lens + n))
    t = torch.arange(T, device="cuda") - lens[:, None]                       # node of a slot, below 0: committed
    i = torch.arange(n, device="cuda")
    L = max(length, 1)
    own = (i - 1).div(L, rounding_mode="floor") * L + 1                      # first node of a node's branch
    see = (t[:, None] <= 0) | ((t[:, None] >= own[:, None]) & (t[:, None] <= i[:, None]))
    z = torch.einsum("bnhd,btd->bnht", q.double(), k) / head_dim ** 0.5
    w = z.masked_fill(~see[:, :, None], float("-inf")).softmax(-1)
    want = torch.einsum("bnht,btd->bnhd", w, v)
    size = torch.einsum("bnht,btd->bnhd", w, v.abs())
    # bfloat16 (2^-8): the weights over and under the fraction, the output; 32-bit sums beside them
    assert ((o.double() - want).abs() <= 2.0 ** -8 * (2.01 * size + want.abs())).all()
    assert c.status() == (0, "ok")
