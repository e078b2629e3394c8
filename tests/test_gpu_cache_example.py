"""The cache around the verification, run together by examples/draft_tree.py:
the cache holds the prompt and every accepted token, and the target's logits
on a tree are those of a dense forward pass over each branch."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

from draft_tree import Decoder, Target  # noqa: E402


def dense(target, tokens):
    """Logits of a token list with plain causal attention in 32 bits."""
    def attend(layer, q, k, v):
        g = target.q_heads // target.kv_heads
        q, k, v = (x.float().transpose(1, 2) for x in (q, k, v))
        k, v = k.repeat_interleave(g, 1), v.repeat_interleave(g, 1)
        z = q @ k.transpose(2, 3) / target.head_dim ** 0.5
        n = z.shape[-1]
        z = z.masked_fill(torch.ones(n, n, device=z.device).triu(1).bool(), float("-inf"))
        return (z.softmax(-1) @ v).transpose(1, 2)
    return target(tokens[None], torch.arange(len(tokens), device="cuda")[None], attend)[0]


@pytest.mark.parametrize("branches,length,scheme", [(4, 3, "WIS"), (2, 4, "single"), (1, 1, "SpecTr")])
def test_decoding_by_trees(branches, length, scheme):
    target = Target()
    prompts = torch.randint(target.vocab, (3, 21), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    d = Decoder(target, prompts, branches, length, 10, scheme)
    text = [p.tolist() for p in prompts]
    accepted = 0
    for i in range(10):
        before = [list(t) for t in text]
        out, accept, logits = d.step(i)
        for b in range(3):
            a = int(accept[b])
            accepted += a
            text[b] += out[b, :a + 1].tolist()
        # all but the last emitted token are in the cache
        assert d.cache.lens[:3].tolist() == [len(t) - 1 for t in text]
        if i in (0, 9):
            # depth 0 of every branch: the text so far.  8-bit keys and values
            # (2^-4 relative) move logits of a standard deviation of 3.
            for b in range(3):
                want = dense(target, torch.tensor(before[b], device="cuda"))[-1]
                for k in range(branches):
                    got = logits[b, k, 0]
                    assert float((got - want).norm() / want.norm()) < 0.1
    assert d.status() == 0
    if branches > 1:
        assert accepted > 0
    # the committed tokens' keys, read back, are those of a dense pass: layer 0's depend on the text alone
    k, _ = d.cache.read(0, d.seqs, None, max(len(t) for t in text), counts=d.cache.lens[:3].clone())
    for b in range(3):
        n = len(text[b]) - 1
        seen = []

        def attend(layer, q, kk, v):
            seen.append(kk[0].float())
            return torch.zeros_like(q)
        target(torch.tensor(text[b][:n], device="cuda")[None], torch.arange(n, device="cuda")[None], attend)
        want = seen[0]
        assert float((k[b, :n].float() - want).norm() / want.norm()) < 2.0 ** -4
