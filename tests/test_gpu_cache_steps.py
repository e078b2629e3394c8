"""Rotary positions, appending, attention over shared prefixes and the page
operations run together: against the 64-bit model, captured and replayed, and
in the decoding example."""
import os
import sys

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

from cache_model import attend, visible  # noqa: E402
from draft_tree import Decoder, Target  # noqa: E402
from paper_2410_18234_gb300 import cache  # noqa: E402
from test_gpu_cache_rotary import depths, turned  # noqa: E402
from test_gpu_cache_shared import both, bound, fork, ints, tokens, wide  # noqa: E402


@pytest.mark.parametrize("D,page,H,Hq,dtype,interleaved", [(64, 16, 2, 4, "bf16", False), (128, 64, 1, 12, "bf16", True),
                                                           (64, 32, 2, 6, "f32", True)])
def test_steps_of_forked_sequences(D, page, H, Hq, dtype, interleaved):
    """Prompts, forks, trees and commits: rotated queries within their
    roundings, what is stored exactly, attention within its bounds."""
    rng = np.random.default_rng(D + page + Hq)
    c, m = both(6000 // page + 60, H, D, 6, 1200 // page + 4, page, dtype)
    r = cache.Rotary(D, interleaved=interleaved, factor=4.0, original=1024, magnitude=1.25)

    def step(seqs, counts, K, L, group=1):
        n = 1 + K * L
        assert m.reserve(seqs, counts) == []
        c.reserve(ints(seqs), n, counts=ints(counts))
        x = tokens(rng, len(seqs), n, Hq + 2 * H, D, dtype=dtype)
        q, k, v = 0.05 * x[:, :, :Hq], x[:, :, Hq:Hq + H], x[:, :, Hq + H:]
        got = c.append_rotated(0, ints(seqs), k, v, r, branches=K, q=q, counts=ints(counts))
        turn = lambda y, b: turned(wide(y[b]), m.lens[seqs[b]] + depths(n, K), r.freqs, D, interleaved, 1.25)[0]  # noqa: E731
        m.append(0, seqs, counts, np.stack([turn(k, b) for b in range(len(seqs))]), wide(v))
        o = c.attend_shared(0, ints(seqs), got, group, branches=K, counts=ints(counts), least_saved=0)
        for b, s in enumerate(seqs):
            T = m.lens[s] + counts[b]
            kk, vv = m.get(s, 0, 0, m.lens[s] + n)
            want, mag, big = attend(wide(got[b]), kk, vv, visible(n, K, m.lens[s]), D ** -0.5)
            err, lim = np.abs(wide(o[b]) - want)[:counts[b]], bound(mag, big, want, T, D, dtype)[:counts[b]]
            assert (err <= lim).all(), (b, s, float((err / lim).max()))
            assert not o[b, counts[b]:].any()
        return n

    # two ragged prompts
    step([0, 3], [700, 333], 1, 699)
    for call, arg in ((m.commit, lambda x: x), (c.commit, ints)):
        call(arg([0, 3]), arg([699, 332]), *(() if call == m.commit else (1, 699)))
    fork(c, m, [0, 0, 3, 3], [1, 2, 4, 5])
    seqs = [0, 1, 2, 3, 4, 5]
    for K, L in [(2, 4), (1, 0), (4, 3), (2, 4)]:
        step(seqs, [1 + K * L] * 6, K, L, 3)
        drafts = rng.integers(0, 50, (6, K, L)).astype(np.int32)
        accept = [int(a) for a in rng.integers(0, L + 1, 6)]
        emitted = np.full((6, L + 1), -1, np.int32)
        for b in range(6):
            emitted[b, :accept[b]] = drafts[b, rng.integers(K), :accept[b]]
            emitted[b, accept[b]] = 7
        m.commit(seqs, accept, K, L, drafts.tolist(), emitted.tolist())
        c.commit(ints(seqs), ints(accept), branches=K, length=L, draft_tokens=torch.tensor(drafts, device="cuda"),
                 out_tokens=torch.tensor(emitted, device="cuda"))
        assert c.lens.tolist() == m.lens
        np.testing.assert_array_equal(c.table.cpu().numpy(), m.table())
        k, v = c.read(0, ints(seqs), None, max(m.lens), counts=ints(m.lens))
        for b, s in enumerate(seqs):
            want = m.get(s, 0, 0, m.lens[s])
            np.testing.assert_array_equal(wide(k[b, :m.lens[s]]), want[0])
            np.testing.assert_array_equal(wide(v[b, :m.lens[s]]), want[1])
    assert c.status() == (0, "ok")


def test_a_captured_step_grows_its_sequences():
    """One graph of reserve, rotated append, shared attention and commit,
    replayed, does what the calls do one by one."""
    rng = np.random.default_rng(3)

    def make():
        c = cache.Cache(1, 200, 2, 64, 4, 40, page_tokens=16)
        c.reserve(ints([0]), 300)
        x = tokens(np.random.default_rng(4), 1, 300, 2, 64)
        c.append(0, ints([0]), x, x)
        c.commit(ints([0]), ints([299]), length=299)
        c.fork(ints([0, 0, 0]), ints([1, 2, 3]))
        return c

    r, seqs, accept = cache.Rotary(64), ints([0, 1, 2, 3]), ints([0, 1, 2, -1])
    x = tokens(rng, 4, 5, 12, 64)
    out = torch.zeros(4, 5, 8, 64, device="cuda", dtype=torch.bfloat16)

    def step(c):
        c.reserve(seqs, 5)
        q = c.append_rotated(0, seqs, x[:, :, 8:10], x[:, :, 10:], r, branches=2, q=x[:, :, :8])
        c.attend_shared(0, seqs, q, 4, branches=2, least_saved=0, out=out)
        c.commit(seqs, accept, branches=2, length=2)

    plain, graphed = make(), make()
    outs = []
    for _ in range(6):
        step(plain)
        outs.append(out.clone())
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(graphed)
    for want in outs:
        out.zero_()
        g.replay()
        assert torch.equal(out, want)
    assert torch.equal(plain.lens, graphed.lens) and torch.equal(plain.table, graphed.table)
    assert plain.status() == graphed.status() == (0, "ok")


def test_two_caches_at_once():
    """Calls on two caches, on two streams, do not share anything."""
    rng = np.random.default_rng(5)
    caches = [cache.Cache(1, 60, 2, 64, 3, 20, page_tokens=16) for _ in range(2)]
    r, seqs = cache.Rotary(64), ints([0, 1, 2])
    x = tokens(rng, 1, 260, 2, 64)
    q = tokens(rng, 3, 1, 8, 64)
    for c in caches:
        c.reserve(seqs[:1], 260)
        c.append_rotated(0, seqs[:1], x, x, r)
        c.commit(seqs[:1], ints([259]), length=259)
        c.fork(ints([0, 0]), ints([1, 2]))
        c.reserve(seqs, 1)
        c.append_rotated(0, seqs, q[:, :, :2], q[:, :, 2:4], r)
    want = [c.attend_shared(0, seqs, c.rotate(seqs, q, r), 3, least_saved=0) for c in caches]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in caches]
    for _ in range(20):
        got = [c.attend_shared(0, seqs, c.rotate(seqs, q, r, stream=s), 3, least_saved=0, stream=s)
               for c, s in zip(caches, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert torch.equal(want[0], want[1])


@pytest.mark.parametrize("samples,rotary", [(1, True), (4, True), (3, False)])
def test_the_example_with_samples_and_rotary_positions(samples, rotary):
    """The target's logits on the trees are those of a dense pass."""
    target = Target(rotary=cache.Rotary(64) if rotary else None)
    prompts = torch.randint(target.vocab, (2, 150), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    d = Decoder(target, prompts, 3, 2, 6, "WIS", samples=samples, least_saved=0)
    text = [prompts[b // samples].tolist() for b in range(d.B)]

    def dense(text):
        def turn(x):
            y = turned(x[0].double().cpu().numpy(), np.arange(x.shape[1]), target.rotary.freqs, 64, False, 1.0)[0]
            return torch.tensor(y, device="cuda")[None].float()

        def run(layer, q, k, v):
            g = target.q_heads // target.kv_heads
            if target.rotary:
                q, k = turn(q), turn(k)
            q, k, v = (x.float().transpose(1, 2) for x in (q, k, v))
            k, v = k.repeat_interleave(g, 1), v.repeat_interleave(g, 1)
            n = q.shape[2]
            z = q @ k.transpose(2, 3) / 8.0
            z = z.masked_fill(torch.ones(n, n, device="cuda").triu(1).bool(), float("-inf"))
            return (z.softmax(-1) @ v).transpose(1, 2)
        return target(torch.tensor(text, device="cuda")[None], torch.arange(len(text), device="cuda")[None], run)[0, -1]

    for i in range(6):
        before = [list(t) for t in text]
        out, accept, logits = d.step(i)
        for b in range(d.B):
            text[b] += out[b, :int(accept[b]) + 1].tolist()
        if i in (0, 5):
            for b in range(d.B):
                # 8-bit keys and values (2^-4 relative) move logits of a standard deviation of 3
                want = dense(before[b])
                assert float((logits[b, 0, 0] - want).norm() / want.norm()) < 0.1
    assert d.cache.lens[:d.B].tolist() == [len(t) - 1 for t in text]
    assert d.status() == 0
