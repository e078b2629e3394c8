"""Rotary positions on the GPU against a 64-bit computation: rotated heads
within their roundings, stored keys exactly (the quantiser's answer on the
rotated keys in 64 bits)."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

from cache_model import Model, quantise  # noqa: E402
from paper_2410_18234_gb300 import cache  # noqa: E402

DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def wide(t):
    return t.double().cpu().numpy()


def tokens(rng, *shape, dtype="bf16"):
    x = rng.standard_normal(shape) * np.exp(rng.standard_normal((*shape[:-2], 1, 1))) + 2 * rng.standard_normal(shape[-1])
    return torch.tensor(x, device=DEV).to(DT[dtype])


def depths(n, branches):
    L = (n - 1) // branches
    return np.array([0 if i == 0 else (i - 1) % L + 1 for i in range(n)])


def turned(x, pos, freqs, dim, interleaved, magnitude):
    """x [n][heads][D] in 64 bits at positions [n], and |a| + |b| of each
    number's pair (0 where it does not turn)."""
    # the frequencies in two parts: products with positions below 2^22 are exact
    high = np.floor(np.ldexp(np.array(freqs), 30)) / 2.0 ** 30
    a0, a1 = pos[:, None, None] * high, pos[:, None, None] * (np.array(freqs) - high)
    c, s = np.cos(a0) * np.cos(a1) - np.sin(a0) * np.sin(a1), np.sin(a0) * np.cos(a1) + np.cos(a0) * np.sin(a1)
    y, mag = x.copy(), np.zeros_like(x)
    u, w = (slice(0, dim, 2), slice(1, dim, 2)) if interleaved else (slice(0, dim // 2), slice(dim // 2, dim))
    a, b = x[..., u], x[..., w]
    y[..., u], y[..., w] = magnitude * (a * c - b * s), magnitude * (a * s + b * c)
    mag[..., u] = mag[..., w] = magnitude * (np.abs(a) + np.abs(b))
    return y, mag


def close(got, want, mag, dtype):
    """A rotated number: cosine and sine are off by 2^-24 relative each from
    the leading float, the magnitude's and the two products' roundings, and by
    2^-40 from the sums; then the sum's rounding (2^-24 of the result), then
    the type's (half a step)."""
    tol = 4 * 2.0 ** -24 * mag + 2.0 ** -24 * np.abs(want)
    if dtype == "bf16":
        tol = tol + 2.0 ** -8 * (np.abs(want) + tol)
    # a number that does not turn is copied
    assert (np.abs(got - want) <= np.where(mag > 0, tol, 0.0)).all()


def at_lengths(c, seqs, lens):
    """Commit lens tokens of zeros."""
    most = max(max(lens), 1)
    c.reserve(ints(seqs), most, counts=ints(lens))
    c.commit(ints(seqs), ints([t - 1 for t in lens]), length=most - 1)


SHAPES = [  # D, dim, interleaved, dtype, kv_heads, q_heads, branches, L, page
    (64, 64, False, "bf16", 2, 4, 1, 0, 16),
    (64, 64, True, "f32", 1, 3, 3, 3, 32),
    (64, 16, False, "bf16", 3, 3, 2, 4, 64),
    (64, 48, True, "bf16", 2, 16, 4, 5, 16),
    (128, 128, False, "bf16", 8, 32, 8, 4, 64),
    (128, 128, True, "bf16", 2, 2, 1, 40, 128),
    (128, 128, False, "f32", 5, 5, 1, 33, 64),
    (128, 112, False, "f32", 1, 8, 2, 1, 16),
    (128, 48, False, "bf16", 9, 9, 1, 6, 32),
    (128, 16, True, "f32", 2, 40, 1, 0, 128),
]


@pytest.mark.parametrize("D,dim,interleaved,dtype,H,Hq,K,L,page", SHAPES)
def test_rotate_and_append(D, dim, interleaved, dtype, H, Hq, K, L, page):
    """A batch with lengths of 0, 1, block and page ends, an unused place and
    an id out of range, live counts of 0 to n: queries, stored keys and values,
    what lies behind them, and `append`'s answer on the values."""
    rng = np.random.default_rng(D + dim + H)
    n = 1 + K * L
    lens = [0, 1, 15, 16, 17, page - 1, page, 3 * page + 5]
    S = len(lens)
    c = cache.Cache(2, 64 + S * (n // page + 2), H, D, S + 1, 12 + n // page, page_tokens=page, dtype=dtype)
    m = Model(2, 64 + S * (n // page + 2), H, D, S + 1, 12 + n // page, page)
    r = cache.Rotary(dim, base=10000.0, interleaved=interleaved, magnitude=1.1875)
    order = [int(q) for q in rng.permutation(S)]
    grown = [lens[q] for q in order]
    first = [tokens(rng, S, max(lens), H, D, dtype=dtype) for _ in range(2)]
    m.reserve(order, grown)
    c.reserve(ints(order), max(lens), counts=ints(grown))
    for layer in range(2):
        m.append(layer, order, grown, *(wide(x) for x in first))
        c.append(layer, ints(order), *first, counts=ints(grown))
    m.commit(order, [t - 1 for t in grown])
    c.commit(ints(order), ints([t - 1 for t in grown]), length=max(lens) - 1)
    seqs = order[:3] + [-1] + order[3:] + [S + 7]
    counts = [n, 0, 1, n, max(n - 1, 1), n, n + 5, n, -3, n]
    live = [min(max(x, 0), n) for x in counts]
    # slices of one projection, as a model has them
    x = tokens(rng, len(seqs), n, Hq + 2 * H, D, dtype=dtype)
    q, k, v = x[:, :, :Hq], x[:, :, Hq:Hq + H], x[:, :, Hq + H:]
    m.reserve([s for s in seqs if 0 <= s < S], [t for s, t in zip(seqs, live) if 0 <= s < S])
    c.reserve(ints(seqs), n, counts=ints(counts))
    assert c.status()[0] == cache.MDS_ST_BADSEQ
    depth = depths(n, K)
    out = torch.full((len(seqs), n, Hq, D), 7.0, device=DEV, dtype=DT[dtype])
    got = c.append_rotated(1, ints(seqs), k, v, r, branches=K, q=q, counts=ints(counts), out=out)
    assert got is out
    alone = c.rotate(ints(seqs), q, r, branches=K, counts=ints(counts))
    assert torch.equal(alone, out)
    assert c.status()[0] == cache.MDS_ST_BADSEQ
    new = np.zeros((2, len(seqs), n, H, D))
    for b, s in enumerate(seqs):
        if not 0 <= s < S:
            assert not out[b].any()
            continue
        pos = lens[s] + depth
        want, mag = turned(wide(q[b]), pos, r.freqs, dim, interleaved, 1.1875)
        close(wide(out[b])[:live[b]], want[:live[b]], mag[:live[b]], dtype)
        assert not out[b, live[b]:].any()
        new[0, b] = turned(wide(k[b]), pos, r.freqs, dim, interleaved, 1.1875)[0]
        new[1, b] = wide(v[b])
    known = [b for b, s in enumerate(seqs) if 0 <= s < S]
    m.append(1, [seqs[b] for b in known], [live[b] for b in known], new[0, known], new[1, known])
    total = [lens[s] + t if 0 <= s < S else 0 for s, t in zip(seqs, live)]
    for layer in range(2):
        ck, cv = c.read(layer, ints(seqs), None, max(total), counts=ints(total))
        for b in known:
            # layer 0 got nothing: its slots behind the length hold the pool's zeros
            upto = total[b] if layer else lens[seqs[b]]
            want = m.get(seqs[b], layer, 0, upto).astype(np.float32)
            want = torch.tensor(want).to(DT[dtype]).double().numpy()
            np.testing.assert_array_equal(wide(ck[b, :upto]), want[0])
            np.testing.assert_array_equal(wide(cv[b, :upto]), want[1])
    assert c.lens.tolist()[:S] == lens


@pytest.mark.parametrize("D,dtype", [(64, "f32"), (128, "bf16")])
def test_far_positions(D, dtype):
    """Positions near 2^20: as exact as near 0."""
    rng = np.random.default_rng(5)
    lens = [(1 << 20) - 200, 900001, 12]
    c = cache.Cache(1, 17000, 1, D, 3, 8192, page_tokens=128, dtype=dtype)
    at_lengths(c, range(3), lens)
    n, K = 1 + 4 * 8, 4
    r = cache.Rotary(D, base=500000.0, factor=32.0, original=32768, magnitude=1.25)
    q, k, v = tokens(rng, 3, n, 6, D, dtype=dtype), *(tokens(rng, 3, n, 1, D, dtype=dtype) for _ in range(2))
    seqs = ints([0, 1, 2])
    c.reserve(seqs, n)
    out = c.append_rotated(0, seqs, k, v, r, branches=K, q=q)
    ck, cv = c.read(0, seqs, ints([t // 16 * 16 for t in lens]), n + 15, counts=ints([t % 16 + n for t in lens]))
    for b, t in enumerate(lens):
        pos = t + depths(n, K)
        want, mag = turned(wide(q[b]), pos, r.freqs, D, False, 1.25)
        close(wide(out[b]), want, mag, dtype)
        at = t % 16
        new = np.concatenate([np.zeros((at, 1, D)), turned(wide(k[b]), pos, r.freqs, D, False, 1.25)[0]])
        for i in range(0, new.shape[0], 16):
            np.testing.assert_array_equal(wide(ck[b, i:min(i + 16, at + n), 0]), quantise(new[i:i + 16, 0]))
    assert c.status() == (0, "ok")


def test_scaled_frequencies():
    """The line between pairs that turn often and those that do not."""
    r = cache.Rotary(64, base=10000.0, factor=8.0, original=4096, slow=1.0, fast=32.0)
    for i, f in enumerate(r.freqs):
        g = 10000.0 ** (-2 * i / 64)
        turns = 4096 * g / (2 * math.pi)
        keep = min(max((turns - 1) / 31, 0), 1)
        assert abs(f - g * (keep + (1 - keep) / 8)) <= 4 * 2.0 ** -52 * g
    c = cache.Cache(1, 8, 1, 64, 1, 8, page_tokens=16)
    at_lengths(c, [0], [77])
    x = torch.randn(1, 1, 2, 64, device=DEV, dtype=torch.bfloat16)
    want, mag = turned(wide(x[0]), np.array([77]), r.freqs, 64, False, 1.0)
    close(wide(c.rotate(ints([0]), x, r)[0]), want, mag, "bf16")


def test_in_place_and_without_queries():
    c = cache.Cache(1, 8, 2, 64, 2, 4, page_tokens=16)
    at_lengths(c, [0, 1], [9, 20])
    r = cache.Rotary(64)
    x = torch.randn(2, 5, 6, 64, device=DEV, dtype=torch.bfloat16)
    want = c.rotate(ints([0, 1]), x, r, branches=2)
    y = x.clone()
    assert c.rotate(ints([0, 1]), y, r, branches=2, out=y) is y
    assert torch.equal(y, want)
    k = x[:, :, :2]
    c.reserve(ints([0, 1]), 5)
    assert c.append_rotated(0, ints([0, 1]), k, k, r, branches=2) is None
    one = c.read(0, ints([0, 1]), None, 25)
    # the same once more: the block that the tokens begin in is quantised again
    c.append_rotated(0, ints([0, 1]), k, k, r, branches=2)
    for a, b in zip(one, c.read(0, ints([0, 1]), None, 25)):
        assert torch.equal(a, b)
    assert c.status() == (0, "ok")


def test_tokens_that_are_not_reserved_or_shared():
    """Queries turn whether or not their slots are reserved; keys are stored
    as far as they are, and never into a page that another sequence holds."""
    c = cache.Cache(1, 12, 1, 64, 3, 4, page_tokens=16)
    at_lengths(c, [0], [10])
    r = cache.Rotary(64)
    x = torch.randn(1, 9, 1, 64, device=DEV, dtype=torch.bfloat16)
    c.reserve(ints([0]), 4)
    want = c.rotate(ints([0]), x, r)
    assert c.status() == (0, "ok")
    q = c.append_rotated(0, ints([0]), x, x, r, q=x)
    assert torch.equal(q, want) and c.status()[0] == cache.MDS_ST_BADSEQ
    k, v = c.read(0, ints([0]), ints([10]), 6)
    assert k[0, :4].any(-1).all() and v[0, :4].any(-1).all() and not k[0, 4:].any() and not v[0, 4:].any()
    c.fork(ints([0]), ints([1]))
    c.append_rotated(0, ints([1]), -x, -x, r)
    assert c.status()[0] == cache.MDS_ST_BADSEQ
    for a, b in zip((k, v), c.read(0, ints([0]), ints([10]), 6)):
        assert torch.equal(a, b)


def test_non_finite_keys_stay_in_their_pairs():
    c = cache.Cache(1, 4, 1, 64, 1, 4, page_tokens=16, dtype="f32")
    at_lengths(c, [0], [3])
    r = cache.Rotary(32)
    k = torch.randn(1, 6, 1, 64, device=DEV)
    clean = k.clone()
    k[0, 1, 0, 4], k[0, 2, 0, 5], k[0, 3, 0, 60] = float("nan"), float("inf"), float("-inf")
    c.reserve(ints([0]), 6)
    c.append_rotated(0, ints([0]), k, k, r)
    got, _ = c.read(0, ints([0]), ints([3]), 6)
    assert c.status()[0] == cache.MDS_ST_NONFINITE
    assert torch.isfinite(got).all()
    new = turned(wide(clean[0]), 3 + np.arange(6), r.freqs, 32, False, 1.0)[0][:, 0]
    hit = np.zeros((6, 64), bool)
    hit[1, [4, 20]] = hit[2, [5, 21]] = hit[3, 60] = True
    # the block's largest finite number decides the scale
    block = np.zeros((16, 64))
    block[3:9] = np.where(hit, 0.0, new)
    np.testing.assert_array_equal(wide(got[0, :, 0])[~hit], quantise(block)[3:9][~hit])
    assert not got[0, 1, 0, [4, 20]].any()
    assert got[0, 2, 0, [5, 21]].abs().eq(got.abs().amax()).all() and got[0, 3, 0, 60] == -got.abs().amax()


def test_rotations_that_pass_the_largest_float():
    """They count as infinite, not as missing."""
    c = cache.Cache(1, 4, 1, 64, 1, 4, page_tokens=16, dtype="f32")
    r = cache.Rotary(16, freqs=[0.75] * 8)
    k = torch.zeros(1, 2, 1, 64, device=DEV)
    k[0, 1, 0, 0], k[0, 1, 0, 8], k[0, 0, 0, 9] = 3e38, 3e38, 2e38
    c.reserve(ints([0]), 2)
    c.append_rotated(0, ints([0]), k, k, r)
    got, _ = c.read(0, ints([0]), None, 2)
    # 3e38 (cos 0.75 - sin 0.75) fits, 3e38 (sin 0.75 + cos 0.75) does not
    assert got[0, 1, 0, 8] == got.abs().amax() and 0 < got[0, 1, 0, 0] < 3e37
    assert c.status()[0] == cache.MDS_ST_NONFINITE


def test_streams_graphs_and_unaligned_views():
    c = cache.Cache(1, 16, 2, 64, 2, 8, page_tokens=16)
    at_lengths(c, [0, 1], [30, 40])
    r = cache.Rotary(64, interleaved=True)
    x = torch.randn(2, 3, 6, 64, device=DEV, dtype=torch.bfloat16)
    want = c.rotate(ints([0, 1]), x, r)
    seqs = ints([0, 1])
    c.reserve(seqs, 3)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = c.rotate(seqs, x, r, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    out = torch.zeros_like(x)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.append_rotated(0, seqs, x[:, :, :2], x[:, :, 2:4], r, q=x, out=out)
    del r   # the angles are in the graph
    out.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    x.mul_(2)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, 2 * want)
    with pytest.raises(cache.MdsError):
        c.rotate(seqs, torch.randn(2, 3, 6, 65, device=DEV, dtype=torch.bfloat16)[..., 1:], cache.Rotary(64))
    assert c.status() == (0, "ok")


def test_refusals():
    c = cache.Cache(1, 16, 2, 64, 2, 8, page_tokens=16)
    r, seqs = cache.Rotary(64), ints([0, 1])
    x = torch.randn(2, 5, 2, 64, device=DEV, dtype=torch.bfloat16)

    def refused(code, fn, *a, **kw):
        with pytest.raises(cache.MdsError) as e:
            fn(*a, **kw)
        assert e.value.code == code

    E, S = cache.MDS_EINVAL, cache.MDS_ESHAPE
    refused(S, c.rotate, seqs, x, cache.Rotary(128))
    refused(S, c.rotate, seqs, x, r, branches=3)
    refused(S, c.rotate, seqs, x, r, branches=0)
    refused(S, c.rotate, seqs, x, r, branches=1 << 32)
    refused(E, c.rotate, seqs, x.float(), r)
    refused(S, c.rotate, seqs, x[:1], r)
    refused(E, c.rotate, seqs, x, r, out=x.transpose(1, 2).contiguous().transpose(1, 2).float())
    wide_x = torch.randn(2, 5, 4, 64, device=DEV, dtype=torch.bfloat16)
    flat = wide_x.flatten()[:x.numel()].view_as(x)
    refused(E, c.rotate, seqs, wide_x[:, :, :2], r, out=flat)      # overlaps, not element for element
    refused(S, c.append_rotated, 1, seqs, x, x, r)
    refused(S, c.append_rotated, 0, seqs, x, x[:, :4], r)
    refused(S, c.append_rotated, 0, seqs, x, x, r, q=x[:, :4])
    refused(S, c.append_rotated, 0, seqs, x, x, r, branches=3)
    refused(E, c.append_rotated, 0, seqs, x, x, r, out=x)
    refused(E, c.append_rotated, 0, seqs, x, x.clone(), r, q=x.clone(), out=x)
    refused(S, c.append_rotated, 0, seqs, wide_x, wide_x, r)
    assert c.status() == (0, "ok")
    # nothing to do
    assert c.rotate(seqs, x[:, :0], r).shape == (2, 0, 2, 64)
    c.append_rotated(0, seqs[:0], x[:0], x[:0], r)
    assert c.status() == (0, "ok")
