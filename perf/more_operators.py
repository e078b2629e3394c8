"""Cases of the operators on either side of the key/value cache's attention:
rotary positions of draft-tree nodes, appending keys with that rotation on the
way, and attention for sequences that share a prefix.

A step of multi-draft decoding runs n = 1 + K * L nodes a sequence (node 0 the
root, node 1 + k * L + j branch k's draft at depth j + 1) behind its committed
tokens; K = 1 is a chain: one token (n = 1), or a chunk of a prompt.  A node's
position is the sequence's length and its depth.

rotate  pairs (x_a, x_b) of a head's first `dim` dimensions become
        m (x_a cos - x_b sin), m (x_a sin + x_b cos) at the angle
        position * f_i; pair i is dimensions (i, i + dim / 2), or
        (2 i, 2 i + 1) where interleaved.  f_i = base^(-2 i / dim), for long
        contexts divided by a factor: wholly where the pair turns less than
        `slow` times in `original` tokens, not where it turns more than
        `fast` times, in between by a line.
append  the keys of the nodes rotated and, like their values, quantised into
        the cache behind the committed tokens: for every 16 tokens and head
        a = max|x|, e the least integer with a <= 448 * 2^e, each value rounded
        to e4m3(x / 2^e); a block that already holds tokens is quantised again
        with the new ones from the values it stands for.  The queries of the
        same nodes are rotated in the same call.  The pass reads the new tokens
        and the block that they begin in back as values.
shared  o = sum_t softmax_t(scale * q . k_t) v_t over the visible tokens, for
        groups of G sequences that were forked from one prefix and went on by
        themselves.

Lengths are spread evenly over the case's range.
"""
import math

import torch

own = False

BLOCK = 16
STORAGE = {"f32": torch.float32, "bf16": torch.bfloat16}


# ------------------------------------------------------------------ cases


def _rope(name, op, B, lo, hi, K=1, L=0, Hq=32, Hkv=8, D=128, page=64, dtype="bf16", dim=0, interleaved=False,
          base=10000.0, factor=1.0, original=0, magnitude=1.0, ragged=False):
    return {"name": name, "op": op, "B": B, "lo": lo, "hi": hi, "K": K, "L": L, "Hq": Hq, "Hkv": Hkv, "D": D,
            "page": page, "dtype": dtype, "dim": dim or D, "interleaved": interleaved, "base": base, "factor": factor,
            "original": original, "magnitude": magnitude, "ragged": ragged}


def _shared(name, B, G, plo, phi, lo, hi, K=1, L=0, Hq=32, Hkv=8, D=128, page=64, dtype="bf16"):
    return {"name": name, "op": "shared", "B": B, "G": G, "plo": plo, "phi": phi, "lo": lo, "hi": hi, "K": K, "L": L,
            "Hq": Hq, "Hkv": Hkv, "D": D, "page": page, "dtype": dtype}


def listed():
    return [
        # one interactive user's next token, queries alone: latency
        _rope("rotate-one-token", "rotate", 1, 4100, 4100),
        # the queries of four prompts of an odd length, neighbouring pairs, long-context frequencies
        _rope("rotate-prompts", "rotate", 4, 0, 0, L=4098, interleaved=True, base=500000.0, factor=8.0, original=8192),
        # a batch that decodes token by token: latency of a whole layer's positions and cache writes
        _rope("append-token", "append", 64, 1, 8191),
        # one layer's trees of the 128k workload's batch
        _rope("append-tree-8x4", "append", 256, 257, 1537, K=8, L=4, base=500000.0),
        # ragged prompts of a 32-bit model that rotates half of each head
        _rope("append-prompt-f32", "append", 4, 0, 0, L=4098, Hq=16, dtype="f32", page=32, dim=64, interleaved=True, ragged=True),
        # trees at the far end of very long contexts: exact angles
        _rope("append-far-4x8", "append", 2, 1000003, 1040007, K=4, L=8, Hq=16, Hkv=2, D=64, factor=32.0, original=32768, magnitude=1.25),
        # eight samples of one prompt: latency
        _shared("shared-8-samples", 8, 8, 4100, 4100, 1, 200),
        # a serving batch under one system prompt
        _shared("shared-system-prompt", 64, 64, 8195, 8195, 1, 2000),
        # sixteen prompts, eight samples of each
        _shared("shared-16x8", 128, 8, 1500, 12001, 1, 1000),
        # the 50k workload's tree on four long documents, eight conversations about each
        _shared("shared-tree-2x4", 32, 8, 20001, 40001, 100, 3001, K=2, L=4, Hq=64, D=64),
        # 32-bit queries, small pages, a tree
        _shared("shared-f32-3x3", 6, 3, 600, 777, 1, 77, K=3, L=3, Hq=12, Hkv=4, D=64, page=16, dtype="f32"),
        # the 128k workload's batch over one long document
        _shared("shared-document", 256, 256, 32771, 32771, 1, 300),
    ]


def draw(rng):
    """A case of the same ranges: batches of 1 to 256, single tokens, trees and
    prompt chunks, both head widths, whole and partly rotated heads in both
    layouts, positions to a million; groups of 2 to 256 over prefixes of 100 to
    40000 tokens; odd lengths throughout."""
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["rotate", "append", "append", "shared", "shared", "shared"])
    D = rng.choice([64, 128, 128])
    page = rng.choice([16, 32, 64, 64, 128])
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    Hkv = rng.choice([1, 2, 4, 8, 8, 32] if op != "shared" else [1, 2, 4, 8, 8])
    g = rng.choice([1, 3, 4, 8]) if Hkv <= 8 else 1
    K, L = rng.choice([(1, 0), (1, 0), (1, 0), (2, 4), (4, 5), (8, 4), (3, 3), (1, 7), (1, -1)])
    if L < 0:
        L = spread(30, 4099) if op != "shared" else 3
    n = 1 + K * L
    if op != "shared":
        # no more than the largest listed case: bytes of the nodes' queries, keys and values
        node = Hkv * (g + 2) * D * (4 if dtype == "f32" else 2)
        if K == 1:
            L = min(L, int(1.3e8 / node))
        n = 1 + K * L
        B = max(1, min(spread(1, 256), int(1.3e8 / (n * node))))
        hi = spread(1, 1040000)
        hi = max(1, min(hi, int(1e9 / (B * Hkv * D)), (1 << 20) - n))
        lo = rng.choice([0, hi // 4, hi])
        factor = rng.choice([1.0, 1.0, 8.0, 32.0])
        c = _rope("", op, B, lo, hi, K, L, Hkv * g, Hkv, D, page, dtype, dim=rng.choice([D, D, D // 2, 16, 48]),
                  interleaved=rng.random() < 0.4, base=rng.choice([10000.0, 500000.0]), factor=factor,
                  original=rng.choice([0, 4096, 32768]) if factor > 1 else 0, magnitude=rng.choice([1.0, 1.25]),
                  ragged=rng.random() < 0.3)
    else:
        G = spread(2, 256)
        B = G * max(1, min(rng.choice([1, 2, 5, 16]), 256 // G))
        phi = spread(100, 40000)
        hi = spread(1, 3000)
        # no more than the largest listed case: cache bytes, products, and pairs of queries and keys
        phi = max(100, min(phi, int(2e10 / (B * n * Hkv * g * D)), int(2.6e8 / (B * n * Hkv * g)), int(8e7 / (B // G * Hkv * D))))
        hi = max(1, min(hi, int(8e7 / (B * Hkv * D)), int(1e8 / (B * n * Hkv * g))))
        c = _shared("", B, G, rng.choice([phi // 2, phi]), phi, rng.choice([0, hi // 4, hi]), hi, K, L, Hkv * g, Hkv, D, page, dtype)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs


def _even(count, lo, hi):
    """`count` lengths of a range: its ends' even spread."""
    return [lo + int((hi - lo + 1) * (((b + 1) * 0.6180339887498949) % 1.0)) for b in range(count)]


def _lens(case):
    """Committed tokens of every sequence (shared: behind its group's prefix)."""
    return _even(case["B"], case["lo"], case["hi"])


def _prefixes(case):
    """Tokens that each group of sequences shares."""
    return _even(case["B"] // case["G"], case["plo"], case["phi"])


def _nodes(case):
    return 1 + case["K"] * case["L"]


def _counts(case):
    """Live nodes of every sequence."""
    n = _nodes(case)
    return [1 + (b * 7919) % n for b in range(case["B"])] if case["ragged"] and n > 1 else [n] * case["B"]


def _depths(case):
    """A node's depth: tokens between the sequence's committed ones and it."""
    i = torch.arange(_nodes(case), device="cuda")
    return torch.where(i > 0, (i - 1) % max(case["L"], 1) + 1, 0)


def _seeded(seed, part):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 64 + part)


def _keys_values(g, shape, offset, dtype):
    """Keys and values [..][T][H][D]: normals with an offset per channel on the
    keys and a magnitude per token."""
    out = []
    for add in (offset, 0.0):
        size = torch.exp(0.5 * torch.randn(*shape[:2], 1, 1, generator=g, device="cuda"))
        out.append(torch.randn(*shape, generator=g, device="cuda").mul_(size).add_(add).to(dtype))
    return out


def _projected(case, seed):
    """Queries, keys and values of the nodes as a model has them: slices of one
    projection [B][n][Hq + 2 Hkv][D]."""
    g, n, st = _seeded(seed, 0), _nodes(case), STORAGE[case["dtype"]]
    Hq, H = case["Hq"], case["Hkv"]
    x = torch.empty(case["B"], n, Hq + 2 * H, case["D"], device="cuda", dtype=st)
    x[:, :, :Hq] = 1.5 * torch.randn(case["B"], n, Hq, case["D"], generator=g, device="cuda")
    offset = 2.0 * torch.randn(H, case["D"], generator=g, device="cuda")
    x[:, :, Hq:Hq + H], x[:, :, Hq + H:] = _keys_values(g, (case["B"], n, H, case["D"]), offset, st)
    return x[:, :, :Hq], x[:, :, Hq:Hq + H], x[:, :, Hq + H:]


def _begun(case, seed):
    """Keys (rotated before) and values [B][16][H][D] of the committed tokens
    in the block that a sequence's length ends in."""
    g = _seeded(seed, 1)
    offset = 2.0 * torch.randn(case["Hkv"], case["D"], generator=g, device="cuda")
    return _keys_values(g, (case["B"], BLOCK, case["Hkv"], case["D"]), offset, STORAGE[case["dtype"]])


def _conversation(case, seed):
    """Queries of the nodes [B][n][Hq][D], and keys and values of the prefixes
    [groups][P][H][D], of what the sequences said since [B][T][H][D], and of
    the nodes [B][n][H][D]."""
    g, st = _seeded(seed, 2), STORAGE[case["dtype"]]
    B, H, D = case["B"], case["Hkv"], case["D"]
    q = (1.5 * torch.randn(B, _nodes(case), case["Hq"], D, generator=g, device="cuda")).to(st)
    offset = 2.0 * torch.randn(H, D, generator=g, device="cuda")
    lengths = (B // case["G"], max(_prefixes(case))), (B, max(max(_lens(case)), 1)), (B, _nodes(case))
    return q, [_keys_values(g, (*s, H, D), offset, st) for s in lengths]


def _frequencies(case):
    """Radians a position of each pair, in 64 bits."""
    f = case["base"] ** (-torch.arange(0, case["dim"], 2, device="cuda", dtype=torch.float64) / case["dim"])
    if case["original"]:
        keep = ((case["original"] * f / (2 * math.pi) - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)   # slow 1, fast 32 turns
    else:
        keep = torch.zeros_like(f)
    return f * (keep + (1.0 - keep) / case["factor"])


# ------------------------------------------------------- the plain forms


def _rotated(x, pos, case):
    """x [B][n][heads][D] at positions [B][n], in x's precision; angles in 64 bits."""
    dim, half = case["dim"], case["dim"] // 2
    angle = (pos[..., None].double() * _frequencies(case))[:, :, None]                     # [B][n][1][dim / 2]
    c, s = (case["magnitude"] * f(angle).to(x.dtype) for f in (torch.cos, torch.sin))
    head, rest = x[..., :dim], x[..., dim:]
    a, b = (head[..., ::2], head[..., 1::2]) if case["interleaved"] else (head[..., :half], head[..., half:])
    a, b = a * c - b * s, a * s + b * c
    head = torch.stack((a, b), -1).flatten(-2) if case["interleaved"] else torch.cat((a, b), -1)
    return torch.cat((head, rest), -1)


def _e4m3(y):
    """The nearest e4m3 numbers to |y| <= 448 in y's precision, ties to even."""
    _, e = torch.frexp(y)
    step = torch.ldexp(torch.ones_like(y), (e - 1).clamp(min=-6) - 3)
    return torch.round(y / step) * step


def _quantise(x):
    """Q on blocks [..., 16, H, D]: e4m3 numbers, and scales [..., H]."""
    a = x.abs().amax(dim=(-3, -1))
    m, e = torch.frexp(a)
    e = torch.where(m <= 0.875, e - 9, e - 8).clamp(-117, 119)
    scale = torch.ldexp(torch.ones_like(a), torch.where(a > 0, e, 0))
    return _e4m3(x / scale[..., None, :, None]).float().to(torch.float8_e4m3fn), scale.float()


def _values(by, scale):
    return by.float() * scale[..., None, :, None]


def _blocks(x):
    """[B, T, H, D] as blocks [B, T / 16, 16, H, D]."""
    return x.unflatten(1, (-1, BLOCK))


def _padded(x, T):
    return torch.nn.functional.pad(x, (0, 0, 0, 0, 0, T - x.shape[1]))


def _stored(old, at, new, count):
    """Values [B][16 * blocks][H][D] of `at` tokens in front, as they were
    stored, and `count` new ones behind them: bytes and scales."""
    T = -(-(BLOCK - 1 + new.shape[1]) // BLOCK) * BLOCK
    t = torch.arange(T, device="cuda")
    i = (t - at[:, None]).clamp(0, new.shape[1] - 1)[..., None, None].expand(-1, -1, *new.shape[2:])
    live = (t < (at + count)[:, None])[..., None, None]
    y = torch.where((t < at[:, None])[..., None, None], _padded(old.to(new.dtype), T),
                    torch.where(live, torch.gather(new, 1, i), 0.0))
    return _quantise(_blocks(y))


class _State:
    pass


def prepare(case, seed):
    s = _State()
    s.case = case
    n, B = _nodes(case), case["B"]
    lens = torch.tensor(_lens(case), device="cuda")
    if case["op"] == "shared":
        s.q, tokens = _conversation(case, seed)
        pre = torch.tensor(_prefixes(case), device="cuda")
        if own:
            return _own_shared(s, tokens, pre, lens)
        # plain: the prefixes' whole blocks, and each sequence's tokens from there on
        s.lens, s.whole, s.tail = lens, pre // BLOCK * BLOCK, (pre % BLOCK).repeat_interleave(case["G"])
        s.prefix, s.mine = [], []
        for p, t, x in zip(*tokens):
            p = _padded(p, -(-p.shape[1] // BLOCK) * BLOCK).float()
            p = torch.where((torch.arange(p.shape[1], device="cuda") < pre[:, None])[..., None, None], p, 0.0)
            by, sc = _quantise(_blocks(p))
            s.prefix.append((by, sc))
            begun = _values(by, sc)[torch.arange(len(pre), device="cuda"), (s.whole // BLOCK).clamp(max=by.shape[1] - 1)]
            by, sc = _stored(begun.repeat_interleave(case["G"], 0), s.tail, t.float(), lens)
            s.mine.append(_join(_values(by, sc).flatten(1, 2), s.tail + lens, x, n))
        return s
    s.q, s.k, s.v = _projected(case, seed)
    s.counts = torch.tensor(_counts(case), device="cuda", dtype=torch.int32)
    if own:
        return _own_rope(s, lens, seed)
    s.lens, s.depth = lens, _depths(case)
    if case["op"] == "append":
        s.at = lens % BLOCK
        live = (torch.arange(BLOCK, device="cuda") < s.at[:, None])[..., None, None]
        s.begun = [_quantise(_blocks(torch.where(live, x.float(), 0.0))) for x in _begun(case, seed)]
    return s


def _join(y, at, x, n):
    """n new tokens x behind the first `at` values of y [B][T][H][D], of which
    the block that they begin in is quantised again."""
    T = -(-(y.shape[1] + n) // BLOCK) * BLOCK
    t = torch.arange(T, device="cuda")
    i = (t - at[:, None]).clamp(0, n - 1)[..., None, None].expand(-1, -1, *x.shape[2:])
    new = torch.where((t < (at + n)[:, None])[..., None, None], torch.gather(x.float(), 1, i), 0.0)
    return _quantise(_blocks(torch.where((t < at[:, None])[..., None, None], _padded(y, T), new)))


def _run_rotate(s):
    pos = s.lens[:, None] + s.depth
    live = (torch.arange(pos.shape[1], device="cuda") < s.counts[:, None])[..., None, None]
    return torch.where(live, _rotated(s.q.float(), pos, s.case), 0.0).to(s.q.dtype)


def _run_append(s):
    c, n = s.case, _nodes(s.case)
    # keys in 64 bits: what is quantised behind them may lie next to a border
    new = _rotated(s.k.double(), s.lens[:, None] + s.depth, c), s.v.float()
    got = []
    for x, old in zip(new, s.begun):
        by, sc = _stored(_values(*old).flatten(1, 2), s.at, x, s.counts)
        got.append(_values(by, sc).flatten(1, 2)[:, :n + BLOCK - 1].to(s.q.dtype))
    return (_run_rotate(s), *got)


def _run_shared(s):
    c = s.case
    B, G, n, Hq, H, D, L = c["B"], c["G"], _nodes(c), c["Hq"], c["Hkv"], c["D"], c["L"]
    g, NG = Hq // H, B // G
    (pk, pv), (mk, mv) = ([_values(*x).flatten(1, 2) for x in y] for y in (s.prefix, s.mine))
    P, T = pk.shape[1], mk.shape[1]
    q = s.q.float().view(B, n, H, g, D).permute(0, 2, 3, 1, 4).reshape(B, H, g * n, D) * (1.0 / math.sqrt(D))
    # scores of a group's queries on its prefix, computed once for all, and of each sequence's on its own tokens
    qg = q.view(NG, G, H, g * n, D).transpose(1, 2).reshape(NG, H, G * g * n, D)
    a = torch.matmul(qg, pk.permute(0, 2, 3, 1))
    a.masked_fill_((torch.arange(P, device="cuda") >= s.whole[:, None])[:, None, None], -math.inf)
    b = torch.matmul(q, mk.permute(0, 2, 3, 1)).view(B, H, g, n, T)
    node = torch.arange(T, device="cuda") - (s.tail + s.lens)[:, None]
    me = torch.arange(n, device="cuda")
    branch, mine = (node - 1) // max(L, 1), (me - 1) // max(L, 1)
    see = (node[:, None] <= 0) | ((branch[:, None] == mine[:, None]) & (node[:, None] <= me[:, None]))
    b.masked_fill_(~see[:, None, None], -math.inf)
    b = b.view(NG, G, H, g * n, T).transpose(1, 2).reshape(NG, H, G * g * n, T)
    top = torch.maximum(a.amax(-1, keepdim=True), b.amax(-1, keepdim=True))
    a, b = a.sub_(top).exp_(), b.sub_(top).exp_()
    total = a.sum(-1, keepdim=True) + b.sum(-1, keepdim=True)
    o = torch.matmul(a, pv.transpose(1, 2)).view(NG, H, G, g * n, D).transpose(1, 2).reshape(B, H, g * n, D)
    b, total = (x.view(NG, H, G, g * n, -1).transpose(1, 2).reshape(B, H, g * n, -1) for x in (b, total))
    o = (o + torch.matmul(b, mv.transpose(1, 2))) / total
    return o.view(B, H, g, n, D).permute(0, 3, 1, 2, 4).reshape(B, n, Hq, D).to(s.q.dtype)


# ----------------------------------------------- the framework's operators


def _own_cache(case, pages, span):
    from paper_2410_18234_gb300 import cache
    return cache.Cache(1, pages, case["Hkv"], case["D"], case["B"], span, page_tokens=case["page"], dtype=case["dtype"])


def _own_rope(s, lens, seed):
    from paper_2410_18234_gb300 import cache
    c, n, lens = s.case, _nodes(s.case), lens.int()
    s.rotary = cache.Rotary(c["dim"], base=c["base"], interleaved=c["interleaved"], factor=c["factor"],
                            original=c["original"], fast=32.0, slow=1.0, magnitude=c["magnitude"])
    held = [-(-(t + n) // c["page"]) for t in _lens(c)]
    s.cache = _own_cache(c, sum(held), max(held))
    s.seqs = torch.arange(c["B"], device="cuda", dtype=torch.int32)
    s.start = lens // BLOCK * BLOCK
    s.live = lens - s.start + s.counts
    # the blocks in front hold nothing that is looked at; then the begun one
    s.cache.reserve(s.seqs, c["hi"] + 1, counts=s.start)
    s.cache.commit(s.seqs, s.start - 1, length=c["hi"])
    s.cache.reserve(s.seqs, BLOCK, counts=lens - s.start)
    s.cache.append(0, s.seqs, *_begun(c, seed), counts=lens - s.start)
    s.cache.commit(s.seqs, lens - s.start - 1, length=BLOCK - 1)
    s.cache.reserve(s.seqs, n)
    return s


def _own_shared(s, tokens, pre, lens):
    c, n, page, B, G = s.case, _nodes(s.case), s.case["page"], s.case["B"], s.case["G"]
    first, both = _prefixes(c), [p + t + n for p, t in zip((p for p in _prefixes(c) for _ in range(G)), _lens(c))]
    pages = sum(-(-p // page) for p in first) + sum(-(-t // page) - p // page for t, p in zip(both, (p for p in first for _ in range(G))))
    s.cache = _own_cache(c, pages, max(-(-t // page) for t in both))
    s.seqs = torch.arange(B, device="cuda", dtype=torch.int32)
    root, lens, pre = s.seqs[::G].contiguous(), lens.int(), pre.int()
    (pk, tk, xk), (pv, tv, xv) = zip(*tokens)
    s.cache.reserve(root, pk.shape[1], counts=pre)
    s.cache.append(0, root, pk, pv, counts=pre)
    s.cache.commit(root, pre - 1, length=pk.shape[1] - 1)
    s.cache.fork(root.repeat_interleave(G - 1), s.seqs.view(-1, G)[:, 1:].contiguous().flatten())
    s.cache.reserve(s.seqs, tk.shape[1], counts=lens)
    s.cache.append(0, s.seqs, tk, tv, counts=lens)
    s.cache.commit(s.seqs, lens - 1, length=tk.shape[1] - 1)
    s.cache.reserve(s.seqs, n)
    s.cache.append(0, s.seqs, xk, xv)
    return s


def _run_own(s):
    c = s.case
    if c["op"] == "rotate":
        return s.cache.rotate(s.seqs, s.q, s.rotary, branches=c["K"], counts=s.counts)
    if c["op"] == "append":
        q = s.cache.append_rotated(0, s.seqs, s.k, s.v, s.rotary, branches=c["K"], q=s.q, counts=s.counts)
        return (q, *s.cache.read(0, s.seqs, s.start, _nodes(c) + BLOCK - 1, counts=s.live))
    return s.cache.attend_shared(0, s.seqs, s.q, c["G"], branches=c["K"])


def run(state):
    if own:
        return _run_own(state)
    return {"rotate": _run_rotate, "append": _run_append, "shared": _run_shared}[state.case["op"]](state)


# ------------------------------------------------------------------ cost


def work(case):
    B, n, Hq, H, D, K, L = case["B"], _nodes(case), case["Hq"], case["Hkv"], case["D"], case["K"], case["L"]
    es = 4 if case["dtype"] == "f32" else 2
    per = 2 * H * (D + 4 / BLOCK)                    # a token's stored bytes, and its share of scales
    if case["op"] == "shared":
        held = sum(_prefixes(case)) + sum(_lens(case))
        pairs = K * (L * (L + 1) // 2) * B
        for b, t in enumerate(_lens(case)):
            pairs += n * (_prefixes(case)[b // case["G"]] + t + 1)
        return {"bytes": (held + B * n) * per + 2 * B * n * Hq * D * es, "flops": 4 * D * Hq * pairs}
    live = sum(_counts(case))
    turned = 2 * live * Hq * D * es
    if case["op"] == "rotate":
        return {"bytes": turned, "flops": 3 * live * Hq * case["dim"]}
    old = sum(t % BLOCK for t in _lens(case))
    new = 2 * H * D * es
    # new tokens in, their bytes out, the begun block in, values back
    return {"bytes": turned + live * (new + per) + old * per + (live + old) * new, "flops": 3 * live * (Hq + H) * case["dim"]}


# ------------------------------------------------------- values in 64 bits


def _exact_angles(case, pos):
    """cos and sin [.., dim / 2] at positions, the frequency in two parts so
    that the products are exact."""
    f = []
    for i in range(case["dim"] // 2):
        x = math.pow(case["base"], -2.0 * i / case["dim"])
        turns = case["original"] * x / (2.0 * math.pi)
        ramp = min(max((turns - 1.0) / 31.0, 0.0), 1.0) if case["original"] else 0.0
        f.append(ramp * x + (1.0 - ramp) * x / case["factor"])
    high = [math.ldexp(math.floor(math.ldexp(x, 31)), -31) for x in f]
    a, b = (pos[..., None].double() * torch.tensor(y, device="cuda", dtype=torch.float64)
            for y in (high, [x - h for x, h in zip(f, high)]))
    return a.cos() * b.cos() - a.sin() * b.sin(), a.sin() * b.cos() + a.cos() * b.sin()


def _exact_rotated(case, x):
    """x [B][n][heads][D] in 64 bits, a pair of dimensions after another."""
    lens = torch.tensor(_lens(case), device="cuda")
    depth = torch.tensor([0] + [j + 1 for _ in range(case["K"]) for j in range(case["L"])], device="cuda")
    c, s = _exact_angles(case, lens[:, None] + depth)
    y, m, half = x.double().clone(), case["magnitude"], case["dim"] // 2
    for i in range(half):
        u, w = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + half)
        a, b = x[..., u].double(), x[..., w].double()
        y[..., u] = m * (a * c[..., None, i] - b * s[..., None, i])
        y[..., w] = m * (a * s[..., None, i] + b * c[..., None, i])
    return y


def _exact_block(x):
    """Values that blocks [..., 16, D] of one head stand for."""
    a = x.abs().amax((-2, -1), keepdim=True)
    e = torch.ceil(torch.log2(a.clamp(min=1e-300) / 448.0)).clamp(-117, 119)
    scale = torch.exp2(e)
    scale = torch.where(a > 448.0 * scale, 2 * scale, torch.where(a <= 224.0 * scale, scale / 2, scale))
    y = x / scale
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    step = torch.where(y.abs() >= 16 * step, 2 * step, torch.where(y.abs().clamp(min=2.0 ** -6) < 8 * step, step / 2, step))
    return torch.round(y / step) * step * scale


def _exact_tokens(*parts):
    """The values of one sequence's tokens [T, H, D], stored part by part."""
    y = parts[0][:0].double()
    for x in parts:
        if x.shape[0]:
            y = torch.cat([y, x.double()])
            t = y.shape[0]
            at = t - x.shape[0]
            at -= at % BLOCK
            z = torch.nn.functional.pad(y[at:], (0, 0, 0, 0, 0, -t % BLOCK)).unflatten(0, (-1, BLOCK))
            z = _exact_block(z.transpose(1, 2)).transpose(1, 2).flatten(0, 1)[:t - at]
            y = torch.cat([y[:at], z])
    return y


def exact(case, seed):
    n, lens, B, H, D = _nodes(case), _lens(case), case["B"], case["Hkv"], case["D"]
    if case["op"] == "shared":
        K, L, G, g = case["K"], case["L"], case["G"], case["Hq"] // case["Hkv"]
        q, tokens = _conversation(case, seed)
        o = torch.empty_like(q, dtype=torch.float64)
        chain = torch.eye(n, dtype=torch.bool, device="cuda")
        chain[:, 0] = True
        for k in range(K):
            at = 1 + k * L
            chain[at:at + L, at:at + L] = torch.ones(L, L, device="cuda").tril().bool()
        for b, t in enumerate(lens):
            p = _prefixes(case)[b // G]
            k, v = (_exact_tokens(tokens[0][i][b // G, :p], tokens[1][i][b, :t], tokens[2][i][b]) for i in range(2))
            see = torch.cat([torch.ones(n, p + t, dtype=torch.bool, device="cuda"), chain], 1)
            for h in range(H):
                z = torch.einsum("ngd,td->gnt", q[b, :, h * g:(h + 1) * g].double(), k[:, h]) / math.sqrt(D)
                z = z.masked_fill(~see, -math.inf)
                o[b, :, h * g:(h + 1) * g] = torch.einsum("gnt,td->ngd", torch.softmax(z, -1), v[:, h])
        return o
    counts = _counts(case)
    q, k, v = _projected(case, seed)
    turned = _exact_rotated(case, q)
    for b in range(B):
        turned[b, counts[b]:] = 0.0
    if case["op"] == "rotate":
        return turned
    got = [torch.zeros(B, n + BLOCK - 1, H, D, dtype=torch.float64, device="cuda") for _ in range(2)]
    for x, old, y in zip((_exact_rotated(case, k), v), _begun(case, seed), got):
        for b, t in enumerate(lens):
            z = _exact_tokens(old[b, :t % BLOCK], x[b, :counts[b]])
            y[b, :z.shape[0]] = z
    return (turned, *got)
