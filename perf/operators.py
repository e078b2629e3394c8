"""Cases of the key/value cache behind the verification of draft trees: the
operators that a target model runs around `mds.Verifier.verify`.

The cache holds keys and values in 8 bits (e4m3) in pages of tokens, with one
power-of-two scale for every block of 16 tokens and head.  A step of
multi-draft decoding appends the n = 1 + K * L tokens of a draft tree (node 0
the root, node 1 + k * L + j branch k's draft at depth j + 1) behind the
committed tokens of each sequence, attends with every node over the committed
tokens, the root and the node's own branch, and, once the tree is verified,
keeps the root and the accepted branch's tokens and gives the other pages
back.  K = 1 is a plain chain: one token (n = 1) or a chunk of a prompt.

Three operators:

attend  o = sum_t softmax_t(scale * q . k_t) v_t over the visible tokens; with
        a window W and S sinks, a key at position p (committed tokens, then
        the tree by depth) is seen from position x if p < S or p > x - W.
append  the block quantiser Q: a = max|x| over the block's live tokens, e the
        least integer with a <= 448 * 2^e, each value rounded to e4m3(x / 2^e);
        a block that already holds tokens is quantised again with the new ones
        from the values it stands for.  The pass reads the new tokens and the
        block they begin in back as values.
pages   fork sequences onto new ones (pages shared), make the forks' tail
        pages their own (copies), keep the accepted branch (compaction), read
        the copies' last tokens, give the forks' pages back.  Page ids go to
        the lowest free page, sequence by sequence.

Sequences' lengths are spread evenly over the case's range.
"""
import math

import torch

own = False

BLOCK = 16
STORAGE = {"f32": torch.float32, "bf16": torch.bfloat16}
VOCAB = 32000


# ------------------------------------------------------------------ cases


def _attend(name, B, lo, hi, K=1, L=0, Hq=32, Hkv=8, D=128, page=64, dtype="bf16", window=0, sinks=0):
    return {"name": name, "op": "attend", "B": B, "lo": lo, "hi": hi, "K": K, "L": L, "Hq": Hq, "Hkv": Hkv, "D": D,
            "page": page, "dtype": dtype, "window": window, "sinks": sinks}


def _append(name, B, lo, hi, K=1, L=0, Hkv=8, D=128, page=64, dtype="bf16"):
    return {"name": name, "op": "append", "B": B, "lo": lo, "hi": hi, "K": K, "L": L, "Hkv": Hkv, "D": D,
            "page": page, "dtype": dtype}


def _pages(name, B, lo, hi, layers, K, L, Hkv=8, D=128, page=64):
    return {"name": name, "op": "pages", "B": B, "lo": lo, "hi": hi, "layers": layers, "K": K, "L": L, "Hkv": Hkv,
            "D": D, "page": page, "dtype": "bf16"}


def listed():
    return [
        # one interactive user, one token: latency
        _attend("attend-one-token", 1, 4100, 4100),
        # a ragged batch that decodes token by token
        _attend("attend-batch-token", 64, 1, 8191),
        # the 32k workload's tree (4 branches of 5), every head with keys of its own
        _attend("attend-tree-4x5", 64, 500, 2000, K=4, L=5, Hq=32, Hkv=32),
        # the 128k workload's batch and tree (8 branches of 4), shared heads
        _attend("attend-tree-8x4", 256, 257, 1537, K=8, L=4),
        # the 50k workload's tree (2 branches of 4) at long context: window and sinks
        _attend("attend-window-2x4", 32, 20001, 40001, K=2, L=4, Hq=64, Hkv=8, D=64, window=4096, sinks=4),
        # a few sequences with long caches
        _attend("attend-long-token", 8, 65537, 131071),
        # 32-bit queries, small pages, a short window
        _attend("attend-f32-3x3", 5, 1, 777, K=3, L=3, Hq=12, Hkv=4, D=64, page=16, dtype="f32", window=100, sinks=3),
        # a chunk of two prompts behind what the cache holds
        _attend("attend-prompt-chunk", 2, 4001, 5003, K=1, L=1020),
        # one layer's trees of the 128k workload's batch
        _append("append-tree-8x4", 256, 257, 1537, K=8, L=4),
        # one layer of four prompts of an odd length, 32-bit inputs, onto empty sequences
        _append("append-prompt-f32", 4, 0, 0, K=1, L=4098, dtype="f32", page=32),
        # a few sequences of a small model
        _pages("pages-small", 8, 100, 400, layers=2, K=2, L=4, Hkv=4, D=64, page=32),
        # every layer of a 16-layer model, the 128k workload's batch and tree
        _pages("pages-tree-8x4", 256, 257, 1537, layers=16, K=8, L=4),
    ]


def draw(rng):
    """A case of the same ranges: batches of 1 to 256, caches of 0 to 131072
    tokens, single tokens, trees and prompt chunks, both head widths, shared
    heads of 1 to 16, odd lengths throughout."""
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["attend", "attend", "attend", "attend", "append", "pages"])
    D = rng.choice([64, 128, 128])
    page = rng.choice([16, 32, 64, 64, 128])
    K, L = rng.choice([(1, 0), (1, 0), (2, 4), (4, 5), (8, 4), (4, 8), (3, 3), (1, 7), (16, 2), (1, -1)])
    if L < 0:
        L = spread(30, 1021) if op == "attend" else spread(30, 4099)
    n = 1 + K * L
    Hkv = rng.choice([1, 2, 4, 8, 8, 32])
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    B = spread(1, 256)
    hi = spread(1, 131071)
    lo = rng.choice([0, hi // 4, hi])
    if op == "attend":
        g = rng.choice([1, 3, 4, 8, 16]) if Hkv <= 8 else 1
        window = rng.choice([0, 0, spread(16, 8192)])
        # no more than the largest listed case: cache bytes, and products of queries and keys
        B = max(1, min(B, int(8e8 / (hi + n) / (Hkv * D))))
        seen = min(hi, window) if window else hi
        B = max(1, min(B, int(4e10 / ((seen + n) * n * Hkv * g * D))))
        hi = max(1, min(hi, int(4e10 / (n * Hkv * g * D)) - n)) if B == 1 else hi
        B = max(1, min(B, int(7e8 / (n * Hkv * g * (hi + n)))))
        hi = max(1, min(hi, int(7e8 / (n * Hkv * g)) - n))
        c = _attend("", B, min(lo, hi), hi, K, L, Hkv * g, Hkv, D, page, dtype, window, rng.choice([0, 1, 4, 40]) if window else 0)
    elif op == "append":
        B = max(1, min(B, int(1.7e7 / (n * Hkv * D))))
        hi = max(1, min(hi, int(4e8 / (B * Hkv * D))))
        c = _append("", B, min(lo, hi), hi, K, L, Hkv, D, page, dtype)
    else:
        layers = rng.choice([1, 2, 5, 16])
        hi = max(1, min(hi, 4099))
        B = max(1, min(B, int(6e9 / ((hi + n + page) * layers * Hkv * D * 2)), int(3e8 / ((page + n) * layers * Hkv * D))))
        c = _pages("", B, min(lo, hi), hi, layers, K, L, Hkv, D, page)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs


def _lens(case):
    """Committed tokens of every sequence: the range's ends' even spread."""
    lo, hi = case["lo"], case["hi"]
    return [lo + int((hi - lo + 1) * (((b + 1) * 0.6180339887498949) % 1.0)) for b in range(case["B"])]


def _nodes(case):
    return 1 + case["K"] * case["L"]


def _span(case):
    """Tokens of the longest sequence with its tree, in whole pages."""
    return -(-(max(_lens(case)) + _nodes(case)) // case["page"]) * case["page"]


def _tokens(case, seed, layer):
    """Keys and values of every sequence's tokens [B][T][Hkv][D]: normals with
    an offset per channel on the keys and a magnitude per token."""
    B, T, H, D = case["B"], _span(case), case["Hkv"], case["D"]
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 64 + layer + 1)
    st = STORAGE[case["dtype"]]
    offset = 2.0 * torch.randn(H, D, generator=g, device="cuda")
    size = torch.exp(0.5 * torch.randn(2, B, T, 1, 1, generator=g, device="cuda"))
    k = torch.randn(B, T, H, D, generator=g, device="cuda").mul_(size[0]).add_(offset).to(st)
    v = torch.randn(B, T, H, D, generator=g, device="cuda").mul_(size[1]).to(st)
    return k, v


def _tail(x, lens, n):
    """The tokens [len, len + n) of every sequence."""
    at = lens[:, None] + torch.arange(n, device=x.device)
    return x[torch.arange(x.shape[0], device=x.device)[:, None], at].contiguous()


def _queries(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 64 + 63)
    q = 1.5 * torch.randn(case["B"], _nodes(case), case["Hq"], case["D"], generator=g, device="cuda")
    return q.to(STORAGE[case["dtype"]])


def _verdict(case, seed):
    """Draft tokens [B][K][L], and a verification's emitted tokens [B][L+1]
    and accepted lengths [B] on them."""
    B, K, L = case["B"], case["K"], case["L"]
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 64 + 62)
    drafts = torch.randint(VOCAB, (B, K, L), generator=g, device="cuda", dtype=torch.int32)
    accept = torch.randint(L + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    branch = torch.randint(K, (B,), generator=g, device="cuda")
    out = torch.full((B, L + 1), -1, device="cuda", dtype=torch.int32)
    if L:
        depth = torch.arange(L, device="cuda")
        out[:, :L] = torch.where(depth < accept[:, None], drafts[torch.arange(B, device="cuda"), branch], -1)
    out.scatter_(1, accept[:, None].long(), torch.randint(VOCAB, (B, 1), generator=g, device="cuda", dtype=torch.int32))
    return drafts, out, accept


# ------------------------------------------------- the plain form's cache


def _quantise(x):
    """Q on blocks [..., 16, H, D] in 32 bits: bytes, and scales [..., H]."""
    a = x.abs().amax(dim=(-3, -1))
    m, e = torch.frexp(a)
    e = torch.where(m <= 0.875, e - 9, e - 8).clamp(-117, 120)
    e = torch.where(a > 0, e, 0)
    return (torch.ldexp(x, -e[..., None, :, None])).to(torch.float8_e4m3fn), torch.ldexp(torch.ones_like(a), e)


def _values(by, scale):
    return by.float() * scale[..., None, :, None]


def _blocks(x):
    """[B, T, H, D] in 32 bits as blocks [B, T / 16, 16, H, D]."""
    return x.float().unflatten(1, (-1, BLOCK))


def _fill(x, lens, n):
    """Blocks of the committed tokens, quantised, then with n more behind them
    (quantised again where a block holds both)."""
    t = torch.arange(x.shape[1], device=x.device)
    live = (t < lens[:, None])[..., None, None]
    x = x.float()
    by, sc = _quantise(_blocks(torch.where(live, x, 0.0)))
    if n:
        new = (t < lens[:, None] + n)[..., None, None] & ~live
        x = torch.where(live, _values(by, sc).flatten(1, 2), torch.where(new, x, 0.0))
        by, sc = _quantise(_blocks(x))
    return by, sc


def _table(case, lens, n):
    """Page ids in the order that the sequences take them: the committed
    tokens' pages, then the pages that n more tokens need."""
    P, width = case["page"], _span(case) // case["page"]
    first, both = (lens + P - 1) // P, (lens + n + P - 1) // P
    i = torch.arange(width, device=lens.device)
    a = (torch.cumsum(first, 0) - first)[:, None] + i
    more = both - first
    b = first.sum() + (torch.cumsum(more, 0) - more)[:, None] + i - first[:, None]
    return torch.where(i < first[:, None], a, torch.where(i < both[:, None], b, -1))


class _Plain:
    """The plain form's state: pools [layers][pages][2][H][page][D] of bytes
    and [layers][pages][2][H][page / 16] of scales, page table, counts."""

    def __init__(self, case, seed, layers, pending):
        P, H, D = case["page"], case["Hkv"], case["D"]
        self.lens = torch.tensor(_lens(case), device="cuda")
        self.table = _table(case, self.lens, pending)
        self.pages = _pool_pages(case)
        self.bytes = torch.zeros(layers, self.pages, 2, H, P, D, dtype=torch.uint8, device="cuda")
        self.scales = torch.ones(layers, self.pages, 2, H, P // BLOCK, device="cuda")
        b, i = torch.nonzero(self.table >= 0, as_tuple=True)
        ids = self.table[b, i]
        for layer in range(layers):
            for kv, x in enumerate(_tokens(case, seed, layer)):
                by, sc = _fill(x, self.lens, pending)
                by = by.view(torch.uint8).flatten(1, 2).unflatten(1, (-1, P))       # [B][page][P][H][D]
                sc = sc.unflatten(1, (-1, P // BLOCK))                              # [B][page][P/16][H]
                self.bytes[layer, ids, kv] = by[b, i].transpose(1, 2)
                self.scales[layer, ids, kv] = sc[b, i].transpose(1, 2)


def _pool_pages(case):
    P, n = case["page"], _nodes(case)
    held = sum(-(-(t + n) // P) for t in _lens(case))
    # the forks' own pages: the one that the tree begins in and those behind it
    return held + (case["B"] * (-(-n // P) + 1) if case["op"] == "pages" else 0)


def _gather(by, sc, table, t, P):
    """Values [.., B, T, H, D] of the tokens t [B, T] under a page table."""
    page = torch.gather(table, 1, t // P)
    off = t % P
    x = by[..., page, :, :, off, :].view(torch.float8_e4m3fn).float()      # the indexed axes come first
    s = sc[..., page, :, :, off // BLOCK]
    return x * s[..., None]


def _layer_values(state, layer, table, t, P):
    """Keys and values [B, T, H, D] of one layer in 32 bits."""
    x = _gather(state.bytes[layer], state.scales[layer], table, t, P)      # [B, T, 2, H, D]
    return x[:, :, 0], x[:, :, 1]


# ------------------------------------------------------------------ passes


class _State:
    pass


def prepare(case, seed):
    s = _State()
    s.case = case
    n = _nodes(case)
    op = case["op"]
    layers = case.get("layers", 1)
    lens = torch.tensor(_lens(case), device="cuda")
    if op == "attend":
        s.q = _queries(case, seed)
    if op == "append":
        s.k, s.v = (_tail(x, lens, n) for x in _tokens(case, seed, 0))
        s.start = (lens // BLOCK * BLOCK).int()
        s.live = (lens + n).int() - s.start
    if op == "pages":
        s.drafts, s.out, s.accept = _verdict(case, seed)
        s.start = (lens // case["page"] * case["page"]).int()
    pending = 0 if op == "append" else n
    if own:
        from paper_2410_18234_gb300 import cache
        B = case["B"]
        s.cache = cache.Cache(layers, _pool_pages(case), case["Hkv"], case["D"], 2 * B if op == "pages" else B,
                              _span(case) // case["page"], page_tokens=case["page"], dtype=case["dtype"])
        s.seqs = torch.arange(B, device="cuda", dtype=torch.int32)
        s.forks = s.seqs + B
        s.cache.reserve(s.seqs, _span(case), counts=lens.int())
        tails = []
        for layer in range(layers):
            k, v = _tokens(case, seed, layer)
            s.cache.append(layer, s.seqs, k, v, counts=lens.int())
            tails.append((_tail(k, lens, n), _tail(v, lens, n)) if pending else ())
        s.cache.commit(s.seqs, lens.int() - 1, length=_span(case) - 1)
        s.cache.reserve(s.seqs, n)
        for layer in range(layers if pending else 0):
            s.cache.append(layer, s.seqs, *tails[layer])
        return s
    s.plain = _Plain(case, seed, layers, pending)
    if op == "append":
        s.plain.table = _table(case, lens, n)
    return s


def _run_own(s):
    c = s.case
    if c["op"] == "attend":
        return s.cache.attend(0, s.seqs, s.q, branches=c["K"], window=c["window"], sinks=c["sinks"])
    if c["op"] == "append":
        s.cache.append(0, s.seqs, s.k, s.v)
        return s.cache.read(0, s.seqs, s.start, _nodes(c) + BLOCK - 1, counts=s.live)
    s.cache.fork(s.seqs, s.forks)
    s.cache.reserve(s.forks, _nodes(c))
    s.cache.commit(s.forks, s.accept, branches=c["K"], length=c["L"], draft_tokens=s.drafts, out_tokens=s.out)
    lens, table = s.cache.lens[c["B"]:].clone(), s.cache.table[c["B"]:].clone()
    k, v = s.cache.read(None, s.forks, s.start, c["page"] + c["L"], counts=lens - s.start)
    s.cache.free(s.forks)
    return lens, table, k, v


def _run_attend(s):
    c, p = s.case, s.plain
    B, n, Hq, H, D, L = c["B"], _nodes(c), c["Hq"], c["Hkv"], c["D"], c["L"]
    t = torch.arange(_span(c), device="cuda")
    k, v = _layer_values(p, 0, p.table.clamp(min=0), t.expand(B, -1), c["page"])
    q = s.q.float().view(B, n, H, Hq // H, D).permute(0, 2, 3, 1, 4).reshape(B, H, -1, D)
    score = torch.matmul(q, k.permute(0, 2, 3, 1)).view(B, H, Hq // H, n, -1) * (1.0 / math.sqrt(D))
    del k
    # node of each slot (below 0: committed), its branch and position
    node = t - p.lens[:, None]                                            # [B, T]
    me = torch.arange(n, device="cuda")
    depth = torch.where(node > 0, (node - 1) % max(L, 1) + 1, node)
    mine = torch.where(me > 0, (me - 1) % max(L, 1) + 1, 0)
    branch, my_branch = (node - 1) // max(L, 1), (me - 1) // max(L, 1)
    see = (node[:, None] <= 0) | ((branch[:, None] == my_branch[:, None]) & (node[:, None] <= me[:, None]))
    if c["window"]:
        pos, my_pos = p.lens[:, None] + depth, p.lens[:, None] + mine
        see &= (pos[:, None] < c["sinks"]) | (pos[:, None] > my_pos[:, :, None] - c["window"])
    score.masked_fill_(~see[:, None, None], -math.inf)
    w = torch.exp(score - score.amax(-1, keepdim=True))
    del score
    w /= w.sum(-1, keepdim=True)
    o = torch.matmul(w.view(B, H, -1, w.shape[-1]), v.permute(0, 2, 1, 3)).view(B, H, Hq // H, n, D)
    return o.permute(0, 3, 1, 2, 4).reshape(B, n, Hq, D).to(s.q.dtype)


def _run_append(s):
    c, p = s.case, s.plain
    P, n = c["page"], _nodes(c)
    count = -(-(n + BLOCK - 1) // BLOCK) * BLOCK
    i = torch.arange(count, device="cuda")
    t = s.start.long()[:, None] + i
    old = i < (p.lens - s.start)[:, None]
    live = i < s.live[:, None]
    table = torch.nn.functional.pad(p.table, (0, -(-count // P) + 1), value=-1)
    b, j = torch.nonzero(live, as_tuple=True)
    page, off = table[b, t[b, j] // P], t[b, j] % P
    head = torch.where(live & ~old, 0, t.clamp(max=_span(c) - 1))
    was = _layer_values(p, 0, table.clamp(min=0), head, P)
    got = []
    for kv, (x, w) in enumerate(zip((s.k, s.v), was)):
        new = torch.gather(x.float(), 1, (t - p.lens[:, None]).clamp(0, n - 1)[..., None, None].expand(-1, -1, *x.shape[2:]))
        y = torch.where(old[..., None, None], w, torch.where(live[..., None, None], new, 0.0))
        by, sc = _quantise(_blocks(y))
        p.bytes[0, page, kv, :, off] = by.view(torch.uint8).flatten(1, 2)[b, j]
        p.scales[0, page, kv, :, off // BLOCK] = sc[b, j // BLOCK]
        got.append((_values(by, sc).flatten(1, 2)[:, :n + BLOCK - 1]).to(x.dtype))
    return tuple(got)


def _run_pages(s):
    c, p = s.case, s.plain
    B, P, K, L, n = c["B"], c["page"], c["K"], c["L"], _nodes(c)
    lens, width = p.lens, p.table.shape[1]
    # fork and copy on write: the pages from len / P on become the fork's own
    i = torch.arange(width, device="cuda")
    need = (lens + n + P - 1) // P
    mine = (i >= (lens // P)[:, None]) & (i < need[:, None])
    ref = torch.zeros(p.pages, device="cuda", dtype=torch.long)
    ref.scatter_add_(0, p.table.clamp(min=0).flatten(), (p.table >= 0).flatten().long())
    free = torch.nonzero(ref == 0).flatten()
    table = p.table.clone()
    b, j = torch.nonzero(mine, as_tuple=True)
    fresh = free[:b.shape[0]]
    p.bytes[:, fresh] = p.bytes[:, table[b, j]]
    p.scales[:, fresh] = p.scales[:, table[b, j]]
    table[b, j] = fresh
    # the lowest branch whose tokens are the emitted ones
    a = s.accept.long()
    depth = torch.arange(L, device="cuda")
    same = ((s.drafts == s.out[:, None, :L]) | (depth >= a[:, None, None])).all(-1)
    branch = same.int().argmax(1)
    # tokens from the tail page's start: committed, root, branch
    total = lens + 1 + a
    t = s.start.long()[:, None] + torch.arange(P + L, device="cuda")
    src = torch.where(t <= lens[:, None], t, t + branch[:, None] * L)
    live = t < total[:, None]
    src = torch.where(live, src, 0)
    t = torch.where(live, t, 0)
    tail = _gather(p.bytes, p.scales, table.clamp(min=0), src, P)          # [B, T, layers, 2, H, D]
    x = torch.where(live[..., None, None, None, None], tail, 0.0)
    pad = -(-(P + L) // BLOCK) * BLOCK - (P + L)
    x = torch.nn.functional.pad(x, (0, 0) * 4 + (0, pad)).permute(0, 2, 3, 1, 4, 5).unflatten(3, (-1, BLOCK))
    by, sc = _quantise(x)                                                  # [B, layers, 2, blocks, 16, H, D]
    val = _values(by, sc).flatten(3, 4)[:, :, :, :P + L]
    # the blocks from the one that holds the root on are written back
    back = live & (t >= (lens // BLOCK * BLOCK)[:, None])
    b, j = torch.nonzero(back, as_tuple=True)
    page, off = table[b, t[b, j] // P], t[b, j] % P
    flat = by.view(torch.uint8).flatten(3, 4)
    p.bytes[:, page, :, :, off] = flat[b, :, :, j]
    p.scales[:, page, :, :, off // BLOCK] = sc[b, :, :, j // BLOCK]
    table[i >= ((total + P - 1) // P)[:, None]] = -1
    k, v = val[:, :, 0].transpose(0, 1), val[:, :, 1].transpose(0, 1)      # [layers, B, T, H, D]
    return total.int(), table.int(), k.bfloat16(), v.bfloat16()


def run(state):
    if own:
        return _run_own(state)
    return {"attend": _run_attend, "append": _run_append, "pages": _run_pages}[state.case["op"]](state)


# ------------------------------------------------------------------ cost


def _visible(case):
    """Per sequence: committed keys that a window leaves to any node, and
    pairs of nodes and visible keys."""
    K, L, W, S = case["K"], case["L"], case.get("window", 0), case.get("sinks", 0)
    keys, pairs = 0, 0
    for t in _lens(case):
        keys += t if not W else min(t, S + max(0, t - max(S, t - W + 1)))
        if not W:
            pairs += (1 + K * L) * (t + 1) + K * (L * (L + 1) // 2)
        else:
            for d in range(L + 1):
                x = t + d + 1
                pairs += (K if d else 1) * min(x, W + min(S, max(0, x - W)))
    return keys, pairs


def work(case):
    B, n, H, D = case["B"], _nodes(case), case["Hkv"], case["D"]
    es = 4 if case["dtype"] == "f32" else 2
    per = 2 * H * (D + 4 / BLOCK)                    # a token's bytes, and its share of scales
    if case["op"] == "attend":
        keys, pairs = _visible(case)
        return {"bytes": (keys + B * n) * per + 2 * B * n * case["Hq"] * D * es, "flops": 4 * D * case["Hq"] * pairs}
    if case["op"] == "append":
        old = sum(t % BLOCK for t in _lens(case))
        new = 2 * H * D * es
        # new tokens in, their bytes out, the begun block in, values back
        return {"bytes": B * n * (new + per) + old * per + (B * n + old) * new, "flops": 0}
    # the copied pages' tokens in and out; values back for those that stay (half the depths on average)
    P = case["page"]
    copied = sum(t % P + n for t in _lens(case))
    kept = sum(t % P + 1 + case["L"] / 2 for t in _lens(case))
    return {"bytes": case["layers"] * (2 * copied * per + kept * 2 * H * D * 2), "flops": 0}


# ------------------------------------------------------- values in 64 bits


def _round_e4m3(y):
    """Nearest e4m3 value, ties to even mantissas, of 64-bit numbers up to 448."""
    _, e = torch.frexp(y)
    step = torch.exp2((e - 1).clamp(min=-6).double() - 3)
    return torch.round(y / step) * step


def _exact_block(x):
    """Values that blocks [..., 16, D] of one head stand for."""
    a = x.abs().amax((-2, -1), keepdim=True)
    e = torch.ceil(torch.log2(a.clamp(min=1e-300) / 448.0)).clamp(-117, 120)
    scale = torch.exp2(e)
    scale = torch.where(a > 448.0 * scale, 2 * scale, torch.where(a <= 224.0 * scale, scale / 2, scale))
    return _round_e4m3(x / scale) * scale


def _exact_tokens(x, t, n):
    """The values of one sequence's t committed and n new tokens [T, H, D]."""
    T = -(-(t + n) // BLOCK) * BLOCK
    y = torch.zeros(T, *x.shape[1:], dtype=torch.float64, device=x.device)
    for upto in ([t, t + n] if n else [t]):
        done = 0 if upto == t else t
        y[done:upto] = x[done:upto].double()
        y = _exact_block(y.view(-1, BLOCK, *x.shape[1:]).transpose(1, 2)).transpose(1, 2).reshape(T, *x.shape[1:])
    return y[:t + n]


def exact(case, seed):
    n, lens = _nodes(case), _lens(case)
    B, H, D, K, L = case["B"], case["Hkv"], case["D"], case["K"], case["L"]
    if case["op"] == "attend":
        k, v = _tokens(case, seed, 0)
        q = _queries(case, seed).double()
        o = torch.empty_like(q)
        for b, t in enumerate(lens):
            kb, vb = (_exact_tokens(x[b], t, n) for x in (k, v))
            see = torch.zeros(n, t + n, dtype=torch.bool, device="cuda")
            pos = torch.arange(t + n, device="cuda")
            for br in range(K):
                at = 1 + br * L
                pos[t + at:t + at + L] = t + 1 + torch.arange(L, device="cuda")
                see[at:at + L, t + at:t + at + L] = torch.ones(L, L, device="cuda").tril().bool()
            see[:, :t + 1] = True
            if case["window"]:
                see &= (pos < case["sinks"]) | (pos > pos[t:, None] - case["window"])
            for h in range(case["Hq"]):
                hk = h // (case["Hq"] // H)
                z = (q[b, :, h] @ kb[:, hk].T) / math.sqrt(D)
                z = z.masked_fill(~see, -math.inf)
                o[b, :, h] = torch.softmax(z, 1) @ vb[:, hk]
        return o
    if case["op"] == "append":
        got = [torch.zeros(B, n + BLOCK - 1, H, D, dtype=torch.float64, device="cuda") for _ in range(2)]
        for x, y in zip(_tokens(case, seed, 0), got):
            for b, t in enumerate(lens):
                z = _exact_tokens(x[b], t, n)[t // BLOCK * BLOCK:]
                y[b, :z.shape[0]] = z
        return tuple(got)
    P = case["page"]
    drafts, out, accept = (x.tolist() for x in _verdict(case, seed))
    got = [torch.zeros(case["layers"], B, P + L, H, D, dtype=torch.float64, device="cuda") for _ in range(2)]
    for layer in range(case["layers"]):
        for x, y in zip(_tokens(case, seed, layer), got):
            for b, t in enumerate(lens):
                a = accept[b]
                br = next(i for i in range(K) if drafts[b][i][:a] == out[b][:a])
                z = _exact_tokens(x[b], t, n)
                at = t + 1 + br * L
                z = torch.cat([z[:t + 1], z[at:at + a]])
                z = _exact_tokens(z, z.shape[0], 0)[t // P * P:]
                y[layer, b, :z.shape[0]] = z
    return (None, None, *got)
