"""A plain 64-bit model of the key/value cache, for the tests: pages are
arrays of values, every rule is taken from include/mds_cache.h.  numpy only;
nothing of the library is used."""
import numpy as np

BLOCK = 16


def round_e4m3(y):
    """Nearest e4m3 number (|y| <= 448), ties to even mantissas."""
    _, e = np.frexp(y)
    step = np.exp2(np.maximum(e - 1, -6) - 3.0)
    return np.rint(y / step) * step


def quantise(x):
    """Values that a block [16, D] stands for."""
    finite = np.where(np.isfinite(x), x, 0.0)
    a = np.abs(finite).max()
    e = 0
    if a > 0:
        e = int(np.clip(np.ceil(np.log2(a / 448.0)), -117, 119))
        while e < 119 and a > 448.0 * 2.0 ** e:
            e += 1
        while e > -117 and a <= 448.0 * 2.0 ** (e - 1):
            e -= 1
    y = np.clip(np.where(np.isnan(x), 0.0, x) / 2.0 ** e, -448.0, 448.0)
    return round_e4m3(y) * 2.0 ** e


class Model:
    def __init__(self, layers, pages, kv_heads, head_dim, max_seqs, max_pages, page_tokens):
        self.layers, self.pages, self.P = layers, pages, page_tokens
        self.H, self.D, self.max_pages = kv_heads, head_dim, max_pages
        self.data = np.zeros((pages, layers, 2, kv_heads, page_tokens, head_dim))
        self.ref = [0] * pages
        self.lens = [0] * max_seqs
        self.rows = [[] for _ in range(max_seqs)]

    def table(self):
        t = np.full((len(self.rows), self.max_pages), -1, np.int32)
        for q, r in enumerate(self.rows):
            t[q, :len(r)] = r
        return t

    def _drop(self, pages):
        for p in pages:
            self.ref[p] -= 1

    def reserve(self, seqs, counts):
        """Ids of the sequences that got none."""
        free = [p for p in range(self.pages) if self.ref[p] == 0]
        shared = [r > 1 for r in self.ref]
        at, short, drop = 0, [], []
        for q, n in zip(seqs, counts):
            if q < 0 or n == 0:
                continue
            first, end = self.lens[q] // self.P, -(-(self.lens[q] + n) // self.P)
            if end > self.max_pages:
                short.append(q)
                continue
            need = [p for p in range(first, end) if p >= len(self.rows[q]) or shared[self.rows[q][p]]]
            if at + len(need) > len(free):
                short.append(q)
                at += len(need)
                continue
            for p in need:
                new = free[at]
                at += 1
                self.ref[new] = 1
                if p < len(self.rows[q]):
                    old = self.rows[q][p]
                    live = -(-min(self.P, self.lens[q] + n - p * self.P) // BLOCK) * BLOCK
                    self.data[new][..., :live, :] = self.data[old][..., :live, :]
                    drop.append(old)
                    self.rows[q][p] = new
                else:
                    self.rows[q].append(new)
        self._drop(drop)
        return short

    def get(self, q, layer, start, n):
        """[2][n][H][D]"""
        out = np.zeros((2, n, self.H, self.D))
        for i in range(n):
            p, r = divmod(start + i, self.P)
            if p < len(self.rows[q]):
                out[:, i] = self.data[self.rows[q][p], layer, :, :, r]
        return out

    def put(self, q, layer, old, new):
        """Values new [2][n][H][D] from slot `old` on; the block that it
        begins in is quantised with the tokens in front."""
        n = new.shape[1]
        if n == 0:
            return
        t0 = old // BLOCK * BLOCK
        x = np.concatenate([self.get(q, layer, t0, old - t0), new], 1)
        for b in range(0, x.shape[1], BLOCK):
            blk = x[:, b:b + BLOCK]
            for kv in range(2):
                for h in range(self.H):
                    y = quantise(blk[kv, :, h])
                    p, r = divmod(t0 + b, self.P)
                    self.data[self.rows[q][p], layer, kv, h, r:r + y.shape[0]] = y

    def append(self, layer, seqs, counts, k, v):
        for b, (q, n) in enumerate(zip(seqs, counts)):
            if q >= 0:
                self.put(q, layer, self.lens[q], np.stack([k[b, :n], v[b, :n]]))

    def commit(self, seqs, accept, K=1, L=0, drafts=None, out=None):
        for b, q in enumerate(seqs):
            if q < 0:
                continue
            a, k, at = accept[b], 0, self.lens[q]
            if drafts is not None and a > 0:
                k = next(i for i in range(K) if list(drafts[b][i][:a]) == list(out[b][:a]))
            if a > 0 and k > 0:
                moved = [self.get(q, layer, at + 1 + k * L, a) for layer in range(self.layers)]
                for layer in range(self.layers):
                    self.put(q, layer, at + 1, moved[layer])
            self._cut(q, at + 1 + a)

    def _cut(self, q, n):
        keep = -(-n // self.P)
        self._drop(self.rows[q][keep:])
        del self.rows[q][keep:]
        self.lens[q] = n

    def fork(self, src, dst):
        for a, b in zip(src, dst):
            self.rows[b] = list(self.rows[a])
            self.lens[b] = self.lens[a]
            for p in self.rows[a]:
                self.ref[p] += 1

    def truncate(self, seqs, lens):
        for q, n in zip(seqs, lens):
            if q >= 0:
                self._cut(q, min(n, self.lens[q]))

    def free(self, seqs):
        self.truncate(seqs, [0] * len(seqs))


def visible(n, branches, length, window=0, sinks=0):
    """see [n][length + n] and the slots' positions, from the tree itself."""
    L = (n - 1) // branches
    depth = np.zeros(n, int)
    chain = [[0] for _ in range(n)]
    for i in range(1, n):
        depth[i] = (i - 1) % L + 1
        chain[i] = [0] + list(range(i - depth[i] + 1, i + 1))
    pos = np.concatenate([np.arange(length), length + depth])
    see = np.zeros((n, length + n), bool)
    for i in range(n):
        see[i, :length] = True
        see[i, length + np.array(chain[i])] = True
        if window:
            see[i] &= (pos < sinks) | (pos > length + depth[i] - window)
    return see


def attend(q, k, v, see, scale):
    """o [n][Hq][D] and, per row, sum w |v| / sum w and the largest
    sum |q k| scale; q [n][Hq][D], k and v [T][H][D]."""
    n, Hq, D = q.shape
    g = Hq // k.shape[1]
    o, mag, big = np.zeros((n, Hq, D)), np.zeros((n, Hq, D)), np.zeros((n, Hq, 1))
    for h in range(Hq):
        z = q[:, h] @ k[:, h // g].T * scale
        z = np.where(see, z, -np.inf)
        w = np.exp(z - z.max(1, keepdims=True))
        w /= w.sum(1, keepdims=True)
        o[:, h] = w @ v[:, h // g]
        mag[:, h] = w @ np.abs(v[:, h // g])
        big[:, h, 0] = np.where(see, np.abs(q[:, h]) @ np.abs(k[:, h // g]).T * scale, 0).max(1)
    return o, mag, big
