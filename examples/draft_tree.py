"""Multi-draft decoding end to end on a small random model: the key/value cache
around the verification of draft trees.

Every step drafts K branches of L tokens for each sequence, runs the target
model once over the 1 + K * L nodes of the tree (their keys and values
appended to the 8-bit cache, their attention read from it), verifies the
branches against the target's logits, and keeps the accepted branch's tokens
in the cache.  Lengths, pages, accepted tokens and the next roots stay on the
GPU: a step copies nothing to the host.

With several samples a prompt, a prompt is put into the cache once and forked,
and the samples' attention reads what they share once.  With rotary positions
keys are rotated on their way into the cache, queries beside them.

The target is a two-layer transformer with random weights.  The draft model is
a table of logits per last token, fitted to nothing: it mixes the target's own
logits of the last token alone with noise, so that some drafts are accepted.

    python examples/draft_tree.py [--steps 12] [--branches 4] [--length 3] [--scheme WIS] [--samples 1] [--rotary]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2410_18234_gb300 import cache, mds  # noqa: E402


class Target:
    """A small decoder: positions as learned vectors, or rotary ones (a
    `cache.Rotary`), which its caller's attention applies."""

    def __init__(self, vocab=512, width=256, layers=2, q_heads=8, kv_heads=2, head_dim=64, positions=512, seed=0,
                 rotary=None):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def w(*shape):
            return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32) / math.sqrt(shape[0])

        self.rotary = rotary
        self.vocab, self.layers, self.q_heads, self.kv_heads, self.head_dim = vocab, layers, q_heads, kv_heads, head_dim
        self.embed, self.place = w(vocab, width) * math.sqrt(vocab), 0.3 * w(positions, width) * math.sqrt(positions)
        self.qkv = [w(width, (q_heads + 2 * kv_heads) * head_dim) for _ in range(layers)]
        self.out = [w(q_heads * head_dim, width) for _ in range(layers)]
        self.up, self.down = [w(width, 2 * width) for _ in range(layers)], [w(2 * width, width) for _ in range(layers)]
        self.head = 3.0 * w(width, vocab)

    def __call__(self, tokens, positions, attend):
        """Logits [B][n][V] of tokens [B][n] at positions [B][n]; attend(layer,
        q, k, v) takes [B][n][heads][head_dim] slices of one projection."""
        x = self.embed[tokens] if self.rotary else self.embed[tokens] + self.place[positions]
        H, G = self.q_heads, self.kv_heads
        for layer in range(self.layers):
            y = torch.nn.functional.layer_norm(x, x.shape[-1:])
            qkv = (y @ self.qkv[layer]).bfloat16().unflatten(-1, (H + 2 * G, self.head_dim))
            o = attend(layer, qkv[:, :, :H], qkv[:, :, H:H + G], qkv[:, :, H + G:])
            x = x + o.float().flatten(2) @ self.out[layer]
            y = torch.nn.functional.layer_norm(x, x.shape[-1:])
            x = x + torch.relu(y @ self.up[layer]) @ self.down[layer]
        return torch.nn.functional.layer_norm(x, x.shape[-1:]) @ self.head


def draft_table(target, noise=0.6, seed=1):
    """Draft logits [V][V] by last token: the target's on that token alone, and noise."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    V = target.vocab
    alone = lambda layer, q, k, v: v.repeat_interleave(target.q_heads // target.kv_heads, dim=2)  # noqa: E731
    tokens = torch.arange(V, device="cuda")[:, None]
    logits = target(tokens, torch.full_like(tokens, 8), alone)[:, 0]
    return logits + noise * torch.randn(V, V, generator=g, device="cuda")


class Decoder:
    """Sequences 0..B-1 of a cache, decoded by draft trees; `samples` of each
    prompt, next to one another.  least_saved: of `cache.Cache.attend_shared`."""

    def __init__(self, target, prompts, branches=4, length=3, steps=12, scheme="WIS", temperature=1.0, page_tokens=16,
                 samples=1, least_saved=None):
        B, T = prompts.shape[0] * samples, prompts.shape[1]
        self.samples, self.least_saved = samples, least_saved
        self.target, self.B, self.K, self.L, self.scheme = target, B, branches, length, scheme
        self.temperature = temperature
        n, per = 1 + branches * length, page_tokens
        most = T + steps * (length + 1) + n
        self.cache = cache.Cache(target.layers, B * (-(-most // per) + 1), target.kv_heads, target.head_dim, B,
                                 -(-most // per) + 1, page_tokens=per)
        self.verifier = mds.Verifier(B, branches, length, target.vocab, dtype="f32")
        self.table = draft_table(target)
        self.seqs = torch.arange(B, device="cuda", dtype=torch.int32)
        self.temps = torch.full((B, 1 + branches), float(temperature), device="cuda")
        # depth of each node, and the node of each (branch, depth)
        self.depth = torch.tensor([0] + [d + 1 for _ in range(branches) for d in range(length)], device="cuda")
        self.node = torch.tensor([[0] + [1 + k * length + d for d in range(length)] for k in range(branches)], device="cuda")
        # the prompt but its last token, which is the first root
        self.root = prompts[:, -1].repeat_interleave(samples)
        if T > 1:
            first = self.seqs[::samples].contiguous()
            self._forward(prompts[:, :-1], torch.arange(T - 1, device="cuda").expand(len(first), -1), 1, first)
            self.cache.commit(first, torch.full_like(first, T - 2), length=T - 2)
            if samples > 1:
                others = self.seqs.view(-1, samples)[:, 1:].contiguous().flatten()
                self.cache.fork(first.repeat_interleave(samples - 1), others)

    def _forward(self, tokens, positions, branches, seqs):
        c = self.cache
        c.reserve(seqs, tokens.shape[1])

        def attend(layer, q, k, v):
            if self.target.rotary:
                q = c.append_rotated(layer, seqs, k, v, self.target.rotary, branches=branches, q=q)
            else:
                c.append(layer, seqs, k, v)
            if self.samples > 1 and seqs is self.seqs:
                return c.attend_shared(layer, seqs, q, self.samples, branches=branches, least_saved=self.least_saved)
            return c.attend(layer, seqs, q, branches=branches)

        return self.target(tokens, positions, attend)

    def step(self, seed):
        """One draft tree for every sequence: emitted tokens [B][L + 1] (-1
        behind the last) and accepted lengths [B]."""
        B, K, L, V = self.B, self.K, self.L, self.target.vocab
        g = torch.Generator(device="cuda").manual_seed(seed)
        # K branches from the draft table, by the Gumbel-max rule
        last = self.root[:, None].expand(B, K)
        drafts, rows = [], []
        for _ in range(L):
            z = self.table[last]                                                # [B][K][V]
            u = torch.rand(B, K, V, generator=g, device="cuda").clamp_(min=1e-12)
            last = (z / self.temperature - torch.log(-torch.log(u))).argmax(-1)
            rows.append(z)
            drafts.append(last)
        tokens = torch.stack(drafts, 2)                                         # [B][K][L]
        tree = torch.cat([self.root[:, None], tokens.flatten(1)], 1)            # [B][1 + K L]
        logits = self._forward(tree, self.cache.lens[:B, None] + self.depth, K, self.seqs)
        target = logits[:, self.node].contiguous()                              # [B][K][L + 1][V]
        draft = torch.stack(rows, 2).transpose(0, 1).contiguous()               # [K][B][L][V]
        tokens = tokens.int()
        out, accept, _ = self.verifier.verify(target, [draft[k] for k in range(K)], [0] * K, tokens, self.temps,
                                              self.scheme, seed)
        self.cache.commit(self.seqs, accept, branches=K, length=L, draft_tokens=tokens, out_tokens=out)
        self.root = out.gather(1, accept[:, None].long())[:, 0].long()
        return out, accept, target

    def status(self):
        return self.cache.status()[0] | self.verifier.status()[0]


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=12)
    ap.add_argument("--branches", type=int, default=4)
    ap.add_argument("--length", type=int, default=3)
    ap.add_argument("--scheme", default="WIS")
    ap.add_argument("--samples", type=int, default=1)
    ap.add_argument("--rotary", action="store_true")
    args = ap.parse_args()
    target = Target(rotary=cache.Rotary(64) if args.rotary else None)
    prompts = torch.randint(target.vocab, (8, 40), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    d = Decoder(target, prompts, args.branches, args.length, args.steps, args.scheme, samples=args.samples)
    emitted = 0
    for i in range(args.steps):
        out, accept, _ = d.step(i)
        emitted += int((accept + 1).sum())
    print(f"{args.steps} steps of {args.branches} branches x {args.length}: {emitted / args.steps / d.B:.2f} tokens a step "
          f"and sequence, lengths {d.cache.lens[:d.B].tolist()}, status {d.status()}")


if __name__ == "__main__":
    main()
