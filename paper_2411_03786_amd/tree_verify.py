"""Greedy decoding of several sequences at once whose drafts are verified as trees, on the framework's operators.

  python -m paper_2411_03786_amd.tree_verify [--batch 4] [--layers 4] [--heads 32] [--kv-heads 8] [--head-dim 128]
         [--vocab 32000] [--prompt 512] [--new 64] [--k 6] [--w 8] [--cycle 40] [--cache bf16|fp8|f32]

Every step takes up to k rows of w tokens that followed earlier occurrences of a sequence's last tokens (the paper's context
N-grams, Section 4.2), merges the rows that begin alike into a tree behind the last token, and runs the trees of all sequences
through the model in one pass: `rotary` on the queries, `KVPages.write` of keys (rotated on the way) and values, `tree_attention`
over each sequence's pages, `token_logprobs` for the greedy token of every node and the log probabilities of its children.  The
path that the greedy tokens follow is kept: its keys and values are read from where the tree left them and written behind the
context.  Output tokens are those of plain greedy decoding (one token a step), which runs beside it for comparison, where no two
tokens are as likely but for the rounding of a 16-bit sum.  The projections are torch matrix products; weights and prompts are synthetic and seeded; one GPU.
"""
from __future__ import annotations

import argparse
import time

import numpy as np
import torch

import paper_2411_03786_amd as ngg


def context_rows(tokens, k, w, q_max=3):
    """Up to k rows of up to w tokens that followed earlier occurrences of the last q tokens, longest q and latest place first."""
    rows, text = [], np.asarray(tokens)
    for q in range(min(q_max, len(tokens) - 1), 0, -1):
        same = np.ones(len(tokens) - q, bool)
        for j in range(q):
            same &= text[j:j + len(same)] == text[len(same) + j]
        for at in np.flatnonzero(same)[::-1].tolist():
            row = tokens[at + q:at + q + w]
            if row not in rows:
                rows.append(row)
            if len(rows) == k:
                return rows
    return rows


def draft_tree(root, rows):
    """The rows behind the root token, shared beginnings once: tokens and parents (-1: the root), parents first."""
    tokens, parents, children = [root], [-1], [{}]
    for row in rows:
        at = 0
        for tok in row:
            if tok not in children[at]:
                children[at][tok] = len(tokens)
                tokens.append(tok)
                parents.append(at)
                children.append({})
            at = children[at][tok]
    return tokens, parents, children


class TreeDecoder:
    """A decoder-only transformer (RMSNorm, grouped heads, rotary positions, SwiGLU) with random weights and a paged cache for
    `batch` sequences of up to max_tokens tokens.  cycle: with a number, the unembedding prefers the tokens that follow each other
    in cycles of that many, so that what the model writes repeats itself as text does; with 0 it is random too."""

    def __init__(self, batch, layers, heads, kv_heads, head_dim, vocab, max_tokens, cache="bf16", page=64, d_ffn=None, seed=0, cycle=0):
        self.batch, self.heads, self.kv_heads, self.hd, self.page = batch, heads, kv_heads, head_dim, page
        self.dtype = torch.float32 if cache == "f32" else torch.bfloat16
        d, d_ffn = heads * head_dim, d_ffn or 4 * heads * head_dim
        g = torch.Generator(device="cuda").manual_seed(seed)

        def weight(n_in, n_out):
            return (torch.randn(n_in, n_out, generator=g, device="cuda") * n_in ** -0.5).to(self.dtype)

        self.embed = torch.randn(vocab, d, generator=g, device="cuda").to(self.dtype)
        self.unembed = weight(d, vocab)
        if cycle:
            v = torch.arange(vocab, device="cuda")
            before = torch.where(v % cycle > 0, v - 1, (v + cycle - 1).clamp(max=vocab - 1))
            self.unembed = (self.embed[before].T.float() * d ** -0.5).to(self.dtype)
        self.layers = [dict(qkv=weight(d, (heads + 2 * kv_heads) * head_dim), proj=weight(d, d), gate=weight(d, d_ffn), up=weight(d, d_ffn),
                            down=weight(d_ffn, d)) for _ in range(layers)]
        per = -(-max_tokens // page)
        self.rope = ngg.Rope(head_dim, per * page)                                # whatever the pages hold
        self.kv = [ngg.KVPages(batch * per, page, kv_heads, head_dim, cache) for _ in range(layers)]
        # a sequence's pages lie scattered over the pool, as they do after some serving
        self.pages = torch.randperm(batch * per, generator=torch.Generator().manual_seed(seed)).view(batch, per).int().cuda()
        self.lens = torch.zeros(batch, dtype=torch.int32, device="cuda")          # cached positions
        self.cached = [0] * batch                                                 # the same on the host

    @staticmethod
    def norm(x):
        x = x.float()
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)

    def slots(self, places):
        """Slots of positions [batch, n]; -1 stays."""
        at = torch.gather(self.pages, 1, (places.clamp(min=0) // self.page).long()) * self.page + places.clamp(min=0) % self.page
        return torch.where(places < 0, -1, at).int().flatten()

    def forward(self, tokens, depth, mask=None, tree_lens=None, logits=True):
        """Logits [batch * tree, vocab] of the trees' tokens [batch, tree] behind the cached positions, or None without `logits`; their
        keys and values are left at the positions behind those, in the trees' order."""
        B, T = tokens.shape
        H, Hkv, hd = self.heads, self.kv_heads, self.hd
        place = self.lens[:, None] + torch.arange(T, dtype=torch.int32, device="cuda")
        if tree_lens is not None:
            place = torch.where(torch.arange(T, device="cuda") < tree_lens[:, None], place, -1)
        longest = max(self.cached) + T
        if longest > self.pages.shape[1] * self.page:
            raise ValueError(f"{longest} positions in pages for {self.pages.shape[1] * self.page}")
        pages = self.pages[:, :-(-longest // self.page)]                # the call is planned for these
        slots, pos = self.slots(place), (self.lens[:, None] + depth).int().flatten()
        x = self.embed[tokens.flatten().long()]
        for w, kv in zip(self.layers, self.kv):
            q, k, v = (self.norm(x).to(self.dtype) @ w["qkv"]).view(B * T, H + 2 * Hkv, hd).split((H, Hkv, Hkv), 1)
            ngg.rotary(self.rope, pos, q, out=q)
            kv.write(k, v, slots, rope=self.rope, positions=pos)
            a = ngg.tree_attention(q.unflatten(0, (B, T)), kv, pages, self.lens, mask=mask, tree_lens=tree_lens)
            x = x + a.reshape(B * T, H * hd) @ w["proj"]
            y = self.norm(x).to(self.dtype)
            x = x + (torch.nn.functional.silu(y @ w["gate"]) * (y @ w["up"])) @ w["down"]
        return self.norm(x).to(self.dtype) @ self.unembed if logits else None

    def prefill(self, prompts, piece=512):
        """Caches all tokens of the prompts [batch, n] but the last."""
        for at in range(0, prompts.shape[1] - 1, piece):
            part = prompts[:, at:min(at + piece, prompts.shape[1] - 1)]
            self.forward(part, torch.arange(part.shape[1], device="cuda"), logits=False)
            self.lens += part.shape[1]
            self.cached = [n + part.shape[1] for n in self.cached]

    def keep(self, paths):
        """Keeps of every sequence's tree the nodes of its path (root first, rising): they move behind the context."""
        n = max(len(p) for p in paths)
        src = torch.tensor([p + [-1] * (n - len(p)) for p in paths], dtype=torch.int32, device="cuda")
        there = src >= 0
        to = torch.where(there, self.lens[:, None] + torch.arange(n, dtype=torch.int32, device="cuda"), -1)
        src, to = self.slots(torch.where(there, self.lens[:, None] + src, -1)), self.slots(to)
        for kv in self.kv:
            kv.write(*kv.read(src), to)
        self.lens += there.sum(1, dtype=torch.int32)
        self.cached = [c + len(p) for c, p in zip(self.cached, paths)]

    def step(self, last, rows):
        """One verify step: last tokens, draft rows of every sequence -> (new tokens, their log probabilities) per sequence."""
        trees = [draft_tree(t, r) for t, r in zip(last, rows)]
        T = max(len(t[0]) for t in trees)
        wide = max(1, max(len(c) for t in trees for c in t[2]))
        tokens, targets = np.zeros((self.batch, T), np.int32), np.full((self.batch, T, wide), -1, np.int32)
        mask, depth = np.zeros((self.batch, T, -(-T // 64)), np.int64), np.zeros((self.batch, T), np.int32)
        for b, (toks, parents, children) in enumerate(trees):
            n = len(toks)
            m, depth[b, :n] = ngg.tree_mask(parents)
            tokens[b, :n], mask[b, :n, :m.shape[1]] = toks, m
            for i, c in enumerate(children):
                targets[b, i, :len(c)] = list(c)
        dev = [torch.from_numpy(a).cuda() for a in (tokens, depth, mask, targets)]
        lens = torch.tensor([len(t[0]) for t in trees], dtype=torch.int32, device="cuda")
        logits = self.forward(dev[0], dev[1], dev[2], lens)
        score = ngg.token_logprobs(logits, dev[3].flatten(0, 1), top_n=1)
        greedy, best = score.top_ids.view(self.batch, T).tolist(), score.top_logprobs.view(self.batch, T).tolist()
        drafted = score.logprobs.view(self.batch, T, wide).tolist()
        out, paths = [], []
        for b, (toks, parents, children) in enumerate(trees):
            path, new, logp = [0], [], []
            while True:
                at = path[-1]
                new.append(greedy[b][at])
                # an accepted child's own log probability is the greedy token's
                child = children[at].get(new[-1])
                logp.append(best[b][at] if child is None else drafted[b][at][list(children[at]).index(new[-1])])
                if child is None:
                    break
                path.append(child)
            paths.append(path)
            out.append((new, logp))
        self.keep(paths)
        return out

    def decode(self, prompts, n_new, draft):
        """n_new greedy tokens behind each prompt (lists of equal length).  draft(sequence index, tokens) -> rows.  Returns the
        sequences' new tokens, their log probabilities, and the steps taken."""
        self.lens.zero_()
        self.cached = [0] * self.batch
        self.prefill(torch.tensor(prompts, dtype=torch.int32, device="cuda"))
        seqs, logps, steps = [list(p) for p in prompts], [[] for _ in prompts], 0
        while min(map(len, logps)) < n_new:
            rows = [draft(b, s) if len(logps[b]) < n_new else [] for b, s in enumerate(seqs)]
            for b, (new, logp) in enumerate(self.step([s[-1] for s in seqs], rows)):
                seqs[b] += new
                logps[b] += logp
            steps += 1
        n = len(prompts[0])
        return [s[n:n + n_new] for s in seqs], [lp[:n_new] for lp in logps], steps


def main():
    ap = argparse.ArgumentParser()
    for name, value in dict(batch=4, layers=4, heads=32, kv_heads=8, head_dim=128, vocab=32000, prompt=512, new=64, k=6, w=8, cycle=40, seed=0).items():
        ap.add_argument("--" + name.replace("_", "-"), type=int, default=value)
    ap.add_argument("--cache", default="bf16", choices=("f32", "bf16", "fp8"))
    args = ap.parse_args()
    # a finished sequence still takes a token a step until the last one is done
    dec = TreeDecoder(args.batch, args.layers, args.heads, args.kv_heads, args.head_dim, args.vocab,
                      args.prompt + 2 * args.new + args.k * args.w + args.w + 2, args.cache, seed=args.seed, cycle=args.cycle)
    rng = np.random.default_rng(args.seed)
    prompts = rng.integers(0, args.vocab, (args.batch, args.prompt)).tolist()
    runs = dict(plain=lambda b, s: [], trees=lambda b, s: context_rows(s, args.k, args.w))
    results = {}
    for name, draft in runs.items():
        dec.decode(prompts, 4, draft)                                   # warm up
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        results[name] = tokens, logps, steps = dec.decode(prompts, args.new, draft)
        torch.cuda.synchronize()
        dt = time.perf_counter() - t0
        print(f"{name}: {args.batch} sequences, {args.new} tokens each, {steps} steps, {dt * 1e3:.1f} ms with the prompts, "
              f"mean log probability {np.mean(logps):.4f}")
    same = sum(a == b for a, b in zip(results["plain"][0], results["trees"][0]))
    print(f"{same} of {args.batch} sequences alike")


if __name__ == "__main__":
    main()
