#!/usr/bin/env python
"""Speculative decoding with a small target model on the library: drafts from the histories, a target forward over
the drafted chunks on the paged cache, greedy verification, commit of tokens and cache.

    python examples/target_forward.py [--steps 40] [--batch 8] [--tree]

The model (random weights) is a plain decoder: root-mean-square norms, attention with rotary positions and shared
key/value heads, a gated feed-forward, in bfloat16.  Its matrix products are torch's; rotary positions, cache and
attention are hvd_rope_append, hvd_attn_paged and hvd_kv_commit.  One decoding step:

    hvd_lookup_score_select    a draft per request (or, with --tree, a tree around it)
    forward                    row 0: the last committed token, rows 1..: the draft
    hvd_verify_commit[_tree]   accepted length, tokens appended to the histories
    hvd_kv_commit              the accepted tokens' cache rows made consecutive, lengths raised
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import numpy as np

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


class TargetModel:
    def __init__(self, *, vocab=256, layers=2, width=256, n_q_heads=8, n_kv_heads=2, head_dim=64, seed=0, device="cuda"):
        import torch
        self.torch, self.vocab, self.layers, self.dev = torch, vocab, layers, device
        self.hq, self.hkv, self.d = n_q_heads, n_kv_heads, head_dim
        g = torch.Generator(device=device).manual_seed(seed)
        w = lambda *s: (torch.randn(*s, generator=g, device=device) / s[-1] ** 0.5).to(torch.bfloat16)
        heads = n_q_heads + 2 * n_kv_heads
        self.embed = w(vocab, width) * width ** 0.5
        self.qkv = [w(heads * head_dim, width) for _ in range(layers)]
        self.out = [w(width, n_q_heads * head_dim) for _ in range(layers)]
        self.up = [w(4 * width, width) for _ in range(layers)]
        self.down = [w(width, 2 * width) for _ in range(layers)]
        self.head = w(vocab, width) * 4

    def norm(self, x):
        return (x.float() * self.torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)

    def forward(self, cache, tokens, **chunk):
        """Logits [rows, vocab] of the chunk's rows; keys and values of the new tokens go into the cache."""
        torch, rows = self.torch, tokens.shape[0]
        x = self.embed[tokens.long()]
        q_out = torch.empty(rows, self.hq, self.d, dtype=torch.bfloat16, device=self.dev)
        attn = torch.zeros_like(q_out)
        for i in range(self.layers):
            qkv = (self.norm(x) @ self.qkv[i].T).view(rows, -1, self.d)
            q, k, v = qkv.split([self.hq, self.hkv, self.hkv], dim=1)
            q_out.zero_()                      # rows that are no new token keep finite values
            cache.append(i, q, k, v, q_out, **chunk)
            cache.attend(i, q_out, attn, **chunk)
            x = x + attn.reshape(rows, -1) @ self.out[i].T
            gate, up = (self.norm(x) @ self.up[i].T).chunk(2, -1)
            x = x + (torch.nn.functional.silu(gate) * up) @ self.down[i].T
        return self.norm(x) @ self.head.T


class Decoder:
    """A batch of requests decoded together.  prompts: token lists, each of two tokens or more."""

    def __init__(self, model, prompts, *, k_cap=8, new_tokens=64, tree=False, page_size=16, seed=0):
        import torch
        import paper_2606_01019_b200 as H
        from paper_2606_01019_b200.runner import DeviceBatch, PagedCache
        self.torch, self.model, self.tree, self.k_cap = torch, model, tree, k_cap
        B, lens = len(prompts), np.array([len(p) for p in prompts], np.int64)
        cap = lens + new_tokens + 2 * (k_cap + 1)
        off = np.concatenate([[0], np.cumsum(cap)])[:-1]
        hist = np.zeros(int(cap.sum()), np.int32)
        for p, o in zip(prompts, off):
            hist[o:o + len(p)] = p
        self.ctx = H.Context(max_batch=B, k_cap=k_cap, max_hist_len=int(cap.max()), max_vocab=model.vocab,
                             max_rows=int(max(B * (k_cap + 1), lens.sum())))
        rng = np.random.default_rng(seed)
        self.rng = rng
        self.ctx.hvd_set_predictor(rng.normal(0, 0.1, (32, 8)), np.zeros(32), rng.normal(0, 0.1, 32), 1.0, 0.0)
        state = np.zeros(B, H.STATE_DTYPE)
        self.batch = DeviceBatch(self.ctx, hist=hist, hist_off=off, hist_cap=cap, hist_len=lens, K=np.full(B, k_cap), prompt_len=lens,
                                 state=state, model_draft=np.zeros((B, k_cap), np.int32), model_len=np.zeros(B, np.int32),
                                 row_off=np.arange(B + 1) * (k_cap + 1), V=model.vocab, dtype="bf16", uniform_rows=True)
        # a request's chunk may pass its last history slot: the cache has room for it
        self.cache = PagedCache(self.ctx, B=B, n_layers=model.layers, max_len=int(cap.max()) + k_cap + 1, n_q_heads=model.hq,
                                n_kv_heads=model.hkv, head_dim=model.d, page_size=page_size)
        # the prompts but their last tokens, which are the first chunks' roots
        rows = torch.as_tensor(np.concatenate([p[:-1] for p in prompts]).astype(np.int32), device=model.dev)
        row_off = torch.as_tensor(np.concatenate([[0], np.cumsum(lens - 1)]), dtype=torch.int64, device=model.dev)
        model.forward(self.cache, rows, row_off=row_off)
        self.cache.commit(torch.as_tensor(lens - 1, dtype=torch.int32, device=model.dev))

    def chunk_tokens(self):
        """[B * (k_cap + 1)] row 0 the last committed token, row i draft token i - 1."""
        torch, b = self.torch, self.batch
        root = b.hist[b.hist_off + b.hist_len - 1]
        return torch.cat([root[:, None], b.sel_draft.clamp(min=0)], 1).reshape(-1)

    def grow_tree(self):
        """A tree around the draft: every second node continues the draft's chain, the others are random siblings."""
        torch, b = self.torch, self.batch
        draft, m = b.sel_draft.cpu().numpy(), b.sel_len.cpu().numpy()
        tok, par, n = np.full_like(draft, -1), np.full_like(draft, -1), np.zeros_like(m)
        for i in range(len(m)):
            at, node = -1, 0
            for t in draft[i, :m[i]]:
                if node + 2 > self.k_cap:
                    break
                tok[i, node], par[i, node] = self.rng.integers(0, self.model.vocab), at
                tok[i, node + 1], par[i, node + 1] = t, at
                at, node = node + 1, node + 2
            n[i] = node
        up = lambda x: torch.as_tensor(x, dtype=torch.int32, device=self.model.dev)
        b.sel_draft, b.sel_len = up(tok), up(n)
        return up(par)

    def step(self):
        b = self.batch
        b.lookup_score_select()
        parent = self.grow_tree() if self.tree else None
        chunk = dict(k_uniform=self.k_cap, sel_len=b.sel_len, parent=parent)
        logits = self.model.forward(self.cache, self.chunk_tokens(), **chunk)
        if self.tree:
            self.ctx.hvd_verify_commit_tree(b.B, logits, b.dtype, b.V, None, self.k_cap, b.total_rows, b.sel_draft, b.sel_len, parent,
                                            b.select, b.hist, b.hist_off, b.hist_cap, b.hist_len, b.state, b.accepted, b.committed,
                                            b.n_commit, None, b.status)
            b.n_max = min(b.cap_max, b.n_max + self.k_cap + 1)
            self.cache.commit(b.n_commit, sel_draft=b.sel_draft, sel_len=b.sel_len, parent=parent, accepted=b.accepted,
                              committed=b.committed)
        else:
            b.verify_commit(logits, target_tok=False)
            self.cache.commit(b.n_commit)

    def histories(self):
        h, o, n = (x.cpu().numpy() for x in (self.batch.hist, self.batch.hist_off, self.batch.hist_len))
        return [h[a:a + m].copy() for a, m in zip(o, n)]

    def close(self):
        self.ctx.close()


def prompts(batch, vocab, seed=0):
    rng = np.random.default_rng(seed)
    return [rng.integers(0, vocab, int(n)) for n in rng.integers(2, 200, batch)]


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--batch", type=int, default=8)
    ap.add_argument("--tree", action="store_true")
    args = ap.parse_args()
    import torch
    model = TargetModel()
    dec = Decoder(model, prompts(args.batch, model.vocab), new_tokens=args.steps * 9, tree=args.tree)
    before = sum(len(h) for h in dec.histories())
    dec.step()
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for _ in range(args.steps - 1):
        dec.step()
    torch.cuda.synchronize()
    t = time.perf_counter() - t0
    made = sum(len(h) for h in dec.histories()) - before
    print(f"{made} tokens for {args.batch} requests in {args.steps} steps ({made / args.batch / args.steps:.2f} a request and step), "
          f"{t / max(1, args.steps - 1) * 1e3:.2f} ms a step")
    dec.close()


if __name__ == "__main__":
    main()
