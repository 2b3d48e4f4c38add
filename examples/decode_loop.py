"""Speculative decoding around retrace_round_sampled, on a toy model of random weights.

One round of the loop, for a batch of sequences on one stream:

  drafter   its block (the anchor and K positions to propose, whose inputs the round
            before has conditioned) goes into its paged cache (retrace_kv_append),
            attends over it both ways within the block (retrace_attend, causal off, a
            sliding window with sinks), and its logits become the draft tokens
            (retrace_sample);
  target    the anchor and the drafts go into the target's cache and attend causally;
  round     retrace_round_sampled verifies the drafts and conditions the drafter's next
            inputs on the rejected ones;
  lengths   grow by the committed tokens; what was rejected is overwritten by the next
            append.

Nothing is read back until the end.  With top_k = 1 the tokens are those that the target
alone gives, one after another.

    python examples/decode_loop.py [--tokens 64] [--batch 4] [--dtype bf16|f32] [--top-k 1]
"""

from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_29748_gb300 import binding as rt  # noqa: E402

PAGE = 16


def rope_table(positions, rot, device="cuda"):
    a = torch.arange(0, rot, 2, dtype=torch.float64, device=device) / rot
    t = torch.arange(positions, dtype=torch.float64, device=device)[:, None] * 10000.0**-a
    return torch.stack([t.cos(), t.sin()], -1).float().contiguous()


class Layer:
    """One attention layer and a head, with a paged cache for a batch."""

    def __init__(self, B, V, d, q_heads, kv_heads, D, positions, dtype, gen, window=0, sinks=0, causal=True):
        w = lambda o, i: (torch.randn((o, i), generator=gen, device="cuda") / i**0.5).to(dtype)  # noqa: E731
        self.shape = (q_heads, kv_heads, D)
        self.qkv, self.o, self.head = w((q_heads + 2 * kv_heads) * D, d), w(d, q_heads * D), w(V, d)
        pages = -(-positions // PAGE)
        # each sequence's pages, in any order
        table = torch.randperm(B * pages, generator=gen, device="cuda").to(torch.int32).view(B, pages)
        k, v = (torch.empty((B * pages, PAGE, kv_heads, D), dtype=dtype, device="cuda") for _ in range(2))
        self.cache = rt.KvCache(k, v, table)
        self.ws = rt.AttendWorkspace(q_heads, kv_heads, D, dtype)
        self.rope = rope_table(positions, D)
        self.mask = {"window": window, "sinks": sinks, "causal": causal}

    def _project(self, x):
        q_heads, kv_heads, D = self.shape
        y = (x @ self.qkv.T).view(-1, q_heads + 2 * kv_heads, D)
        return y.split([q_heads, kv_heads, kv_heads], 1)

    def append(self, x, length):
        """The keys and values of x [B, n, d] at positions length, length + 1, ..."""
        _, k, v = self._project(x)
        rt.retrace_kv_append(None, k, v, self.cache, length, self.rope)

    def states(self, x, length):
        """The states of x [B, n, d], whose keys and values enter the cache."""
        q, k, v = self._project(x)
        turned = torch.empty_like(q, memory_format=torch.contiguous_format)
        rt.retrace_kv_append(q, k, v, self.cache, length, self.rope, turned)
        out = torch.empty_like(turned)
        rt.retrace_attend(turned, self.cache, length, out, self.ws, **self.mask)
        return x + (out.view(*x.shape[:2], -1) @ self.o.T)


class Decoder:
    """A target, a drafter and the state of a batch of sequences."""

    def __init__(self, B=4, K=8, V=1024, d=256, dtype=torch.bfloat16, positions=512, seed=0, temperature=1.0, top_k=1, top_p=1.0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.B, self.K, self.V, self.d, self.dtype, self.gen = B, K, V, d, dtype, gen
        self.setting = (float(temperature), int(top_k), float(top_p))
        self.embed = torch.randn((V, d), generator=gen, device="cuda").to(dtype)
        self.target = Layer(B, V, d, 4, 2, 64, positions, dtype, gen)
        # the drafter is the target seen through a window, so that it is often right
        self.drafter = Layer(B, V, d, 4, 2, 64, positions, dtype, gen, window=64, sinks=4, causal=False)
        self.drafter.qkv, self.drafter.o, self.drafter.head = self.target.qkv, self.target.o, self.target.head
        w = lambda i: (torch.randn((d, i), generator=gen, device="cuda") * 0.02).to(dtype)  # noqa: E731
        self.weights = (w(2 * d), w(d), w(2 * d))
        self.ws = rt.Workspace(B, K, V, d, dtype)
        self.mask_input = (torch.randn((d,), generator=gen, device="cuda") * 0.02).to(dtype)
        full = lambda x, t: torch.full((B,), x, dtype=t, device="cuda")  # noqa: E731
        self.temperature, self.top_k, self.top_p = (full(x, t) for x, t in zip(self.setting, (torch.float32, torch.int32, torch.float32)))
        # state: the anchor, tokens before it, the drafter's next inputs, tokens not in its cache yet
        self.anchor = torch.randint(0, V, (B,), generator=gen, device="cuda")
        self.length = torch.zeros(B, dtype=torch.int32, device="cuda")
        self.inputs = self.mask_input.expand(B, K, d).contiguous()
        self.fresh, self.fresh_at = None, None

    def round(self):
        """One round; returns the committed tokens [B, K + 1] (-1 after the last) and their number."""
        B, K, V, d = self.B, self.K, self.V, self.d
        anchor = self.embed[self.anchor][:, None]
        if self.fresh is not None:  # the tokens of the round before, over the drafts it left
            self.drafter.append(self.embed[self.fresh], self.fresh_at)
        h = self.drafter.states(torch.cat([anchor, self.inputs], 1), self.length)
        draft_states = h[:, 1:].contiguous()
        draft_logits = draft_states @ self.drafter.head.T
        draft = torch.empty((B, K), dtype=torch.int32, device="cuda")
        rt.retrace_sample(draft_logits, torch.rand((B, K), generator=self.gen, device="cuda"), draft, temperature=self.temperature,
                          top_k=self.top_k, top_p=self.top_p)

        h = self.target.states(torch.cat([anchor, self.embed[draft.long()]], 1), self.length)
        logits = h @ self.target.head.T
        out = rt.RoundBuffers(B, K, d, self.dtype)
        rt.retrace_round_sampled(logits, draft_logits, draft, torch.rand((B, K + 1), generator=self.gen, device="cuda"), *self.setting,
                                 draft_states, h[:, 1:].contiguous(), self.mask_input, *self.weights, 1.0, out.accept_len,
                                 out.committed, out.bonus, out.e_out, self.ws, n_out=out.n)
        count = out.accept_len + 1
        # the drafter has the anchor; it lacks the committed tokens but the last, which is the next anchor
        self.fresh, self.fresh_at = out.committed.clamp(min=0).long(), self.length + 1
        self.anchor, self.length, self.inputs = out.bonus.long(), self.length + count, out.e_out
        return out.committed, count


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--batch", type=int, default=4)
    ap.add_argument("--dtype", choices=["bf16", "f32"], default="bf16")
    ap.add_argument("--top-k", type=int, default=1)
    args = ap.parse_args()
    dec = Decoder(B=args.batch, dtype=torch.bfloat16 if args.dtype == "bf16" else torch.float32, top_k=args.top_k,
                  positions=2 * args.tokens + 64)
    rounds, total = [], torch.zeros(args.batch, dtype=torch.int64, device="cuda")
    t0 = time.perf_counter()
    while len(rounds) < args.tokens and (not rounds or int(total.min()) < args.tokens):
        rounds.append(dec.round()[0])
        total += (rounds[-1] >= 0).sum(1)
    torch.cuda.synchronize()
    if dec.ws.check() or dec.target.ws.check() or dec.drafter.ws.check():
        raise RuntimeError("device status flag raised")
    print(f"{len(rounds)} rounds, {float(total.float().mean()) / len(rounds):.2f} tokens a round and sequence, "
          f"{(time.perf_counter() - t0) / len(rounds) * 1e6:.0f} us a round")
    for b in range(args.batch):
        print([int(t) for r in rounds for t in r[b] if t >= 0][: args.tokens])


if __name__ == "__main__":
    main()
