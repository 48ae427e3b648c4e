"""Answers over a long cache that do not read, or do not keep, all of it: one attention layer.

    python examples/long_answers.py

1. Every sequence's context lies in pages (ba_paged_append); the question attends to all of it (ba_paged_attention), and its log-sum-exps
   say how much attention every cached key got from it (ba_paged_key_weights).
2. ``keep``: the heaviest keys of every head, the first and the last ones among them, move to fewer pages (ba_paged_evict), and the answers go
   on from there: a token's row is the sequence's new length, its rotation its place in the text.
3. ``pages``: the pages' keys are bounded in 8 bits (ba_page_bounds); a step takes its own key in, selects the pages that promise its queries the
   largest scores (ba_page_select) and attends to those (ba_paged_attention_selected).  Captured once and replayed.

Activations are random numbers: what stands around attention in a model is left out.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2409_15355_amd import binding as ba  # noqa: E402


class LongAnswers:
    def __init__(self, heads, n_seqs, context, question, steps, page_rows=16, keep=0, pages=0, seed=0):
        """keep: tokens that stay of a context (0: all); pages: pages that a step reads (0: all)."""
        self.heads, self.n, self.question, self.pages = heads, n_seqs, question, pages
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        hq, hkv, d = heads.n_q_heads, heads.n_kv_heads, heads.head_dim
        prompt = context + question
        self.ws = torch.empty(256, dtype=torch.uint8, device="cuda")
        self.prompt_len, self.kept = prompt, min(keep or prompt, prompt)
        self.max_len = self.kept + steps
        # the prompt
        cache, lens = self.new_cache(prompt if keep else self.max_len, page_rows), self.ints([prompt] * n_seqs)
        k, v, q = self.randn(n_seqs * prompt, hkv), self.randn(n_seqs * prompt, hkv), self.randn(n_seqs * question, hq, 2.0)
        at, seq = torch.arange(prompt, device="cuda").repeat(n_seqs).int(), torch.arange(n_seqs, device="cuda").repeat_interleave(prompt).int()
        ba.ba_paged_append(heads, None, cache, None, k, v, None, at, seq)
        self.o_question, lse = torch.empty_like(q), torch.empty((n_seqs * question, hq), device="cuda")
        ba.ba_paged_attention(heads, cache, q, self.o_question, lse, lens, prompt, None, None, question,
                              self.scratch(ba.ba_paged_attention_workspace_bytes(heads, n_seqs, question, prompt)))
        self.weights = torch.empty((n_seqs, hkv, prompt), device="cuda")
        ba.ba_paged_key_weights(heads, cache, q, lse, None, self.weights, 0.0, lens, prompt, None, None, question,
                                self.scratch(ba.ba_paged_key_weights_workspace_bytes(heads, n_seqs, question, prompt)))
        self.cache, self.len, self.position = cache, lens, lens.clone()
        if keep:
            self.cache = self.new_cache(self.max_len, page_rows)
            self.kept_tokens = torch.empty((n_seqs, hkv, keep), dtype=torch.int32, device="cuda")
            self.len = torch.empty_like(lens)
            ba.ba_paged_evict(heads, cache, self.cache, self.weights, lens, prompt, keep, min(4, keep // 4), keep // 4, self.kept_tokens, None, self.len,
                              self.scratch(ba.ba_paged_evict_workspace_bytes(heads, n_seqs, prompt, keep)))
        if pages:
            n_pages = self.cache.k_pages.shape[0]
            self.bounds = ba.PageBounds(torch.empty((n_pages, hkv, 2, d), dtype=torch.int8, device="cuda"),
                                        torch.empty((n_pages, hkv), dtype=torch.int8, device="cuda"))
            ba.ba_page_bounds(heads, self.cache, self.bounds, None, self.len, self.max_len)
            self.selected = torch.empty((n_seqs, hkv, pages), dtype=torch.int32, device="cuda")
        # a step's rows
        self.q, self.q_rot, self.o = (torch.empty((n_seqs, hq, d), dtype=torch.bfloat16, device="cuda") for _ in range(3))
        self.k, self.v = (torch.empty((n_seqs, hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.row = torch.empty_like(self.len)
        sizes = [ba.ba_paged_attention_workspace_bytes(heads, n_seqs, 1, self.max_len)]
        if pages:
            sizes += [ba.ba_page_select_workspace_bytes(heads, n_seqs, page_rows, self.max_len),
                      ba.ba_paged_attention_selected_workspace_bytes(heads, n_seqs, 1, page_rows, self.max_len, pages)]
        self.step_ws = self.scratch(max(sizes))
        self.graph = None

    def ints(self, x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    def randn(self, tokens, n_heads, scale=1.0):
        return (torch.randn((tokens, n_heads, self.heads.head_dim), generator=self.gen, device="cuda") * scale).bfloat16()

    def scratch(self, nbytes):
        if self.ws.numel() < nbytes:
            self.ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        return self.ws

    def new_cache(self, tokens, rows):
        per_seq = -(-tokens // rows)
        k, v = (torch.empty((self.n * per_seq, rows, self.heads.n_kv_heads, self.heads.head_dim), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        return ba.PagedCache(k, v, torch.arange(self.n * per_seq, dtype=torch.int32, device="cuda").view(self.n, per_seq))

    def calls(self):
        self.row.copy_(self.len)
        # the token's row is behind what is kept, its rotation its place in the text
        ba.ba_paged_append(self.heads, None, self.cache, self.q, self.k, self.v, self.q_rot, self.row, None, self.position)
        self.len.add_(1)
        self.position.add_(1)
        if not self.pages:
            ba.ba_paged_attention(self.heads, self.cache, self.q_rot, self.o, None, self.len, self.max_len, ws=self.step_ws)
            return
        ba.ba_page_bounds(self.heads, self.cache, self.bounds, self.row, self.len, self.max_len)
        ba.ba_page_select(self.heads, self.cache, self.bounds, self.q_rot, self.len, self.max_len, self.selected, ws=self.step_ws)
        ba.ba_paged_attention_selected(self.heads, self.cache, self.q_rot, self.o, None, self.len, self.max_len, self.selected, ws=self.step_ws)

    def step(self):
        """One token of every sequence; -> its attention output."""
        self.q.copy_(self.randn(self.n, self.heads.n_q_heads, 2.0))
        self.k.copy_(self.randn(self.n, self.heads.n_kv_heads))
        self.v.copy_(self.randn(self.n, self.heads.n_kv_heads))
        if self.graph is None:
            self.calls()  # (ahead of the capture)
            self.graph = torch.cuda.CUDAGraph()
            done = self.o.clone()
            with torch.cuda.graph(self.graph):
                self.calls()
            return done
        self.graph.replay()
        return self.o


def main():
    heads = ba.Heads(32, 8, 128, 500000.0)
    for what, how in (("all keys", {}), ("1,024 kept", {"keep": 1024}), ("64 pages a step", {"pages": 64})):
        run = LongAnswers(heads, 16, 8000, 64, 65, **how)
        run.step()
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        for _ in range(64):
            run.step()
        end.record()
        torch.cuda.synchronize()
        print(f"16 sequences of 8,064 tokens, {what}: {begin.elapsed_time(end) / 64 * 1e3:.0f} us a token and layer")


if __name__ == "__main__":
    main()
