"""Many questions over one set of passages, answered token by token: one attention layer of a model that norms its queries and keys.

    python examples/answer_questions.py

1. The passages are encoded once, each on its own (ba_norm_rotate at local positions, ba_encode_blocks): their rotated keys and
   their values are the cache that Block-attention keeps.
2. A prompt's passages go into pages, every key turned by its passage's shift on the way (ba_paged_append, no norm).  All questions
   share these pages.
3. The questions are appended and attend to the passages and themselves, all of them in one call (ba_paged_append with norm,
   rotation and queries; ba_paged_attention with q_per_seq = the question's length).
4. The answers: one token of every question at a time, append and attention captured in a graph once and replayed.

``tune`` is the same layer in a fine-tune step: head norms in front of Block-attention's forward and backward pass, the gradients of the
gains at the end.  Activations are random numbers: what stands around attention in a model is left out.
"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2409_15355_amd import binding as ba  # noqa: E402


class Layer:
    """What a program keeps for one attention layer: head shapes, the norm's gains, a workspace that grows."""

    def __init__(self, n_q_heads=32, n_kv_heads=8, head_dim=128, rope_base=500000.0, rope_layout=ba.ROPE_INTERLEAVED, seed=0):
        self.heads = ba.Heads(n_q_heads, n_kv_heads, head_dim, rope_base, rope_layout=rope_layout)
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.q_gain, self.k_gain = (1.0 + 0.2 * self.randn(head_dim, dtype=torch.float32) for _ in range(2))
        self.norm = ba.HeadNorm(self.q_gain, self.k_gain, eps=1e-6)
        self.ws = torch.empty(256, dtype=torch.uint8, device="cuda")

    def randn(self, *shape, dtype=torch.bfloat16):
        return torch.randn(shape, generator=self.gen, device="cuda").to(dtype)

    def qkv(self, tokens):
        """Stand-in for the projections: tokens x (query, key, value) heads, side by side in one matrix."""
        h = self.heads
        x = self.randn(tokens, h.n_q_heads + 2 * h.n_kv_heads, h.head_dim)
        return x.split([h.n_q_heads, h.n_kv_heads, h.n_kv_heads], dim=1)

    def scratch(self, nbytes):
        if self.ws.numel() < nbytes:
            self.ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        return self.ws


def positions_of(lens):
    """Each block's tokens from 0 on."""
    return torch.cat([torch.arange(n, dtype=torch.int32) for n in lens]).cuda()


def encode_passages(layer, lens):
    """-> (rotated keys, values) of all passages, as cached: positions local to the passage."""
    q, k, v = layer.qkv(sum(lens))
    offs = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    q_rot, k_rot = torch.empty_like(q, memory_format=torch.contiguous_format), torch.empty_like(k, memory_format=torch.contiguous_format)
    ba.ba_norm_rotate(layer.heads, layer.norm, q, k, q_rot, k_rot, positions_of(lens))
    o = torch.empty_like(q_rot)  # (what the layers behind this one would go on with)
    ws = layer.scratch(ba.ba_encode_blocks_workspace_bytes(layer.heads, offs, ba.ROPE_NONE))
    ba.ba_encode_blocks(layer.heads, q_rot, k_rot, v.contiguous(), o, None, offs, ba.ROPE_NONE, ws)
    return k_rot, v.contiguous()


def answer(layer, passage_lens, n_questions, question, steps, page_rows=16):
    """Returns everything that a check wants: the cache, and per step the rotated queries, the outputs and log-sum-exps."""
    h = layer.heads
    k_cached, v_cached = encode_passages(layer, passage_lens)
    context = sum(passage_lens)
    max_len = context + question + steps
    # pages: those that lie wholly in the context are everybody's, the others each question's own
    shared, pages = context // page_rows, -(-max_len // page_rows)
    own = pages - shared
    order = torch.randperm(shared + n_questions * own, generator=torch.Generator().manual_seed(1)).int()
    table = torch.empty((n_questions, pages), dtype=torch.int32)
    table[:, :shared] = order[:shared]
    table[:, shared:] = order[shared:].view(n_questions, own)
    k_pages, v_pages = (torch.empty((len(order), page_rows, h.n_kv_heads, h.head_dim), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache = ba.PagedCache(k_pages, v_pages, table.cuda())

    # the passages, in the prompt's order: a key of passage b turns by the place of the passage's first token.  What lies in pages of
    # their own goes to every question's.
    starts = np.concatenate([[0], np.cumsum(passage_lens)[:-1]])
    shift = torch.from_numpy(np.repeat(starts, passage_lens).astype(np.int32)).cuda()
    at = torch.arange(context, dtype=torch.int32, device="cuda")
    tail = context % page_rows
    ba.ba_paged_append(h, None, cache, None, k_cached, v_cached, None, at, torch.zeros_like(at), shift)
    if tail and n_questions > 1:
        rows = slice(context - tail, context)
        others = torch.arange(1, n_questions, dtype=torch.int32, device="cuda").repeat_interleave(tail)
        again = (n_questions - 1, 1, 1)
        ba.ba_paged_append(h, None, cache, None, k_cached[rows].repeat(again), v_cached[rows].repeat(again), None,
                           at[rows].repeat(n_questions - 1), others, shift[rows].repeat(n_questions - 1))

    cu_group, prefix = np.array([0, n_questions], dtype=np.int32), np.array([context], dtype=np.int32)
    need = max(ba.ba_paged_attention_workspace_bytes(h, n_questions, n, max_len, cu_group, prefix) for n in (question, 1))
    ws = layer.scratch(need)
    done = []

    # the questions, all tokens at once
    q, k, v = layer.qkv(n_questions * question)
    seq = torch.arange(n_questions, dtype=torch.int32, device="cuda").repeat_interleave(question)
    at = (context + torch.arange(question, dtype=torch.int32, device="cuda")).repeat(n_questions)
    lens = torch.full((n_questions,), context + question, dtype=torch.int32, device="cuda")
    q_rot = torch.empty(q.shape, dtype=q.dtype, device="cuda")
    o, lse = torch.empty_like(q_rot), torch.empty(q.shape[:2], device="cuda")
    ba.ba_paged_append(h, layer.norm, cache, q, k, v, q_rot, at, seq)
    ba.ba_paged_attention(h, cache, q_rot, o, lse, lens, max_len, cu_group, prefix, question, ws)
    done.append((q_rot, o, lse, lens.clone()))

    # the answers, a token each at a time; the step is captured once
    q, k, v = layer.qkv(n_questions)
    q_rot, at = torch.empty(q.shape, dtype=q.dtype, device="cuda"), lens.clone()
    o, lse = torch.empty_like(q_rot), torch.empty(q.shape[:2], device="cuda")
    lens += 1

    def step():
        ba.ba_paged_append(h, layer.norm, cache, q, k, v, q_rot, at)
        ba.ba_paged_attention(h, cache, q_rot, o, lse, lens, max_len, cu_group, prefix, 1, ws)

    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    for i in range(steps):
        if i:
            for x, new in zip((q, k, v), layer.qkv(n_questions)):
                x.copy_(new)
            at += 1
            lens += 1
        graph.replay()
        done.append((q_rot.clone(), o.clone(), lse.clone(), lens.clone()))
    return {"cache": cache, "k_cached": k_cached, "context": context, "done": done}


def tune(layer, block_lens, q, k, v, d_out):
    """Forward and backward of one prompt's attention, the last block seeing the others -> (output, gradients of q, k, v and of the gains)."""
    h = layer.heads
    offs = np.concatenate([[0], np.cumsum(block_lens)]).astype(np.int32)
    cu_blk = np.array([0, len(block_lens)], dtype=np.int32)
    tokens = int(offs[-1])
    new = lambda x: torch.empty(x.shape, dtype=x.dtype, device="cuda")  # noqa: E731
    # normed here, rotated inside: the backward pass returns the gradients of the un-rotated rows
    q_n, k_n, o, lse = new(q), new(k), new(q), torch.empty((tokens, h.n_q_heads), device="cuda")
    ba.ba_norm_rotate(h, layer.norm, q, k, q_n, k_n, None, ba.ROPE_NONE)
    ws = layer.scratch(max(ba.ba_block_attention_prompts_workspace_bytes(h, cu_blk, offs),
                           ba.ba_block_attention_prompts_backward_workspace_bytes(h, cu_blk, offs),
                           ba.ba_norm_rotate_backward_workspace_bytes(h, tokens)))
    ba.ba_block_attention_prompts(h, q_n, k_n, v, o, None, lse, cu_blk, offs, ba.ROPE_APPLY, ws)
    dq, dk, dv = new(q), new(k), new(v)
    ba.ba_block_attention_prompts_backward(h, q_n, k_n, v, o, lse, d_out, dq, dk, dv, cu_blk, offs, ws)
    d_q_gain, d_k_gain = torch.empty_like(layer.q_gain), torch.empty_like(layer.k_gain)
    ba.ba_norm_rotate_backward(h, layer.norm, q, k, dq, dk, dq, dk, d_q_gain, d_k_gain, None, ba.ROPE_NONE, ws)  # (in place)
    return o, dq, dk, dv, d_q_gain, d_k_gain


def main():
    layer = Layer()
    got = answer(layer, [1024] * 31, n_questions=64, question=16, steps=32)
    torch.cuda.synchronize()
    q, k, v = layer.qkv(2064)
    grads = tune(layer, [200] * 10 + [64], q, k, v, layer.randn(*q.shape))
    torch.cuda.synchronize()
    print(f"64 questions over {got['context']} tokens of passages: {len(got['done']) - 1} tokens each; "
          f"the gains' gradients of a fine-tune step: {grads[4].norm():.3f}, {grads[5].norm():.3f}")


if __name__ == "__main__":
    main()
