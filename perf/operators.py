"""The operators around the paged cache of answers, as timed cases.

Three operators and one gradient, each over the range of sizes in which it is used:

  norm       ba_norm_rotate: queries and keys normed per head and turned by their positions, in one pass
  norm_back  ba_norm_rotate_backward: the gradients of that, of the gains among them
  append     ba_paged_append: new (or cached) keys and values into pages, normed and turned on the way
  attend     ba_paged_attention: one or a few query tokens of every sequence over its pages; groups of
             sequences share the pages of a long prefix, which is attended to once for all

``listed`` names the cases, ``draw`` makes further ones of the same ranges, ``prepare`` builds what a
program has in hand before the call, ``run`` makes one pass, ``work`` says what a pass cannot do
without, ``exact`` what it returns, in 64 bits.
"""
import math
import random

import torch

own = False

LLAMA = {"n_q_heads": 32, "n_kv_heads": 8, "head_dim": 128, "rope_base": 500000.0}
SMALL = {"n_q_heads": 4, "n_kv_heads": 4, "head_dim": 64, "rope_base": 10000.0}
GEOMETRIES = [LLAMA, LLAMA, LLAMA, SMALL,
              {"n_q_heads": 8, "n_kv_heads": 2, "head_dim": 64, "rope_base": 10000.0},
              {"n_q_heads": 16, "n_kv_heads": 8, "head_dim": 128, "rope_base": 500000.0}]
EPS = 1e-6


def listed():
    return [
        # a 64-token question in front of its final block: launches and host work count
        {"name": "norm_question", "kind": "norm", **LLAMA, "layout": "interleaved", "tokens": 64, "dtype": "bf16", "rope": True},
        # one layer of a 32,000-token prompt
        {"name": "norm_prompt", "kind": "norm", **LLAMA, "layout": "half", "tokens": 32000, "dtype": "bf16", "rope": True},
        # a batch of a fine-tune step kept in 32 bits, an odd number of tokens, small heads
        {"name": "norm_f32", "kind": "norm", "n_q_heads": 8, "n_kv_heads": 2, "head_dim": 64, "rope_base": 10000.0, "layout": "interleaved",
         "tokens": 2077, "dtype": "f32", "rope": True},
        # one layer of a fine-tune step of eight prompts of some 4,000 tokens; the attention behind it rotates by itself
        {"name": "norm_back_train", "kind": "norm_back", **LLAMA, "layout": "interleaved", "tokens": 32513, "dtype": "bf16", "rope": False},
        # the same in 32 bits for one prompt of 2,064 tokens, rotation included
        {"name": "norm_back_f32", "kind": "norm_back", "n_q_heads": 16, "n_kv_heads": 8, "head_dim": 128, "rope_base": 500000.0,
         "layout": "half", "tokens": 2064, "dtype": "f32", "rope": True},
        # one sequence, one new token: the latency of a decoding step's append
        {"name": "append_one", "kind": "append", **LLAMA, "layout": "interleaved", "n_seqs": 1, "q_per_seq": 1, "len_min": 2064, "len_max": 2064,
         "page_rows": 16, "normed": True, "with_q": True, "shape_seed": 1},
        # a decoding step of 256 sequences of ragged length
        {"name": "append_batch", "kind": "append", **LLAMA, "layout": "half", "n_seqs": 256, "q_per_seq": 1, "len_min": 100, "len_max": 1000,
         "page_rows": 64, "normed": True, "with_q": True, "shape_seed": 2},
        # a context of 31 cached passages of 1,024 tokens goes into pages, each key turned by its passage's shift
        {"name": "append_context", "kind": "append", **LLAMA, "layout": "interleaved", "n_seqs": 1, "q_per_seq": 31744, "len_min": 31744,
         "len_max": 31744, "page_rows": 16, "normed": False, "with_q": False, "shape_seed": 3},
        # one sequence over ten passages of 200 tokens and a question: the latency of a decoding step's attention
        {"name": "attend_one", "kind": "attend", **LLAMA, "n_groups": 1, "members": 1, "q_per_seq": 1, "prefix_min": 0, "prefix_max": 0,
         "own_min": 2064, "own_max": 2064, "page_rows": 16, "shape_seed": 4},
        # 64 answers over one context of 31 passages of 1,024 tokens
        {"name": "attend_shared", "kind": "attend", **LLAMA, "n_groups": 1, "members": 64, "q_per_seq": 1, "prefix_min": 31744, "prefix_max": 31744,
         "own_min": 1, "own_max": 256, "page_rows": 64, "shape_seed": 5},
        # eight prompts of some 4,000 tokens, six drafted continuations of each, four tokens a step
        {"name": "attend_drafts", "kind": "attend", "n_q_heads": 16, "n_kv_heads": 8, "head_dim": 128, "rope_base": 500000.0, "n_groups": 8,
         "members": 6, "q_per_seq": 4, "prefix_min": 3400, "prefix_max": 4600, "own_min": 5, "own_max": 400, "page_rows": 16, "shape_seed": 6},
        # 128 unrelated conversations of very different length: nothing is shared
        {"name": "attend_apart", "kind": "attend", **LLAMA, "n_groups": 128, "members": 1, "q_per_seq": 1, "prefix_min": 0, "prefix_max": 0,
         "own_min": 1, "own_max": 8000, "page_rows": 64, "shape_seed": 7},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    case = {"kind": rng.choice(["norm", "norm_back", "append", "attend", "attend"]), **rng.choice(GEOMETRIES)}
    if case["kind"] in ("norm", "norm_back"):
        f32 = rng.random() < 0.3
        case.update(layout=rng.choice(["interleaved", "half"]), tokens=_log_int(rng, 1, 16000 if f32 else 32000), dtype="f32" if f32 else "bf16",
                    rope=rng.random() < 0.7)
        return case
    case.update(page_rows=rng.choice([16, 16, 32, 64, 128]), shape_seed=rng.randrange(1, 1 << 30))
    if case["kind"] == "append":
        n_seqs = _log_int(rng, 1, 256)
        per_seq = 1 if rng.random() < 0.5 else _log_int(rng, 1, max(1, 31744 // n_seqs))
        longest = max(per_seq, min(32000, 200000 // n_seqs))
        mean = _log_int(rng, per_seq, longest)
        case.update(layout=rng.choice(["interleaved", "half"]), n_seqs=n_seqs, q_per_seq=per_seq, len_min=max(per_seq, mean // 2),
                    len_max=max(per_seq, min(longest, mean + mean // 2)), normed=rng.random() < 0.6, with_q=rng.random() < 0.8)
        return case
    shared = rng.random() < 0.6
    if shared:
        prefix = _log_int(rng, 200, 31744)
        n_groups = _log_int(rng, 1, max(1, min(16, 64000 // prefix)))
        members = _log_int(rng, 2, max(2, min(64, 64 * 31744 // (n_groups * prefix), 512 // n_groups)))
        own_most = _log_int(rng, 1, max(1, min(1024, 200000 // (n_groups * members))))
        case.update(prefix_min=max(1, prefix // 2 + rng.randrange(3)), prefix_max=prefix)
    else:
        own_most = _log_int(rng, 1, 16000)
        n_groups, members = _log_int(rng, 1, max(1, min(256, 500000 // own_most))), 1
        case.update(prefix_min=0, prefix_max=0)
    per_seq = rng.choice([1, 1, 2, 3, 4, 8])
    case.update(n_groups=n_groups, members=members, q_per_seq=per_seq if members * per_seq <= 64 else 1, own_min=max(1, own_most // 8), own_max=own_most)
    return case


# ---- shapes -------------------------------------------------------------------------------------------------
def _between(rng, lo, hi, n):
    return [rng.randint(lo, hi) for _ in range(n)]


def _shape(case):
    """Lengths of the sequences (all tokens, the new ones among them), the prefixes of the groups, and pages a sequence."""
    rng = random.Random(case["shape_seed"])
    if case["kind"] == "append":
        lens = _between(rng, case["len_min"], case["len_max"], case["n_seqs"])
        prefix = [0] * case["n_seqs"]
    else:
        prefix = _between(rng, case["prefix_min"], case["prefix_max"], case["n_groups"])
        behind = _between(rng, case["own_min"], case["own_max"], case["n_groups"] * case["members"])
        # (a step's new tokens are its own: they lie behind the prefix)
        lens = [prefix[s // case["members"]] + max(n, case["q_per_seq"]) for s, n in enumerate(behind)]
    return {"lens": lens, "prefix": prefix, "pages": -(-max(lens) // case["page_rows"])}


def work(case):
    hq, hkv, d = case["n_q_heads"], case["n_kv_heads"], case["head_dim"]
    if case["kind"] in ("norm", "norm_back"):
        n = case["tokens"] * (hq + hkv) * d
        size = 4 if case["dtype"] == "f32" else 2
        back = case["kind"] == "norm_back"
        return {"bytes": n * size * (3 if back else 2) + 4 * case["tokens"], "flops": n * (14 if back else 7)}
    s = _shape(case)
    if case["kind"] == "append":
        t = case["n_seqs"] * case["q_per_seq"]
        rows = (2 * hkv + (hq if case["with_q"] else 0)) * d
        return {"bytes": 4 * t * rows + 8 * t, "flops": 7 * t * rows}
    nq, m = case["q_per_seq"], case["members"]
    # the pages of a prefix count once, a sequence's own once; of the pairs those that the tokens see
    keys = sum(s["prefix"]) + sum(n - s["prefix"][i // m] for i, n in enumerate(s["lens"]))
    pairs = sum(nq * n - nq * (nq - 1) / 2 for n in s["lens"])
    rows = len(s["lens"]) * nq * hq
    return {"bytes": 4 * d * hkv * keys + 4 * d * rows + 4 * rows, "flops": 4 * d * hq * pairs}


# ---- inputs -------------------------------------------------------------------------------------------------
def _dtype(case):
    return torch.float32 if case.get("dtype") == "f32" else torch.bfloat16


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    hq, hkv, d = case["n_q_heads"], case["n_kv_heads"], case["head_dim"]

    def randn(*shape, dtype=torch.bfloat16, scale=1.0):
        return (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * scale).to(dtype)

    def gains():  # of a trained model: about one, in the type of its weights
        return (1.0 + 0.2 * torch.randn(d, generator=gen, device="cuda")).to(_dtype(case))

    if case["kind"] in ("norm", "norm_back"):
        t, dtype = case["tokens"], _dtype(case)
        # projected activations; a step's gradients are small
        st = {"q": randn(t, hq, d, dtype=dtype, scale=1.5), "k": randn(t, hkv, d, dtype=dtype, scale=0.7), "q_weight": gains(), "k_weight": gains()}
        # several prompts one after the other, each from position 0 on
        st["positions"] = (torch.arange(t, device="cuda") % (4064 if case["kind"] == "norm_back" else 32000)).int()
        if case["kind"] == "norm_back":
            st.update(d_q=randn(t, hq, d, dtype=dtype, scale=0.02), d_k=randn(t, hkv, d, dtype=dtype, scale=0.05))
        return st
    s = _shape(case)
    lens = torch.tensor(s["lens"], device="cuda", dtype=torch.int32)
    n_seqs, pages, rows = len(s["lens"]), s["pages"], case["page_rows"]
    members = case.get("members", 1)
    prefix = torch.tensor(s["prefix"], device="cuda").repeat_interleave(members)[:, None]  # [sequences, 1]
    # the pool's pages are handed out in any order; those that lie wholly in a prefix are its group's first sequence's
    page = torch.arange(pages, device="cuda")[None, :]
    first = (torch.arange(n_seqs, device="cuda") // members * members)[:, None]
    owner = torch.where((page + 1) * rows <= prefix, first, torch.arange(n_seqs, device="cuda")[:, None])
    used = page * rows < lens[:, None]
    flat = owner * pages + page
    n_pages = int(used.sum()) + 3
    ids, where = torch.unique(flat[used], return_inverse=True)
    order = torch.randperm(n_pages, generator=gen, device="cuda")
    table = torch.full((n_seqs, pages), -1, device="cuda", dtype=torch.int64)
    table[used] = order[where]
    st = {"table": table.int(), "lens": lens, "k_pages": randn(n_pages, rows, hkv, d), "v_pages": randn(n_pages, rows, hkv, d)}
    if case["kind"] == "append":
        nq = case["q_per_seq"]
        t = n_seqs * nq
        st.update(k=randn(t, hkv, d), v=randn(t, hkv, d), q=randn(t, hq, d) if case["with_q"] else None)
        st["seq"] = torch.arange(n_seqs, device="cuda").repeat_interleave(nq).int()
        st["at"] = (lens[:, None] - nq + torch.arange(nq, device="cuda")[None, :]).reshape(-1).int()
        # cached passages carry their own rotation: they turn by the place of their first token
        st["turn"] = st["at"] if case["with_q"] else (st["at"] // 1024 * 1024).int()
        if case["normed"]:
            st.update(q_weight=gains(), k_weight=gains())
        return st
    # a page that a prefix ends in is a copy of its own for every other sequence of the group: the prefix's rows are the same in it
    split = (prefix % rows > 0) & (page == prefix // rows)  # [sequences, pages], one a sequence at most
    copies = table[split]
    source = torch.where(split, table[first[:, 0]], 0).sum(1)[split.any(1)]
    shared = (torch.arange(rows, device="cuda")[None, :] < (prefix % rows)[split.any(1)])[:, :, None, None]
    for pool in (st["k_pages"], st["v_pages"]):
        pool[copies] = torch.where(shared, pool[source], pool[copies])
    # normed queries and keys: scores of a standard deviation of about two
    st["q"] = randn(n_seqs * case["q_per_seq"], hq, d, scale=2.0)
    st["prefix"] = s["prefix"]
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    st["case"] = case
    if case["kind"] == "attend":
        lens = _shape(case)["lens"]
        st["max_len"] = max(lens)
        st["behind"] = max(n - st["prefix"][i // case["members"]] for i, n in enumerate(lens))
    if own:
        st.update(_handles(case, st))
    return st


def _handles(case, st):
    """What a program keeps between the calls: descriptions of heads, norm and cache, the outputs' memory, a workspace."""
    from paper_2409_15355_amd import binding as ba
    heads = ba.Heads(case["n_q_heads"], case["n_kv_heads"], case["head_dim"], case["rope_base"],
                     rope_layout=ba.ROPE_HALF if case.get("layout") == "half" else ba.ROPE_INTERLEAVED)
    got = {"ba": ba, "heads": heads, "q_out": None if st["q"] is None else torch.empty_like(st["q"])}
    if "q_weight" in st:
        got["norm"] = ba.HeadNorm(st["q_weight"], st["k_weight"], EPS)
    nbytes = 0
    if case["kind"] == "norm":
        got["k_out"] = torch.empty_like(st["k"])
    elif case["kind"] == "norm_back":
        d = case["head_dim"]
        got.update(dk=torch.empty_like(st["k"]), dwq=torch.empty(d, device="cuda"), dwk=torch.empty(d, device="cuda"))
        nbytes = ba.ba_norm_rotate_backward_workspace_bytes(heads, case["tokens"])
    else:
        got["cache"] = ba.PagedCache(st["k_pages"], st["v_pages"], st["table"])
    if case["kind"] == "attend":
        n_seqs, m = len(st["lens"]), case["members"]
        got["lse"] = torch.empty(st["q"].shape[:2], device="cuda")
        # sequences of their own need no groups
        got["cu_group"] = torch.arange(0, n_seqs + 1, m).int().numpy() if case["prefix_max"] else None
        got["prefix_len"] = torch.tensor(st["prefix"]).int().numpy() if case["prefix_max"] else None
        nbytes = ba.ba_paged_attention_workspace_bytes(heads, n_seqs, case["q_per_seq"], st["max_len"], got["cu_group"], got["prefix_len"])
    got["ws"] = torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device="cuda")
    return got


# ---- one pass -----------------------------------------------------------------------------------------------
def run(st):
    return (_run_own if own else _run_plain)(st)


def _run_own(st):
    case, ba = st["case"], st["ba"]
    mode = ba.ROPE_APPLY if case.get("rope", True) else ba.ROPE_NONE
    if case["kind"] == "norm":
        ba.ba_norm_rotate(st["heads"], st["norm"], st["q"], st["k"], st["q_out"], st["k_out"], st["positions"], mode)
        return [st["q_out"], st["k_out"]]
    if case["kind"] == "norm_back":
        ba.ba_norm_rotate_backward(st["heads"], st["norm"], st["q"], st["k"], st["d_q"], st["d_k"], st["q_out"], st["dk"], st["dwq"], st["dwk"],
                                   st["positions"], mode, st["ws"])
        return [st["q_out"], st["dk"], st["dwq"], st["dwk"]]
    if case["kind"] == "append":
        ba.ba_paged_append(st["heads"], st.get("norm"), st["cache"], st["q"], st["k"], st["v"], st["q_out"], st["at"], st["seq"], st["turn"], mode)
        return [st["q_out"], st["k_pages"], st["v_pages"]]
    ba.ba_paged_attention(st["heads"], st["cache"], st["q"], st["q_out"], st["lse"], st["lens"], st["max_len"], st["cu_group"], st["prefix_len"],
                          case["q_per_seq"], st["ws"])
    return [st["q_out"], st["lse"]]


# ---- the plain forms ----------------------------------------------------------------------------------------
def _angles(case, positions):
    """cos and sin of position * theta_j (the angle itself needs 64 bits: it has thousands of turns)."""
    d = case["head_dim"]
    freq = case["rope_base"] ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device="cuda") / d)
    angle = positions.double()[:, None, None] * freq
    return angle.cos().float(), angle.sin().float()


def _turned(case, x, c, s):
    d = case["head_dim"]
    if case["layout"] == "half":
        a, b = x[..., : d // 2], x[..., d // 2:]
        return torch.cat([c * a - s * b, s * a + c * b], dim=-1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([c * a - s * b, s * a + c * b], dim=-1).reshape(x.shape)


def _normed(x, w):
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()


def _norm_back(x, w, g):
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    n, b = x * r, g * w.float()
    return r * (b - n * (b * n).mean(-1, keepdim=True)), (g * n).sum(dim=(0, 1))


def _run_plain(st):
    case = st["case"]
    if case["kind"] == "attend":
        return _attend_plain(st)
    if case["kind"] == "append":
        c, s = _angles(case, st["turn"])
        k, q = st["k"].float(), None if st["q"] is None else st["q"].float()
        if case["normed"]:
            k = _normed(k, st["k_weight"])
            q = None if q is None else _normed(q, st["q_weight"])
        page = st["table"][st["seq"].long(), (st["at"] // case["page_rows"]).long()].long()
        row = (st["at"] % case["page_rows"]).long()
        st["k_pages"][page, row] = _turned(case, k, c, s).bfloat16()
        st["v_pages"][page, row] = st["v"]
        return [None if q is None else _turned(case, q, c, s).bfloat16(), st["k_pages"], st["v_pages"]]
    q, k = st["q"].float(), st["k"].float()
    c, s = _angles(case, st["positions"]) if case["rope"] else (None, None)
    if case["kind"] == "norm":
        q, k = _normed(q, st["q_weight"]), _normed(k, st["k_weight"])
        if case["rope"]:
            q, k = _turned(case, q, c, s), _turned(case, k, c, s)
        return [q.to(_dtype(case)), k.to(_dtype(case))]
    gq, gk = st["d_q"].float(), st["d_k"].float()
    if case["rope"]:  # the rotation's transpose turns back
        gq, gk = _turned(case, gq, c, -s), _turned(case, gk, c, -s)
    dq, dwq = _norm_back(q, st["q_weight"], gq)
    dk, dwk = _norm_back(k, st["k_weight"], gk)
    return [dq.to(_dtype(case)), dk.to(_dtype(case)), dwq, dwk]


def _gathered(pages, table, at):
    """Rows `at` [n, keys] of the sequences whose pages `table` [n, pages] names, as [n, KV heads, keys, D]."""
    rows = pages.shape[1]
    page = table.long().gather(1, (at // rows).clamp(max=table.shape[1] - 1)).clamp(min=0)
    return pages[page, at % rows].float().transpose(1, 2).contiguous()


def _attend_plain(st):
    case = st["case"]
    hq, hkv, d, nq, m = case["n_q_heads"], case["n_kv_heads"], case["head_dim"], case["q_per_seq"], case["members"]
    n_seqs, n_groups, g = len(st["lens"]), case["n_groups"], hq // hkv
    prefix = torch.tensor(st["prefix"], device="cuda")
    longest, behind = max(st["prefix"]), st["behind"]
    lens, before = st["lens"].long(), prefix.repeat_interleave(m)
    last = lens[:, None] - nq + torch.arange(nq, device="cuda")[None, :]  # the last key that a token sees
    q = st["q"].float().view(n_seqs, nq, hkv, g, d).permute(0, 2, 1, 3, 4) / math.sqrt(d)
    # a sequence's own keys
    at = before[:, None] + torch.arange(behind, device="cuda")[None, :]
    k, v = _gathered(st["k_pages"], st["table"], at), _gathered(st["v_pages"], st["table"], at)
    there = (at < lens[:, None])[:, None, :, None]
    sc = torch.matmul(q.reshape(n_seqs, hkv, nq * g, d), k.transpose(2, 3).contiguous()).view(n_seqs, hkv, nq, g, behind)
    sc = sc.masked_fill((at[:, None, :] > last[:, :, None])[:, None, :, None, :], -math.inf)
    top = sc.amax(-1, keepdim=True)
    if longest:
        # the prefixes, once for all rows of a group
        at = torch.arange(longest, device="cuda").expand(n_groups, -1)
        kp, vp = _gathered(st["k_pages"], st["table"][::m], at), _gathered(st["v_pages"], st["table"][::m], at)
        there_p = (at < prefix[:, None])[:, None, :, None]
        qg = q.reshape(n_groups, m, hkv, nq * g, d).transpose(1, 2).reshape(n_groups, hkv, m * nq * g, d)
        sp = torch.matmul(qg, kp.transpose(2, 3).contiguous())
        sp = sp.masked_fill((at >= prefix[:, None])[:, None, None, :], -math.inf)
        of_group = lambda x: x.reshape(n_groups, m, hkv, nq * g, -1).transpose(1, 2).reshape(n_groups, hkv, m * nq * g, -1)  # noqa: E731
        of_seq = lambda x: x.view(n_groups, hkv, m, nq * g, -1).transpose(1, 2).reshape(n_seqs, hkv, nq, g, -1)  # noqa: E731
        top = torch.maximum(top, of_seq(sp.amax(-1, keepdim=True)))
        sp = torch.exp(sp - of_group(top))
        more, out = of_seq(sp.sum(-1, keepdim=True)), of_seq(torch.matmul(sp, vp * there_p))
    else:
        more, out = 0.0, 0.0
    p = torch.exp(sc - top)
    total = p.sum(-1, keepdim=True) + more
    out = out + torch.matmul(p.view(n_seqs, hkv, nq * g, behind), v * there).view(n_seqs, hkv, nq, g, d)
    lse = (top + torch.log(total)).squeeze(-1)
    to_rows = lambda x: x.permute(0, 2, 1, 3, *range(4, x.dim())).reshape(n_seqs * nq, hq, *x.shape[4:])  # noqa: E731
    return [to_rows(out / total).bfloat16(), to_rows(lse)]


# ---- the same in 64 bits, one head or one sequence after the other ----------------------------------------------
def _rotation(case, positions, sign=1.0):
    """exp(i position theta_j), [tokens, 1, D / 2]."""
    j = torch.arange(case["head_dim"] // 2, device="cuda", dtype=torch.float64)
    theta = torch.exp(-2.0 * j / case["head_dim"] * math.log(case["rope_base"]))
    return torch.exp(1j * sign * positions.double()[:, None, None] * theta)


def _as_pairs(case, x):
    half = case["head_dim"] // 2
    return torch.complex(x[..., :half], x[..., half:]) if case["layout"] == "half" else torch.view_as_complex(x.unflatten(-1, (half, 2)).contiguous())


def _from_pairs(case, z):
    return torch.cat([z.real, z.imag], dim=-1) if case["layout"] == "half" else torch.view_as_real(z).flatten(-2)


def _norm64(case, x, w, positions):
    y = x / ((x ** 2).sum(-1, keepdim=True) / case["head_dim"] + EPS).sqrt()
    y = y if w is None else y * w.double()
    return y if positions is None else _from_pairs(case, _as_pairs(case, y) * _rotation(case, positions))


def exact(case, seed):
    st = _inputs(case, seed)
    if case["kind"] == "attend":
        return _attend64(case, st)
    if case["kind"] == "append":
        turn = lambda x: _from_pairs(case, _as_pairs(case, x) * _rotation(case, st["turn"]))  # noqa: E731
        rows = lambda x, w: _norm64(case, x.double(), st[w], st["turn"]) if case["normed"] else turn(x.double())  # noqa: E731
        pools = [st["k_pages"].double(), st["v_pages"].double()]
        place = st["table"].reshape(-1)[(st["seq"] * st["table"].shape[1] + torch.div(st["at"], case["page_rows"], rounding_mode="floor")).long()].long()
        place = place * case["page_rows"] + st["at"].long() % case["page_rows"]
        for pool, new in zip(pools, (rows(st["k"], "k_weight"), st["v"].double())):
            pool.view(-1, *pool.shape[2:])[place] = new
        return [None if st["q"] is None else rows(st["q"], "q_weight"), *pools]
    at = st["positions"] if case["rope"] else None
    if case["kind"] == "norm":
        return [_norm64(case, st["q"].double(), st["q_weight"], at), _norm64(case, st["k"].double(), st["k_weight"], at)]
    outs, gains = [], []
    for x, w, g in ((st["q"], st["q_weight"], st["d_q"]), (st["k"], st["k_weight"], st["d_k"])):
        dx, dw = torch.empty(x.shape, dtype=torch.float64, device="cuda"), torch.zeros(case["head_dim"], dtype=torch.float64, device="cuda")
        for h in range(x.shape[1]):  # a head at a time
            xh, gh = x[:, h:h + 1].double(), g[:, h:h + 1].double()
            if case["rope"]:
                gh = _from_pairs(case, _as_pairs(case, gh) * _rotation(case, at, -1.0))
            norm = ((xh ** 2).sum(-1, keepdim=True) / case["head_dim"] + EPS).sqrt()
            dw += (gh * xh / norm).sum(dim=(0, 1))
            gw = gh * w.double()
            dx[:, h:h + 1] = gw / norm - xh * (gw * xh).sum(-1, keepdim=True) / (case["head_dim"] * norm ** 3)
        outs.append(dx)
        gains.append(dw)
    return outs + gains


def _attend64(case, st):
    hq, hkv, d, nq = case["n_q_heads"], case["n_kv_heads"], case["head_dim"], case["q_per_seq"]
    lens = st["lens"].tolist()
    out = torch.empty((len(lens), nq, hq, d), dtype=torch.float64, device="cuda")
    lse = torch.empty((len(lens), nq, hq), dtype=torch.float64, device="cuda")
    q = st["q"].double().view(len(lens), nq, hkv, hq // hkv, d)
    for s, n in enumerate(lens):
        pages = st["table"][s, : -(-n // case["page_rows"])].long()
        k, v = (x[pages].flatten(0, 1)[:n].double().transpose(0, 1).contiguous() for x in (st["k_pages"], st["v_pages"]))
        for i in range(nq):
            seen = n - nq + i + 1
            sc = (q[s, i] @ k[:, :seen].transpose(1, 2).contiguous()) / math.sqrt(d)  # [KV heads, group, keys]
            norm = torch.logsumexp(sc, dim=-1)
            out[s, i] = (torch.exp(sc - norm[..., None]) @ v[:, :seen]).reshape(hq, d)
            lse[s, i] = norm.reshape(hq)
    return [out.reshape(-1, hq, d), lse.reshape(-1, hq)]
