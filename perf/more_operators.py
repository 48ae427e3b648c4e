"""The operators that keep long paged caches affordable, as timed cases.

Five operators, each over the range of sizes in which it is used:

  weights  ba_paged_key_weights: how much attention every cached key has been given, added up over the queries
           of a step, of a question, or of all the answers that share a prefix
  evict    ba_paged_evict: the heaviest keys of every sequence and head, and their values, move to fewer pages
  bounds   ba_page_bounds: for every page the largest and the smallest key in each dimension, in 8 bits
  select   ba_page_select: the pages whose bounds promise a sequence's newest queries the largest scores
  attend   ba_paged_attention_selected: attention over the selected pages alone

``listed`` names the cases, ``draw`` makes further ones of the same ranges, ``prepare`` builds what a
program has in hand before the call, ``run`` makes one pass, ``work`` says what a pass cannot do
without, ``exact`` what it returns, in 64 bits.
"""
import math
import random

import torch

own = False

WIDE = {"n_q_heads": 32, "n_kv_heads": 8, "head_dim": 128}
GEOMETRIES = [WIDE, WIDE, WIDE,
              {"n_q_heads": 4, "n_kv_heads": 4, "head_dim": 64},
              {"n_q_heads": 8, "n_kv_heads": 2, "head_dim": 64},
              {"n_q_heads": 16, "n_kv_heads": 8, "head_dim": 128}]
MIN_EXP, MAX_EXP = -60, 40  # of the bounds' and the queries' powers of two


def listed():
    return [
        # one sequence over ten passages of 200 tokens and a question, one new token: the latency of a decoding step
        {"name": "weights_step", "kind": "weights", **WIDE, "n_groups": 1, "members": 1, "q_per_seq": 1, "prefix_min": 0, "prefix_max": 0,
         "own_min": 2064, "own_max": 2064, "page_rows": 16, "decay": 1.0, "shape_seed": 1},
        # a question of 256 tokens says which keys of 31 passages of 1,024 tokens matter
        {"name": "weights_question", "kind": "weights", **WIDE, "n_groups": 1, "members": 1, "q_per_seq": 256, "prefix_min": 0, "prefix_max": 0,
         "own_min": 32000, "own_max": 32000, "page_rows": 64, "decay": 0.0, "shape_seed": 2},
        # a step of 64 answers over one context of 31 passages of 1,024 tokens: each answer counts for itself
        {"name": "weights_shared", "kind": "weights", **WIDE, "n_groups": 1, "members": 64, "q_per_seq": 1, "prefix_min": 31744,
         "prefix_max": 31744, "own_min": 1, "own_max": 256, "page_rows": 64, "decay": 0.96875, "shape_seed": 3},
        # one conversation of 2,064 tokens is cut to 512
        {"name": "evict_one", "kind": "evict", **WIDE, "n_seqs": 1, "len_min": 2064, "len_max": 2064, "page_rows": 16, "to_rows": 16, "n_keep": 512,
         "n_first": 4, "n_last": 64, "shape_seed": 4},
        # 64 of very different length to 1,024 at most; those that are shorter only move
        {"name": "evict_batch", "kind": "evict", **WIDE, "n_seqs": 64, "len_min": 500, "len_max": 8000, "page_rows": 16, "to_rows": 64, "n_keep": 1024,
         "n_first": 16, "n_last": 256, "shape_seed": 5},
        # a decoding step of 128 sequences: their newest page takes one more key each
        {"name": "bounds_step", "kind": "bounds", **WIDE, "n_seqs": 128, "len_min": 100, "len_max": 4000, "page_rows": 32, "new": 1, "shape_seed": 6},
        # a context of 31 cached passages of 1,024 tokens, all of it
        {"name": "bounds_context", "kind": "bounds", **WIDE, "n_seqs": 1, "len_min": 31744, "len_max": 31744, "page_rows": 16, "new": 0,
         "shape_seed": 7},
        # one answer over 32,000 tokens: 128 pages of 16 out of 2,000
        {"name": "select_one", "kind": "select", **WIDE, "n_seqs": 1, "q_per_seq": 1, "len_min": 32000, "len_max": 32000, "page_rows": 16,
         "n_select": 128, "n_first": 1, "n_last": 4, "shape_seed": 8},
        # a step of 64 sequences of very different length, two drafted tokens each
        {"name": "select_batch", "kind": "select", **WIDE, "n_seqs": 64, "q_per_seq": 2, "len_min": 500, "len_max": 16000, "page_rows": 16,
         "n_select": 96, "n_first": 1, "n_last": 3, "shape_seed": 9},
        # the attention behind the one answer's selection
        {"name": "attend_one", "kind": "attend", **WIDE, "n_seqs": 1, "q_per_seq": 1, "len_min": 32000, "len_max": 32000, "page_rows": 16,
         "n_select": 128, "shape_seed": 10},
        # 128 sequences that each read 2,048 keys of some thousands
        {"name": "attend_batch", "kind": "attend", **WIDE, "n_seqs": 128, "q_per_seq": 1, "len_min": 1000, "len_max": 6000, "page_rows": 32,
         "n_select": 64, "shape_seed": 11},
        # 24 sequences of the smaller geometry, four drafted tokens each
        {"name": "attend_drafts", "kind": "attend", "n_q_heads": 16, "n_kv_heads": 8, "head_dim": 128, "n_seqs": 24, "q_per_seq": 4,
         "len_min": 3000, "len_max": 9000, "page_rows": 64, "n_select": 24, "shape_seed": 12},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    case = {"kind": rng.choice(["weights", "weights", "evict", "bounds", "select", "attend"]), **rng.choice(GEOMETRIES)}
    case.update(page_rows=rng.choice([16, 16, 32, 64, 128]), shape_seed=rng.randrange(1, 1 << 30))
    if case["kind"] == "weights":
        case["decay"] = rng.choice([0.0, 1.0, 0.96875])
        if rng.random() < 0.4:  # a shared prefix
            prefix = _log_int(rng, 200, 31744)
            n_groups = _log_int(rng, 1, max(1, min(8, 64000 // prefix)))
            members = _log_int(rng, 2, max(2, min(64, 64 * 31744 // (n_groups * prefix), 256 // n_groups)))
            own_most = _log_int(rng, 1, max(1, min(1024, 100000 // (n_groups * members))))
            per_seq = rng.choice([1, 1, 2, 4])
            case.update(prefix_min=max(1, prefix // 2 + rng.randrange(3)), prefix_max=prefix)
        else:
            own_most, members = _log_int(rng, 1, 31744), 1
            n_groups = _log_int(rng, 1, max(1, min(128, 250000 // own_most)))
            most = max(1, min(256, own_most, 8000000 // (n_groups * own_most)))
            per_seq = 1 if rng.random() < 0.4 else _log_int(rng, 1, most)
            case.update(prefix_min=0, prefix_max=0)
        case.update(n_groups=n_groups, members=members, q_per_seq=per_seq, own_min=max(1, own_most // 8), own_max=own_most)
        return case
    longest = _log_int(rng, 1, 32000)
    n_seqs = _log_int(rng, 1, max(1, min(128, 400000 // longest)))
    case.update(n_seqs=n_seqs, len_min=max(1, longest // rng.choice([1, 2, 8])), len_max=longest)
    if case["kind"] == "evict":
        n_keep = _log_int(rng, 1, max(1, min(4096, 65536 // n_seqs)))
        first = rng.choice([0, min(4, n_keep // 4)])
        case.update(to_rows=rng.choice([16, 32, 64]), n_keep=n_keep, n_first=first, n_last=min(n_keep - first, rng.choice([0, 1, 32, n_keep // 2])))
    elif case["kind"] == "bounds":
        case.update(new=0 if rng.random() < 0.4 else _log_int(rng, 1, min(256, case["len_min"])))
    else:
        pages = -(-longest // case["page_rows"])
        per_seq = min(case["len_min"], rng.choice([1, 1, 2, 3, 4, 8]))
        newest = (per_seq + case["page_rows"] - 2) // case["page_rows"] + 1
        case.update(q_per_seq=per_seq, n_select=newest + 1 + _log_int(rng, 1, max(1, min(pages, 256, 200000 // (n_seqs * case["page_rows"])))))
        if case["kind"] == "select":
            case.update(n_first=rng.choice([0, 1]), n_last=newest)
    return case


# ---- shapes -------------------------------------------------------------------------------------------------
def _shape(case):
    """Lengths of the sequences (all tokens, the new ones among them), the prefixes of the groups, and pages a sequence."""
    rng = random.Random(case["shape_seed"])
    if case["kind"] == "weights":
        prefix = [rng.randint(case["prefix_min"], case["prefix_max"]) for _ in range(case["n_groups"])]
        behind = [rng.randint(case["own_min"], case["own_max"]) for _ in range(case["n_groups"] * case["members"])]
        # (a step's new tokens are its own: they lie behind the prefix)
        lens = [prefix[s // case["members"]] + max(n, case["q_per_seq"]) for s, n in enumerate(behind)]
    else:
        prefix = None
        lens = [rng.randint(case["len_min"], case["len_max"]) for _ in range(case["n_seqs"])]
    return {"lens": lens, "prefix": prefix, "pages": -(-max(lens) // case["page_rows"])}


def work(case):
    hq, hkv, d = case["n_q_heads"], case["n_kv_heads"], case["head_dim"]
    s = _shape(case)
    lens, rows = s["lens"], case["page_rows"]
    if case["kind"] == "weights":
        nq, m = case["q_per_seq"], case["members"]
        # the pages of a prefix count once, a sequence's own once; every sequence has weights of its own, read where they go on
        keys = sum(s["prefix"]) + sum(n - s["prefix"][i // m] for i, n in enumerate(lens))
        pairs = sum(nq * n - nq * (nq - 1) / 2 for n in lens)
        q_rows = len(lens) * nq * hq
        return {"bytes": 2 * d * hkv * keys + 4 * hkv * sum(lens) * (2 if case["decay"] else 1) + (2 * d + 4) * q_rows, "flops": 2 * d * hq * pairs}
    if case["kind"] == "evict":
        kept = sum(min(n, case["n_keep"]) for n in lens)
        # the weights, the kept rows out of the one set of pages and into the other, their numbers and weights
        return {"bytes": hkv * (4 * sum(lens) + kept * (8 * d + 8)) + 8 * len(lens), "flops": hkv * sum(lens)}
    if case["kind"] == "bounds":
        new = [case["new"] or n for n in lens]
        touched = sum(-(-n // rows) - (n - c) // rows for n, c in zip(lens, new))
        again = sum((n - c) % rows > 0 for n, c in zip(lens, new))
        return {"bytes": hkv * (2 * d * sum(new) + (2 * d + 1) * (touched + again)), "flops": 2 * hkv * d * sum(new)}
    nq = case["q_per_seq"]
    pages = [-(-n // rows) for n in lens]
    if case["kind"] == "select":
        out = sum(min(n, case["n_select"]) for n in pages)
        return {"bytes": hkv * ((2 * d + 1) * sum(pages) + 8 * out) + 4 * sum(pages) + 2 * d * hq * nq * len(lens),
                "flops": 4 * d * hq * nq * sum(pages)}
    keys = sum(min(n, min(p, case["n_select"]) * rows) for n, p in zip(lens, pages))
    return {"bytes": 4 * d * hkv * keys + (4 * d + 4) * len(lens) * nq * hq, "flops": 4 * d * hq * nq * keys}


# ---- inputs -------------------------------------------------------------------------------------------------
def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    hq, hkv, d, rows = case["n_q_heads"], case["n_kv_heads"], case["head_dim"], case["page_rows"]

    def randn(*shape, dtype=torch.bfloat16, scale=1.0):
        return (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * scale).to(dtype)

    s = _shape(case)
    lens, pages, n_seqs = torch.tensor(s["lens"], device="cuda", dtype=torch.int32), s["pages"], len(s["lens"])
    members = case.get("members", 1)
    seqs = torch.arange(n_seqs, device="cuda")
    before = torch.zeros(n_seqs, device="cuda", dtype=torch.int64) if s["prefix"] is None else torch.tensor(s["prefix"], device="cuda").repeat_interleave(members)
    # the pool's pages are handed out in any order; those that lie wholly in a prefix are its group's first sequence's
    page = torch.arange(pages, device="cuda")[None, :]
    owner = torch.where((page + 1) * rows <= before[:, None], (seqs // members * members)[:, None], seqs[:, None])
    used = page * rows < lens[:, None]
    ids, where = torch.unique((owner * pages + page)[used], return_inverse=True)
    n_pages = len(ids) + 3
    table = torch.full((n_seqs, pages), -1, device="cuda", dtype=torch.int64)
    table[used] = torch.randperm(n_pages, generator=gen, device="cuda")[where]
    st = {"table": table.int(), "lens": lens, "k_pages": randn(n_pages, rows, hkv, d)}
    kind = case["kind"]
    if kind in ("evict", "attend"):
        st["v_pages"] = randn(n_pages, rows, hkv, d)
    if kind in ("weights", "select", "attend"):  # normed queries and keys: scores of a standard deviation of about two
        st["q"] = randn(n_seqs * case["q_per_seq"], hq, d, scale=2.0)
    if kind == "weights":
        # a page that a prefix ends in is a copy of its own for every other sequence of the group: the prefix's rows are the same in it
        split = (before[:, None] % rows > 0) & (page == before[:, None] // rows)  # [sequences, pages], one a sequence at most
        source = torch.where(split, table[seqs // members * members], 0).sum(1)[split.any(1)]
        shared = (torch.arange(rows, device="cuda")[None, :] < (before % rows)[split.any(1)][:, None])[:, :, None, None]
        st["k_pages"][table[split]] = torch.where(shared, st["k_pages"][source], st["k_pages"][table[split]])
        st["prefix"] = s["prefix"]
        st["lse"] = _log_sums(case, st)
        # what the steps before have left
        st["weights"] = randn(n_seqs, hkv, max(s["lens"]), dtype=torch.float32, scale=1.5).exp() * 0.01
    elif kind == "evict":
        w = randn(n_seqs, hkv, max(s["lens"]), dtype=torch.float32, scale=2.0).exp()
        # far from every query: weights that have come to nothing, and many that are alike
        few = torch.rand(w.shape, generator=gen, device="cuda")
        st["weights"] = torch.where(few < 0.1, 0.0, torch.where(few < 0.2, w.bfloat16().float(), w))
        kept = [min(n, case["n_keep"]) for n in s["lens"]]
        st["kept_pages"] = -(-max(kept) // case["to_rows"])
        ends = torch.arange(st["kept_pages"], device="cuda")[None, :] * case["to_rows"] < torch.tensor(kept, device="cuda")[:, None]
        n_to = int(ends.sum()) + 3
        to = torch.full(ends.shape, -1, device="cuda", dtype=torch.int64)
        to[ends] = torch.randperm(n_to, generator=gen, device="cuda")[: n_to - 3]
        st.update(to_table=to.int(), to_k=randn(n_to, case["to_rows"], hkv, d), to_v=randn(n_to, case["to_rows"], hkv, d))
        st["weights_out"] = torch.zeros((n_seqs, hkv, case["n_keep"]), device="cuda")
    elif kind in ("bounds", "select"):
        # bounds of every page as far as the call has not to find them
        st["codes"] = torch.zeros((n_pages, hkv, 2, d), device="cuda", dtype=torch.int8)
        st["exps"] = torch.zeros((n_pages, hkv), device="cuda", dtype=torch.int8)
        new = case.get("new", 0)
        st["from"] = lens - new if kind == "bounds" and new else torch.zeros_like(lens)
        if kind == "select" or new:
            of = {**st, "lens": lens if kind == "select" else st["from"], "from": torch.zeros_like(lens)}
            _bounds_plain(case, of, pages)
    else:
        # what a selection has left: the first page, the newest, and any others, in order
        held = -(-lens.long() // rows)
        newest = torch.div(lens.long() - case["q_per_seq"], rows, rounding_mode="floor")
        at = torch.arange(pages, device="cuda")
        rank = torch.rand((n_seqs, hkv, pages), generator=gen, device="cuda")
        rank = torch.where((at == 0) | (at >= newest[:, None])[:, None, :], 2.0, rank)
        rank = torch.where((at >= held[:, None])[:, None, :], -1.0, rank)
        st["selected"] = _heaviest(rank, torch.clamp(held, max=case["n_select"]), case["n_select"])
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    lens = _shape(case)["lens"]
    st.update(case=case, max_len=max(lens))
    if case["kind"] == "weights":
        st["behind"] = max(n - st["prefix"][i // case["members"]] for i, n in enumerate(lens))
    if own:
        st.update(_handles(case, st))
    return st


def _handles(case, st):
    """What a program keeps between the calls: descriptions of heads, cache and bounds, the outputs' memory, a workspace."""
    from paper_2409_15355_amd import binding as ba
    heads = ba.Heads(case["n_q_heads"], case["n_kv_heads"], case["head_dim"], 500000.0)
    # (keys alone are what bounds, selection and weights read)
    got = {"ba": ba, "heads": heads, "cache": ba.PagedCache(st["k_pages"], st.get("v_pages", st["k_pages"]), st["table"])}
    kind, n_seqs, hkv, nbytes = case["kind"], len(st["lens"]), case["n_kv_heads"], 0
    if kind == "weights":
        shared = case["prefix_max"] > 0
        got["cu_group"] = torch.arange(0, n_seqs + 1, case["members"]).int().numpy() if shared else None
        got["prefix_len"] = torch.tensor(st["prefix"]).int().numpy() if shared else None
        got["weights_now"] = torch.zeros_like(st["weights"])  # (places of tokens that a sequence has not are nobody's)
        nbytes = ba.ba_paged_key_weights_workspace_bytes(heads, n_seqs, case["q_per_seq"], st["max_len"], got["cu_group"], got["prefix_len"])
    elif kind == "evict":
        got["to"] = ba.PagedCache(st["to_k"], st["to_v"], st["to_table"])
        got["kept"] = torch.empty((n_seqs, hkv, case["n_keep"]), device="cuda", dtype=torch.int32)
        got["len_out"] = torch.empty_like(st["lens"])
        nbytes = ba.ba_paged_evict_workspace_bytes(heads, n_seqs, st["max_len"], case["n_keep"])
    elif kind in ("bounds", "select"):
        got["bounds"] = ba.PageBounds(st["codes"], st["exps"])
        if kind == "select":
            got["selected_out"] = torch.empty((n_seqs, hkv, case["n_select"]), device="cuda", dtype=torch.int32)
            got["scores_out"] = torch.empty((n_seqs, hkv, case["n_select"]), device="cuda")
            nbytes = ba.ba_page_select_workspace_bytes(heads, n_seqs, case["page_rows"], st["max_len"])
    else:
        got.update(o=torch.empty_like(st["q"]), lse=torch.empty(st["q"].shape[:2], device="cuda"))
        nbytes = ba.ba_paged_attention_selected_workspace_bytes(heads, n_seqs, case["q_per_seq"], case["page_rows"], st["max_len"], case["n_select"])
    got["ws"] = torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device="cuda")
    return got


# ---- one pass -----------------------------------------------------------------------------------------------
def run(st):
    return (_run_own if own else _run_plain)(st)


def _run_own(st):
    case, ba, kind = st["case"], st["ba"], st["case"]["kind"]
    if kind == "weights":
        ba.ba_paged_key_weights(st["heads"], st["cache"], st["q"], st["lse"], st["weights"], st["weights_now"], case["decay"], st["lens"],
                                st["max_len"], st["cu_group"], st["prefix_len"], case["q_per_seq"], st["ws"])
        return [st["weights_now"]]
    if kind == "evict":
        ba.ba_paged_evict(st["heads"], st["cache"], st["to"], st["weights"], st["lens"], st["max_len"], case["n_keep"], case["n_first"], case["n_last"],
                          st["kept"], st["weights_out"], st["len_out"], st["ws"])
        return [st["to_k"], st["to_v"], st["kept"], st["weights_out"], st["len_out"]]
    if kind == "bounds":
        ba.ba_page_bounds(st["heads"], st["cache"], st["bounds"], st["from"], st["lens"], st["max_len"])
        return [st["codes"], st["exps"]]
    if kind == "select":
        ba.ba_page_select(st["heads"], st["cache"], st["bounds"], st["q"], st["lens"], st["max_len"], st["selected_out"], st["scores_out"],
                          case["n_first"], case["n_last"], case["q_per_seq"], st["ws"])
        return [st["selected_out"], st["scores_out"]]
    ba.ba_paged_attention_selected(st["heads"], st["cache"], st["q"], st["o"], st["lse"], st["lens"], st["max_len"], st["selected"],
                                   case["q_per_seq"], st["ws"])
    return [st["o"], st["lse"]]


# ---- the plain forms ----------------------------------------------------------------------------------------
def _run_plain(st):
    return {"weights": _weights_plain, "evict": _evict_plain, "bounds": lambda c, s: _bounds_plain(c, s, _touched(c, s)), "select": _select_plain,
            "attend": _attend_plain}[st["case"]["kind"]](st["case"], st)


def _gathered(pages, table, at):
    """Rows `at` [n, keys] of the sequences whose pages `table` [n, pages] names, as [n, KV heads, keys, D]."""
    rows = pages.shape[1]
    page = table.long().gather(1, (at // rows).clamp(max=table.shape[1] - 1)).clamp(min=0)
    return pages[page, at % rows].float().transpose(1, 2).contiguous()


def _scores(case, st):
    """Masked scores of all rows with the prefixes' keys [groups, KV heads, members * tokens * heads, longest prefix] (None without one) and with
    the sequences' own [sequences, KV heads, tokens * heads, longest]."""
    hq, hkv, d, nq, m = case["n_q_heads"], case["n_kv_heads"], case["head_dim"], case["q_per_seq"], case["members"]
    n_seqs, n_groups, g = len(st["lens"]), case["n_groups"], hq // hkv
    prefix = torch.tensor(st["prefix"], device="cuda")
    behind = int((st["lens"].long() - prefix.repeat_interleave(m)).max()) if "behind" not in st else st["behind"]
    lens, before, longest = st["lens"].long(), prefix.repeat_interleave(m), max(st["prefix"])
    last = lens[:, None] - nq + torch.arange(nq, device="cuda")[None, :]  # the last key that a token sees
    q = st["q"].float().view(n_seqs, nq, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(n_seqs, hkv, nq * g, d) / math.sqrt(d)
    at = before[:, None] + torch.arange(behind, device="cuda")[None, :]
    k = _gathered(st["k_pages"], st["table"], at)
    mine = torch.matmul(q, k.transpose(2, 3).contiguous()).view(n_seqs, hkv, nq, g, behind)
    mine = mine.masked_fill((at[:, None, :] > last[:, :, None])[:, None, :, None, :], -math.inf).view(n_seqs, hkv, nq * g, behind)
    if not longest:
        return None, mine
    at = torch.arange(longest, device="cuda").expand(n_groups, -1)
    k = _gathered(st["k_pages"], st["table"][::m], at)
    q = q.view(n_groups, m, hkv, nq * g, d).transpose(1, 2).reshape(n_groups, hkv, m * nq * g, d)
    theirs = torch.matmul(q, k.transpose(2, 3).contiguous())
    return theirs.masked_fill((at >= prefix[:, None])[:, None, None, :], -math.inf), mine


def _as_rows(case, x):
    """[sequences, KV heads, tokens * heads] as the [tokens, query heads] of a log-sum-exp, or back."""
    hq, hkv, nq = case["n_q_heads"], case["n_kv_heads"], case["q_per_seq"]
    if x.dim() == 3:
        return x.view(-1, hkv, nq, hq // hkv).transpose(1, 2).reshape(-1, hq)
    return x.view(-1, nq, hkv, hq // hkv).transpose(1, 2).reshape(-1, hkv, nq * (hq // hkv))


def _by_group(case, x):
    """[sequences, KV heads, rows, ...] as [groups, KV heads, members * rows, ...]."""
    return x.view(case["n_groups"], case["members"], *x.shape[1:]).transpose(1, 2).flatten(2, 3)


def _log_sums(case, st):
    theirs, mine = _scores(case, st)
    sums = torch.logsumexp(mine, -1)
    if theirs is not None:
        more = torch.logsumexp(theirs, -1).view(case["n_groups"], case["n_kv_heads"], case["members"], -1).transpose(1, 2).reshape(sums.shape)
        sums = torch.logaddexp(sums, more)
    return _as_rows(case, sums).contiguous()


def _weights_plain(case, st):
    theirs, mine = _scores(case, st)
    m, hkv, n_groups = case["members"], case["n_kv_heads"], case["n_groups"]
    lse, prefix = _as_rows(case, st["lse"])[..., None], torch.tensor(st["prefix"], device="cuda")
    lens, before = st["lens"].long(), prefix.repeat_interleave(m)
    place = torch.arange(st["weights"].shape[2], device="cuda")[None, :]
    # of a sequence's own keys, put where they belong
    own_sums = torch.exp(mine - lse).sum(2)
    where = (place - before[:, None]).clamp(0, own_sums.shape[2] - 1)
    total = torch.where(((place >= before[:, None]) & (place < lens[:, None]))[:, None, :], own_sums.gather(2, where[:, None, :].expand(-1, hkv, -1)), 0.0)
    if theirs is not None:
        sums = torch.exp(theirs - _by_group(case, lse)).view(n_groups, hkv, m, -1, theirs.shape[-1]).sum(3).transpose(1, 2).flatten(0, 1)
        total[..., : sums.shape[-1]] += sums
    if case["decay"]:
        # new tokens have had no weight before
        total += torch.where((place < lens[:, None] - case["q_per_seq"])[:, None, :], case["decay"] * st["weights"], 0.0)
    return [total]


def _heaviest(x, n, width):
    """The places of the n [sequences] largest of x [sequences, heads, places], in order, -1 behind them; of equal ones the lowest places."""
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices[..., :width]
    at = torch.arange(order.shape[-1], device="cuda")
    order = torch.sort(torch.where(at < n[:, None, None], order, x.shape[-1]), dim=-1).values
    order = torch.where(at < n[:, None, None], order, -1)
    return torch.nn.functional.pad(order, (0, width - order.shape[-1]), value=-1).int()


def _evict_plain(case, st):
    lens, hkv = st["lens"].long(), case["n_kv_heads"]
    n = torch.clamp(lens, max=case["n_keep"])
    at = torch.arange(st["weights"].shape[2], device="cuda")
    held = (at < case["n_first"]) | (at >= lens[:, None] - case["n_last"])
    w = torch.where(held[:, None, :], math.inf, st["weights"])
    kept = _heaviest(torch.where((at < lens[:, None])[:, None, :], w, -math.inf), n, case["n_keep"])
    seq, head, to = torch.nonzero(kept >= 0, as_tuple=True)
    of = kept[seq, head, to].long()
    for pages, out in ((st["k_pages"], st["to_k"]), (st["v_pages"], st["to_v"])):
        rows = pages[st["table"][seq, of // case["page_rows"]].long(), of % case["page_rows"], head]
        out[st["to_table"][seq, to // case["to_rows"]].long(), to % case["to_rows"], head] = rows
    # (places behind the kept ones stay as they were)
    st["weights_out"][seq, head, to] = st["weights"][seq, head, of]
    return [st["to_k"], st["to_v"], kept, st["weights_out"], n.int()]


def _exponent(top):
    """The least e with top <= 127 * 2^e, within limits (an infinity's is the largest)."""
    m, e = torch.frexp(top)
    e = torch.where(m <= 127 / 128, e - 7, e - 6)
    return torch.where(top == 0, MIN_EXP, torch.where(torch.isinf(top), MAX_EXP, e)).clamp(MIN_EXP, MAX_EXP)


def _two_to(e):
    """2^e, exactly."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _touched(case, st):
    """Pages of a sequence that a call changes, at most."""
    return st["table"].shape[1] if not case["new"] else (case["new"] + case["page_rows"] - 2) // case["page_rows"] + 1


def _bounds_plain(case, st, width):
    rows, table = case["page_rows"], st["table"].long()
    since, lens = st["from"].long(), st["lens"].long()
    at = since[:, None] // rows + torch.arange(width, device="cuda")[None, :]  # pages of the sequences' [sequences, width]
    place = at[..., None] * rows + torch.arange(rows, device="cuda")
    new = (place >= since[:, None, None]) & (place < lens[:, None, None])
    live = new.any(-1)
    seq, i = torch.nonzero(live, as_tuple=True)
    page, new, fresh = table[seq, at[seq, i]], new[seq, i], at[seq, i] * rows >= since[seq]
    k = st["k_pages"][page].float()  # [pages, rows, KV heads, D]
    k = torch.where(torch.isnan(k), 0.0, k)
    new = new[:, :, None, None]
    e = _exponent(torch.where(new, k.abs(), 0.0).amax(dim=(1, 3)))
    old_e = torch.where(fresh[:, None], MIN_EXP, st["exps"][page].int())
    both = torch.maximum(e, old_e)
    scale, by = _two_to(-both)[..., None], _two_to(old_e - both)[..., None]
    hi = torch.ceil(torch.where(new, k, -math.inf).amax(1) * scale).clamp(-127, 127)
    lo = torch.floor(torch.where(new, k, math.inf).amin(1) * scale).clamp(-127, 127)
    old, fresh = st["codes"][page].float(), fresh[:, None, None]
    hi = torch.where(fresh, hi, torch.maximum(hi, torch.ceil(old[:, :, 0] * by)))
    lo = torch.where(fresh, lo, torch.minimum(lo, torch.floor(old[:, :, 1] * by)))
    st["codes"][page] = torch.stack([hi, lo], dim=2).to(torch.int8)
    st["exps"][page] = both.to(torch.int8)
    return [st["codes"], st["exps"]]


def _select_plain(case, st):
    hq, hkv, d, nq, rows = case["n_q_heads"], case["n_kv_heads"], case["head_dim"], case["q_per_seq"], case["page_rows"]
    n_seqs, n = len(st["lens"]), st["table"].shape[1]
    q = torch.where(torch.isnan(st["q"]), 0.0, st["q"].float())
    q = q.view(n_seqs, nq, hkv, hq // hkv, d).transpose(1, 2).reshape(n_seqs, hkv, nq * (hq // hkv), d)
    e = _exponent(q.abs().amax(-1))
    c = torch.round(q * _two_to(-e)[..., None]).clamp(-127, 127)  # (half to even)
    page = st["table"].long().clamp(min=0)
    codes = st["codes"][page].float().permute(0, 2, 3, 4, 1)  # [sequences, KV heads, 2, D, pages]
    dots = torch.matmul(c.clamp(min=0), codes[:, :, 0].contiguous()) + torch.matmul(c.clamp(max=0), codes[:, :, 1].contiguous())  # (whole numbers below 2^24)
    score = (dots * _two_to(e)[..., None]).amax(2) * _two_to(st["exps"][page]).transpose(1, 2)
    held, at = -(-st["lens"].long() // rows), torch.arange(n, device="cuda")
    newest = torch.div(st["lens"].long() - nq, rows, rounding_mode="floor")
    always = (at < case["n_first"]) | (at >= torch.minimum(held - case["n_last"], newest)[:, None])
    there = (at < held[:, None]) & (st["table"] >= 0)
    rank = torch.where(there[:, None, :], torch.where(always[:, None, :], math.inf, score), -math.inf)
    selected = _heaviest(rank, torch.clamp(there.sum(1), max=case["n_select"]), case["n_select"])
    return [selected, torch.where(selected >= 0, score.gather(2, selected.long().clamp(min=0)), -math.inf)]


def _attend_plain(case, st):
    hq, hkv, d, nq, rows = case["n_q_heads"], case["n_kv_heads"], case["head_dim"], case["q_per_seq"], case["page_rows"]
    n_seqs, g, sel = len(st["lens"]), hq // hkv, st["selected"].long()
    page = st["table"].long().gather(1, sel.clamp(min=0).flatten(1)).view(sel.shape).clamp(min=0)
    head, r = torch.arange(hkv, device="cuda")[None, :, None, None], torch.arange(rows, device="cuda")
    k, v = (x[page[..., None], r, head].float().flatten(2, 3) for x in (st["k_pages"], st["v_pages"]))  # [sequences, KV heads, keys, D]
    last = st["lens"].long()[:, None] - nq + torch.arange(nq, device="cuda")[None, :]
    place = torch.where(sel[..., None] >= 0, sel[..., None] * rows + r, 1 << 40).flatten(2)[:, :, None, :]
    q = st["q"].float().view(n_seqs, nq, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(n_seqs, hkv, nq * g, d) / math.sqrt(d)
    s = torch.matmul(q, k.transpose(2, 3).contiguous()).masked_fill(place > last.repeat_interleave(g, 1)[:, None, :, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    out, lse = torch.matmul(p, v) / total, top + torch.log(total)
    to_rows = lambda x: x.view(n_seqs, hkv, nq, g, -1).transpose(1, 2).reshape(n_seqs * nq, hq, -1)  # noqa: E731
    return [to_rows(out).bfloat16(), to_rows(lse).squeeze(-1)]


# ---- the same in 64 bits, one sequence after the other -------------------------------------------------------------
def _rows64(case, st, pool, s, n):
    """Keys or values of a sequence's first n tokens, [KV heads, n, D]."""
    pages = st["table"][s, : -(-n // case["page_rows"])].long()
    return pool[pages].flatten(0, 1)[:n].double().transpose(0, 1).contiguous()


def exact(case, seed):
    st = _inputs(case, seed)
    st["case"] = case
    return {"weights": _weights64, "evict": _evict64, "bounds": _bounds64, "select": _select64, "attend": _attend64}[case["kind"]](case, st)


def _weights64(case, st):
    hkv, d, nq = case["n_kv_heads"], case["head_dim"], case["q_per_seq"]
    g = case["n_q_heads"] // hkv
    lens = st["lens"].tolist()
    out = torch.zeros(st["weights"].shape, dtype=torch.float64, device="cuda")
    for s, n in enumerate(lens):
        k = _rows64(case, st, st["k_pages"], s, n)
        if case["decay"]:
            out[s, :, : n - nq] = st["weights"][s, :, : n - nq].double() * case["decay"]
        for i in range(0, nq, 32):  # some tokens at a time
            step = min(32, nq - i)
            q = st["q"][s * nq + i:s * nq + i + step].double().view(step, hkv, g, d)
            lse = st["lse"][s * nq + i:s * nq + i + step].double().view(step, hkv, g)
            for h in range(hkv):
                sc = (q[:, h].reshape(step * g, d) @ k[h].t().contiguous()).view(step, g, n) / math.sqrt(d) - lse[:, h, :, None]
                seen = torch.arange(n, device="cuda") <= n - nq + i + torch.arange(step, device="cuda")[:, None]
                out[s, h, :n] += (sc.exp() * seen[:, None, :]).sum(dim=(0, 1))
    return [out]


def _evict64(case, st):
    lens, keep, hkv = st["lens"].tolist(), case["n_keep"], case["n_kv_heads"]
    kept = torch.full((len(lens), hkv, keep), -1, dtype=torch.int32)
    w_out, k_out, v_out = st["weights_out"].double(), st["to_k"].double(), st["to_v"].double()
    for s, n in enumerate(lens):
        w = st["weights"][s, :, :n].cpu().numpy()
        to = torch.arange(min(n, keep), device="cuda")
        page, row = st["to_table"][s, to // case["to_rows"]].long(), to % case["to_rows"]
        k, v = _rows64(case, st, st["k_pages"], s, n), _rows64(case, st, st["v_pages"], s, n)
        for h in range(hkv):
            if n <= keep:
                mine = list(range(n))
            else:
                ends = list(range(case["n_first"])) + list(range(n - case["n_last"], n))
                middle = (-w[h, case["n_first"]:n - case["n_last"]]).argsort(kind="stable")[: keep - len(ends)] + case["n_first"]
                mine = sorted(ends + middle.tolist())
            kept[s, h, : len(mine)] = torch.tensor(mine, dtype=torch.int32)
            of = torch.tensor(mine, device="cuda")
            w_out[s, h, : len(mine)] = st["weights"][s, h, of].double()
            k_out[page, row, h], v_out[page, row, h] = k[h, of], v[h, of]
    return [k_out, v_out, kept.cuda(), w_out, torch.clamp(st["lens"], max=keep)]


def _exponent64(top):
    # (values of 8 bits: none is nearer to 127 * 2^e than 2^-8 of it without being it)
    return torch.where(top > 0, torch.ceil(torch.log2(torch.where(top > 0, top, 1.0) / 127) - 1e-6), MIN_EXP).clamp(MIN_EXP, MAX_EXP)


def _two_to64(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _codes64(x):
    """Keys [pages, rows, KV heads, D] in 64 bits: the codes of their bounds and the exponents."""
    e = _exponent64(x.abs().amax(dim=(1, 3)))
    scale = _two_to64(e)[..., None]
    return torch.clamp(torch.ceil(x.amax(1) / scale), -127, 127), torch.clamp(torch.floor(x.amin(1) / scale), -127, 127), e


def _bounds64(case, st):
    # (bounds of all rows that a page has: those that a call adds to and those that it finds are the same)
    codes, exps, rows = st["codes"].clone(), st["exps"].clone(), case["page_rows"]
    for s, n in enumerate(st["lens"].tolist()):
        since = int(st["from"][s])
        for first, last, full in ((since // rows, n // rows, True), (max(since // rows, n // rows), -(-n // rows), False)):
            if last <= first:
                continue
            page = st["table"][s, first:last].long()
            hi, lo, e = _codes64(st["k_pages"][page][:, : rows if full else n % rows].double())
            codes[page], exps[page] = torch.stack([hi, lo], dim=2).to(torch.int8), e.to(torch.int8)
    return [codes, exps]


def _select64(case, st):
    hkv, d, nq, rows = case["n_kv_heads"], case["head_dim"], case["q_per_seq"], case["page_rows"]
    g = case["n_q_heads"] // hkv
    out = torch.full((len(st["lens"]), hkv, case["n_select"]), -1, dtype=torch.int32)
    of = torch.full(out.shape, -math.inf, dtype=torch.float64)
    for s, n in enumerate(st["lens"].tolist()):
        pages = -(-n // rows)
        page = st["table"][s, :pages].long()
        hi, lo = ((st["codes"][page, :, i].double() * _two_to64(st["exps"][page])[..., None]).transpose(0, 1) for i in range(2))
        q = st["q"][s * nq:(s + 1) * nq].double().view(nq, hkv, g, d).transpose(0, 1).reshape(hkv, nq * g, d)
        step = _two_to64(_exponent64(q.abs().amax(-1)))[..., None]
        q = torch.clamp(torch.round(q / step), -127, 127) * step
        score = torch.stack([torch.maximum(q[:, r, None] * hi, q[:, r, None] * lo).sum(-1) for r in range(nq * g)]).amax(0).cpu().numpy()
        always = [i for i in range(pages) if i < case["n_first"] or i >= pages - case["n_last"] or (i + 1) * rows > n - nq]
        held = set(always)
        for h in range(hkv):
            others = [i for i in (-score[h]).argsort(kind="stable").tolist() if i not in held]
            mine = sorted((always + others)[: min(pages, case["n_select"])])
            out[s, h, : len(mine)] = torch.tensor(mine, dtype=torch.int32)
            of[s, h, : len(mine)] = torch.from_numpy(score[h, mine])
    return [out.cuda(), of.cuda()]


def _attend64(case, st):
    hkv, d, nq, rows = case["n_kv_heads"], case["head_dim"], case["q_per_seq"], case["page_rows"]
    g = case["n_q_heads"] // hkv
    lens = st["lens"].tolist()
    out = torch.empty((len(lens), nq, hkv, g, d), dtype=torch.float64, device="cuda")
    lse = torch.empty((len(lens), nq, hkv, g), dtype=torch.float64, device="cuda")
    q = st["q"].double().view(len(lens), nq, hkv, g, d)
    lists = st["selected"].cpu()
    for s, n in enumerate(lens):
        for h in range(hkv):
            mine = lists[s, h][lists[s, h] >= 0].long().cuda()
            place = (mine[:, None] * rows + torch.arange(rows, device="cuda")).flatten()
            page = st["table"][s, mine].long()
            k, v = (x[page, :, h].flatten(0, 1).double() for x in (st["k_pages"], st["v_pages"]))
            sc = (q[s, :, h].reshape(nq * g, d) @ k.t().contiguous()).view(nq, g, -1) / math.sqrt(d)
            sc = sc.masked_fill((place > n - nq + torch.arange(nq, device="cuda")[:, None])[:, None, :], -math.inf)
            norm = torch.logsumexp(sc, dim=-1)
            out[s, :, h] = torch.exp(sc - norm[..., None]) @ v
            lse[s, :, h] = norm
    return [out.reshape(-1, hkv * g, d), lse.reshape(-1, hkv * g)]
