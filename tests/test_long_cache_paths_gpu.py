"""Long paged caches on the paths that only larger calls take: pages scored apart from the choice among them by more query rows than a product has; groups and
questions of more rows than a workgroup notes at a time; eviction past the caches.  Checks and tolerances are those of test_long_cache_gpu.py."""
import pytest

import test_long_cache_gpu as forms
from test_long_cache_gpu import ba, ints  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv,d,rows,lens,nq,n_select,first,last", [
    (16, 2, 64, 16, [5000, 4200], 5, 40, 1, 2), (6, 2, 128, 4, [5000], 7, 100, 3, 1), (8, 1, 64, 1, [300, 0, 290], 1, 20, 0, 0), (17, 1, 128, 2, [600, 9], 1, 70, 0, 5)])
def test_selection_out_of_many_pages(ba, hq, hkv, d, rows, lens, nq, n_select, first, last):  # noqa: F811
    forms.test_page_select(ba, hq, hkv, d, rows, lens, nq, n_select, first, last)


@pytest.mark.parametrize("hq,hkv,d,rows,nq,members,prefix,behind", [
    (8, 2, 64, 16, 1, [140], [130], [1 + i % 7 for i in range(140)]), (8, 1, 128, 16, 3, [30], [200], [3 + i % 9 for i in range(30)]),
    (5, 1, 64, 7, 1, [2, 70], [20, 90], [1 + i % 11 for i in range(72)]),                                                                # few rows a sequence
    (16, 2, 64, 16, 40, [5], [300], [40, 41, 70, 2, 300]), (12, 2, 128, 16, 50, [4], [100], [50, 60, 55, 300])])                         # many
def test_key_weights_of_large_groups(ba, hq, hkv, d, rows, nq, members, prefix, behind):  # noqa: F811
    forms.test_key_weights_over_shared_prefixes(ba, hq, hkv, d, rows, nq, members, prefix, behind)


@pytest.mark.parametrize("hq,hkv,d,rows,lens,nq", [(16, 2, 64, 16, [1100], 1040), (9, 3, 64, 16, [900, 40], 700)])
def test_key_weights_of_long_questions(ba, hq, hkv, d, rows, lens, nq):  # noqa: F811
    forms.test_key_weights(ba, hq, hkv, d, rows, lens, nq, 0.5)


@pytest.mark.parametrize("hq,d,members,prefix", [(32, 64, 140, 8400), (24, 128, 70, 8321), (32, 64, 9, 1000)])
def test_key_weights_of_many_answers_on_a_long_prefix(ba, hq, d, members, prefix):  # noqa: F811
    """More rows than a workgroup notes at a time; with old weights, and in parts of a group's sequences."""
    import torch
    hkv, rows = 8, 16
    g, pages = hq // hkv, -(-prefix // rows)
    gen = torch.Generator(device="cuda").manual_seed(3)
    kp = torch.randn((pages + members, rows, hkv, d), generator=gen, device="cuda").bfloat16()
    order = torch.randperm(pages + members, generator=gen, device="cuda")
    table = order[:pages].expand(members, pages).clone()
    table = torch.cat([table, order[pages:, None]], 1)
    lens = [pages * rows + 1 + s % rows for s in range(members)]
    n = pages * rows + rows
    q = (torch.randn((members, hq, d), generator=gen, device="cuda") * 2).bfloat16()
    old = torch.rand((members, hkv, n), generator=gen, device="cuda")
    shared, own = kp[order[:pages]].double().view(-1, hkv, d), kp[order[pages:]].double()
    lse = torch.empty((members, hq), device="cuda")
    want, off = torch.zeros((2, members, hkv, n), dtype=torch.float64, device="cuda")
    scale, u = d ** -0.5, forms.U
    for h in range(hkv):
        qh = q[:, h * g:(h + 1) * g].double()
        sizes, scores = [], []
        for f in (lambda x: x, torch.abs):
            first = (f(qh).reshape(-1, d) @ f(shared[:, h]).T).view(members, g, -1)
            last = (f(qh)[:, :, None] * f(own[:, None, :, h])).sum(-1)
            (sizes if f is torch.abs else scores).append(torch.cat([first, last], 2) * scale)
        s, size = scores[0], sizes[0]
        for m, x in enumerate(lens):
            s[m, :, x:] = -float("inf")
        lse[:, h * g:(h + 1) * g] = s.logsumexp(-1).float()
        l = lse[:, h * g:(h + 1) * g, None].double()
        p = (s - l).exp()
        want[:, h] = p.sum(1)
        off[:, h] = (p * (d * u * size + (s.abs().nan_to_num(posinf=0.0) + l.abs() + 4 + g) * u)).sum(1)
    out = torch.full((members, hkv, n), -7.0, device="cuda")
    heads, cache = ba.Heads(hq, hkv, d), ba.PagedCache(kp, kp, table.int())
    ba.ba_paged_key_weights(heads, cache, q, lse, old, out, 0.5, ints(lens), n, [0, members], [prefix], 1)
    for m, x in enumerate(lens):
        want[m, :, : x - 1] += 0.5 * old[m, :, : x - 1].double()
        off[m, :, : x - 1] += 2 * u * want[m, :, : x - 1]
        assert bool((out[m, :, x:] == -7).all()), m
        assert bool(((out[m, :, :x].double() - want[m, :, :x]).abs() <= off[m, :, :x] + 1e-37).all()), m


@pytest.mark.parametrize("hq,hkv,d,nq", [(32, 8, 64, 1), (40, 8, 64, 1), (16, 8, 128, 7)])
def test_key_weights_of_groups_of_unequal_prefixes(ba, hq, hkv, d, nq):  # noqa: F811
    """Sequences that go on far behind a short prefix beside others that end behind a long one."""
    import torch
    members, prefix, rows = [32, 34], [1200, 90], 16
    g, n_seqs, scale, u = hq // hkv, sum(members), d ** -0.5, forms.U
    lens = [1200 + nq + s % 40 for s in range(32)] + [90 + nq + (s * 331) % 1100 for s in range(34)]
    n, pages = max(lens), -(-max(lens) // rows)
    gen = torch.Generator(device="cuda").manual_seed(9)
    kp = torch.randn((n_seqs * pages, rows, hkv, d), generator=gen, device="cuda").bfloat16()
    table = torch.randperm(n_seqs * pages, generator=gen, device="cuda").view(n_seqs, pages)
    table[:32, : 1200 // rows] = table[0, : 1200 // rows].clone()
    table[32:, : 90 // rows] = table[32, : 90 // rows].clone()
    for s in range(33, n_seqs):  # (the page that the prefix ends in: a copy of its part)
        kp[table[s, 5], :10] = kp[table[32, 5], :10]
    q = (torch.randn((n_seqs * nq, hq, d), generator=gen, device="cuda") * 2).bfloat16()
    old = torch.rand((n_seqs, hkv, n), generator=gen, device="cuda")
    lse, out = torch.empty((n_seqs * nq, hq), device="cuda"), torch.full((n_seqs, hkv, n), -7.0, device="cuda")
    want, off = [], []
    for s, m in enumerate(lens):
        k = kp[table[s]].double().view(-1, hkv, d)[:m].permute(1, 2, 0).contiguous()  # [heads, D, keys]
        r = q[s * nq:(s + 1) * nq].double().view(nq, hkv, g, d).transpose(0, 1).reshape(hkv, nq * g, d)
        x, size = torch.stack([r[h] @ k[h] for h in range(hkv)]) * scale, torch.stack([r[h].abs() @ k[h].abs() for h in range(hkv)]) * scale
        seen = torch.arange(m, device="cuda") <= (m - nq + torch.arange(nq, device="cuda"))[:, None]
        x = x.masked_fill(~seen.repeat_interleave(g, 0), -float("inf"))
        l = x.logsumexp(-1).float()
        lse[s * nq:(s + 1) * nq] = l.view(hkv, nq, g).transpose(0, 1).reshape(nq, hq)
        p = (x - l.double()[..., None]).exp()
        w, e = p.sum(1), (p * (d * u * size + (x.abs().nan_to_num(posinf=0.0) + l.abs().double()[..., None] + 4 + nq * g) * u)).sum(1)
        w[:, : m - nq] += 0.5 * old[s, :, : m - nq].double()
        want.append(w), off.append(e + 2 * u * w)
    cache = ba.PagedCache(kp, kp, table.int())
    ba.ba_paged_key_weights(ba.Heads(hq, hkv, d), cache, q, lse, old, out, 0.5, ints(lens), n, [0, 32, 66], prefix, nq)
    for s, m in enumerate(lens):
        assert bool((out[s, :, m:] == -7).all()) and bool(((out[s, :, :m].double() - want[s]).abs() <= off[s] + 1e-37).all()), s


@pytest.mark.parametrize("d,keep,n_seqs", [(128, 512, 64), (64, 1024, 64), (64, 64, 70), (128, 128, 40)])
def test_eviction_of_many_lists(ba, d, keep, n_seqs):  # noqa: F811
    """A quarter of a gigabyte and more that goes past the caches, or short lists in one launch: every row at its place, and none beside."""
    import torch
    hkv, rows, to_rows = 8, 16, 32
    lens = [keep + 1 + s % 50 for s in range(n_seqs)]
    n, pages, to_pages = max(lens), -(-max(lens) // rows), keep // to_rows
    gen = torch.Generator(device="cuda").manual_seed(1)
    kp, vp = (torch.randn((n_seqs * pages, rows, hkv, d), generator=gen, device="cuda").bfloat16() for _ in range(2))
    to_k, to_v = (torch.full((n_seqs * to_pages + 1, to_rows, hkv, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    old, new = torch.randperm(n_seqs * pages, generator=gen, device="cuda").view(n_seqs, pages), torch.randperm(n_seqs * to_pages, generator=gen, device="cuda").view(n_seqs, to_pages)
    w = torch.randperm(n_seqs * hkv * n, generator=gen, device="cuda").float().view(n_seqs, hkv, n)  # (below 2^24: no two alike)
    kept = torch.empty((n_seqs, hkv, keep), dtype=torch.int32, device="cuda")
    ba.ba_paged_evict(ba.Heads(hkv, hkv, d), ba.PagedCache(kp, vp, old.int()), ba.PagedCache(to_k, to_v, new.int()), w, ints(lens), n, keep, 0, 0, kept)
    for s, m in enumerate(lens):
        w[s, :, m:] = -1.0
    want = w.topk(keep).indices.sort().values
    assert torch.equal(kept.long(), want)
    j, head = torch.arange(keep, device="cuda"), torch.arange(hkv, device="cuda")[:, None]
    for s in range(n_seqs):
        for pool, to in ((kp, to_k), (vp, to_v)):
            assert torch.equal(to[new[s][j // to_rows], j % to_rows].transpose(0, 1), pool[old[s][want[s] // rows], want[s] % rows, head]), s
    assert bool((to_k[-1] == 7).all()) and bool((to_v[-1] == 7).all())
