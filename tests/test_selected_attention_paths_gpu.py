"""Attention over selected pages on the paths of its larger calls: rows that go past the caches, work items whose part of the list fills its place in LDS, or that take
as many keys as one may.  Sequences share the pages of one pool, each in an order of its own.  Tolerances as in test_long_cache_gpu.py."""
import numpy as np
import pytest

from test_long_cache_gpu import BF16_STEP, U, ba, ints, rand  # noqa: F401

pytestmark = pytest.mark.gpu

BIG = 1 << 30


def attend64(q, keys, values, seen, scale):
    """[rows, D], [tokens, D] twice, [rows, tokens] in 64 bits: outputs, log-sum-exps, sum p |v|, how far the log-sum-exps may be off."""
    s = (q @ keys.T * scale).masked_fill(~seen, -float("inf"))
    lse = s.logsumexp(-1)
    p = (s - lse[:, None]).exp().nan_to_num(0.0)  # (rows that see nothing: zero)
    most = s.abs().masked_fill(~seen, 0.0).amax(-1)
    size = (q.abs() @ keys.abs().T * scale).masked_fill(~seen, 0.0).amax(-1)
    off = q.shape[1] * U * size + (2 * most + seen.sum(-1) + 8) * U
    return p @ values, lse, p @ values.abs(), off


def case(ba, seed, hq, hkv, d, rows, lens, nq, n_select, max_len, parts=None):  # noqa: F811
    """parts: (how many parts, keys of a part) that the call is expected to be cut into."""
    import torch
    heads, n, g = ba.Heads(hq, hkv, d), len(lens), hq // hkv
    gen = torch.Generator(device="cuda").manual_seed(seed)
    pages = -(-max_len // rows)
    n_pages = pages + 3
    kp, vp = (torch.randn((n_pages, rows, hkv, d), generator=gen, device="cuda").bfloat16() for _ in range(2))
    kp[-1], vp[-1] = float("nan"), float("inf")  # (nobody's)
    table = torch.stack([torch.randperm(n_pages - 1, generator=gen, device="cuda")[:pages] for _ in range(n)])
    sel = np.full((n, hkv, n_select), -1, dtype=np.int64)
    rng = np.random.default_rng(seed)
    cut = np.zeros((n, hkv), dtype=np.int64)  # entries that count
    for s, m in enumerate(lens):
        held = -(-m // rows)
        for h in range(hkv):
            mine = np.sort(rng.permutation(held)[:n_select])
            cut[s, h] = len(mine)
            sel[s, h, :len(mine)] = mine
            if len(mine) > 4 and (s + h) % 3 == 0:  # ends early: an entry that is not above the one in front of it, with others behind it
                cut[s, h] = len(mine) // 2
                sel[s, h, cut[s, h]] = sel[s, h, cut[s, h] - 1] - (s % 2)
        if held > 2 and s % 2:
            table[s, held // 2], table[s, 1] = [-1, n_pages, BIG][s % 3], -7  # pages that are not there
    q = rand(seed + 1, n * nq, hq, d, scale=2.0)
    cache = ba.PagedCache(kp, vp, table.int())
    nbytes = ba.ba_paged_attention_selected_workspace_bytes(heads, n, nq, rows, max_len, n_select)
    if parts is not None:
        up = lambda x: -(-x // 256) * 256  # noqa: E731
        assert -(-min(n_select * rows, max_len) // parts[1]) == parts[0]
        assert nbytes == (0 if parts[0] == 1 else up(n * nq * hq * parts[0] * d * 2) + up(n * nq * hq * parts[0] * 16))
    results = []
    for _ in range(2):
        ws = torch.full((max(256, nbytes),), 255, dtype=torch.uint8, device="cuda")
        o, lse = torch.full_like(q, float("nan")), torch.full(q.shape[:2], float("nan"), device="cuda")
        ba.ba_paged_attention_selected(heads, cache, q, o, lse, ints(lens), max_len, ints(sel), nq, ws)
        results.append((o, lse))
    (o, lse), again = results
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1])  # the same call, the same bits
    at = torch.arange(rows, device="cuda")
    for s, m in enumerate(lens):
        for h in range(hkv):
            mine = torch.from_numpy(sel[s, h, :cut[s, h]]).cuda()
            ids = table[s, mine]
            there = (ids >= 0) & (ids < n_pages)
            tokens = (mine[there, None] * rows + at).flatten()
            k, v = (x[ids[there], :, h].reshape(-1, d).double() for x in (kp, vp))
            r = q[s * nq:(s + 1) * nq, h * g:(h + 1) * g].reshape(-1, d).double()
            seen = (tokens[None] <= (m - nq + torch.arange(nq, device="cuda"))[:, None]).repeat_interleave(g, 0)
            if seen.shape[1] == 0:
                k, v, seen = torch.zeros((1, d), dtype=torch.float64, device="cuda"), torch.zeros((1, d), dtype=torch.float64, device="cuda"), seen.new_zeros((nq * g, 1))
            out, l64, size, off = attend64(r, k, v, seen, d ** -0.5)
            got = o[s * nq:(s + 1) * nq, h * g:(h + 1) * g].reshape(-1, d).double()
            tol = (BF16_STEP + 2.0 ** -11 + 2 * off[:, None]) * size + BF16_STEP * (out.abs() + (BF16_STEP + 2.0 ** -11) * size) + 1e-30
            assert bool(((got - out).abs() <= tol).all()), (s, h, float(((got - out).abs() / tol).max()))
            l = lse[s * nq:(s + 1) * nq, h * g:(h + 1) * g].reshape(-1).double()
            fine = l64 > -float("inf")
            assert torch.equal(l > -float("inf"), fine) and bool(((l - l64).abs()[fine] <= off[fine]).all()), (s, h)


@pytest.mark.parametrize("rows,nq", [(16, 1), (20, 1), (64, 7), (7, 7), (16, 9), (33, 9), (128, 40)])
def test_selected_rows_past_the_caches(ba, rows, nq):  # noqa: F811
    """By the bound on the lists: 96 MB of keys and values and more.  Most sequences are short, one is as long as the bound."""
    max_len = 3000
    n_select = -(-max_len // rows)
    assert 16 * min(max_len, n_select * rows) * 8 * 128 * 4 > 1.5 * 96 * 2 ** 20
    case(ba, 500 + nq, 32, 8, 128, rows, [0, 1, nq, 17, 900, 33] + [50 + 13 * i for i in range(9)] + [max_len], nq, n_select, max_len)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("nq", [1, 9])
def test_selected_lists_that_fill_their_place(ba, nq, d):  # noqa: F811
    """Pages of one row: 1,152 entries of the list and of the page table a work item, the most that it has room for."""
    case(ba, 520 + nq, 32, 8, d, 1, [2304] * 6 + [2303, 1153, 1152, 1151, 5, 0, 2000, 1, 1300, 2304], nq, 2304, 2304, parts=(2, 1152))


@pytest.mark.parametrize("rows,nq", [(16, 1), (64, 1), (16, 9)])
def test_selected_keys_of_the_longest_parts(ba, rows, nq):  # noqa: F811
    """4,096 keys a work item, every row in one part."""
    case(ba, 540 + nq, 32, 8, 128, rows, [4096] * 20 + [4095, 4000, 2049, 17, 0, 1, 3000, 2048, 100, 4096, 4090, 64], nq, 4096 // rows, 4096, parts=(1, 4096))
