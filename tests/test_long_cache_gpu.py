"""Weights of cached keys, eviction by them, bounds of pages, selection by them and attention over the selected pages, against plain
implementations in 64 bits.  Tolerances follow from the arithmetic and are set ahead of any run, with u = 2^-24:
  a score is a sum of D products in 32 bits, off by D u sum |q k| scale at most; its exponential by that and by (|s| + |lse| + 4) u (the
  scaling by log2(e), the power of two), relative to itself; a sum of n such terms by n u of the sum.  Attention rounds its probabilities to bf16 once, its
  parts to fp16 once, its result to bf16 once.  Everything else here is whole numbers, or copies, and has to be equal."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16_STEP = 2.0 ** -8


@pytest.fixture(scope="module")
def ba():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2409_15355_amd import binding
    binding.load()
    return binding


def rand(seed, *shape, scale=1.0):
    import torch
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).bfloat16().cuda()


def f64(t):
    return t.detach().double().cpu().numpy()


def ints(x):
    import torch
    return torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


class Pool:
    """Sequences of tokens in shuffled pages; every row that is nobody's, keys and values, is NaN."""

    def __init__(self, ba, seed, lens, hkv, d, rows, extra=2, padded=False, prefix=0):
        import torch
        rng = np.random.default_rng(seed)
        self.lens, self.rows, self.hkv, self.d = list(lens), rows, hkv, d
        pages = max(1, max(-(-n // rows) for n in lens))
        n_pages = sum(-(-n // rows) for n in lens) + extra
        order = rng.permutation(n_pages)
        self.table = np.full((len(lens), pages), -1, dtype=np.int64)
        self.k, self.v = (rng.standard_normal((len(lens), pages * rows, hkv, d)).astype(np.float32) for _ in range(2))
        if prefix:  # all sequences begin alike
            self.k[:, :prefix], self.v[:, :prefix] = self.k[:1, :prefix], self.v[:1, :prefix]
        at = 0
        shape = (n_pages, rows + 3, hkv + 1, d + 8) if padded else (n_pages, rows, hkv, d)  # (rows, heads and pages further apart)
        pool = [torch.full(shape, float("nan"), dtype=torch.bfloat16)[:, :rows, :hkv, :d] for _ in range(2)]
        for s, n in enumerate(lens):
            for i in range(-(-n // rows)):
                self.table[s, i] = order[at]
                m = min(rows, n - i * rows)
                for x, p in ((self.k, pool[0]), (self.v, pool[1])):
                    p[order[at], :m] = torch.from_numpy(x[s, i * rows:i * rows + m]).bfloat16()
                at += 1
        def move(p):
            if not padded:
                return p.cuda()
            whole = torch.full(shape, float("nan"), dtype=torch.bfloat16, device="cuda")
            whole[:, :rows, :hkv, :d] = p.cuda()
            return whole[:, :rows, :hkv, :d]
        self.kp, self.vp = move(pool[0]), move(pool[1])
        self.k, self.v = (torch.from_numpy(x).bfloat16().double().numpy() for x in (self.k, self.v))
        self.cache = ba.PagedCache(self.kp, self.vp, ints(self.table))
        self.max_len = max(lens)


def p_of(pool, s, nq, i):
    return pool.lens[s] - nq + i


def lse64(pool, q, nq, scale, seen=None):
    """[tokens, heads] log-sum-exps of the keys that a row sees (seen(s, g, t): which of those)."""
    hq = q.shape[1]
    g = hq // pool.hkv
    out = np.full(q.shape[:2], -np.inf)
    for s in range(len(pool.lens)):
        for i in range(nq):
            n = p_of(pool, s, nq, i) + 1
            if n <= 0:
                continue
            for h in range(hq):
                sc = pool.k[s, :n, h // g] @ q[s * nq + i, h] * scale
                m = sc.max()
                out[s * nq + i, h] = m + np.log(np.exp(sc - m).sum())
    return out


def weights64(pool, q, lse, nq, scale, holes=()):
    """New weights [sequences, KV heads, tokens], and how far 32 bits may be off."""
    hq = q.shape[1]
    g = hq // pool.hkv
    w = np.zeros((len(pool.lens), pool.hkv, pool.max_len))
    err = np.zeros_like(w)
    for s in range(len(pool.lens)):
        for i in range(nq):
            n = p_of(pool, s, nq, i) + 1
            if n <= 0:
                continue
            for h in range(hq):
                l = lse[s * nq + i, h]
                if l == -np.inf:
                    continue
                k = pool.k[s, :n, h // g]
                sc = k @ q[s * nq + i, h] * scale
                size = np.abs(k) @ np.abs(q[s * nq + i, h]) * scale
                p = np.exp(sc - l)
                w[s, h // g, :n] += p
                err[s, h // g, :n] += p * (pool.d * U * size + (np.abs(sc) + abs(l) + 4 + nq * g) * U)
    for s, i in holes:
        w[s, :, i * pool.rows:(i + 1) * pool.rows] = 0
    return w, err


# ---- weights of cached keys -----------------------------------------------------------------------------------------
@pytest.mark.parametrize("hq,hkv,d,rows,lens,nq", [
    (4, 4, 64, 16, [1], 1), (32, 8, 128, 16, [2064], 1), (8, 2, 64, 7, [0, 1, 130, 129, 33], 1), (6, 2, 128, 64, [300, 5], 1), (16, 2, 64, 32, [257, 100, 3], 1),
    (8, 2, 128, 16, [70, 3, 0, 40], 5), (5, 1, 64, 1, [90, 31], 3), (8, 8, 64, 128, [200, 130], 33), (32, 8, 128, 16, [400], 64), (4, 1, 128, 100, [513, 1], 16), (16, 2, 128, 16, [300, 150], 100), (12, 2, 64, 16, [290], 150)])
@pytest.mark.parametrize("decay", [0.0, 1.0, 0.75])
def test_key_weights(ba, hq, hkv, d, rows, lens, nq, decay):
    import torch
    pool, heads = Pool(ba, 1, lens, hkv, d, rows, padded=rows == 7), ba.Heads(hq, hkv, d)
    scale = 1 / math.sqrt(d)
    q = rand(2, len(lens) * nq, hq, d, scale=2.0)
    lse = torch.from_numpy(lse64(pool, f64(q), nq, scale)).float().cuda()
    old = torch.rand((len(lens), hkv, pool.max_len + 3), generator=torch.Generator().manual_seed(3)).cuda()
    for s, n in enumerate(lens):  # (nothing is read there)
        old[s, :, max(0, n - nq):] = float("nan")
    out = torch.full_like(old, -7.0)
    ws = torch.empty(max(256, ba.ba_paged_key_weights_workspace_bytes(heads, len(lens), nq, pool.max_len)), dtype=torch.uint8, device="cuda")
    ba.ba_paged_key_weights(heads, pool.cache, q, lse, old, out, decay, ints(lens), pool.max_len, None, None, nq, ws)
    w, err = weights64(pool, f64(q), f64(lse), nq, scale)
    before = np.nan_to_num(f64(old)) * decay
    got = f64(out)
    for s, n in enumerate(lens):
        want, tol = w[s, :, :n].copy(), err[s, :, :n].copy()
        m = max(0, n - nq)
        want[:, :m] += before[s, :, :m]
        tol[:, :m] += 2 * U * (before[s, :, :m] + w[s, :, :m])
        assert (np.abs(got[s, :, :n] - want) <= tol + 1e-37).all(), (s, float((np.abs(got[s, :, :n] - want) / (tol + 1e-37)).max()))
        assert (got[s, :, n:] == -7.0).all()
    again = old.clone()  # in place, the same bits
    ba.ba_paged_key_weights(heads, pool.cache, q, lse, again, again, decay, ints(lens), pool.max_len, None, None, nq, ws)
    for s, n in enumerate(lens):
        assert torch.equal(again[s, :, :n], out[s, :, :n])
        assert torch.equal(again[s, :, n:].isnan(), old[s, :, n:].isnan())
    if decay == 0:
        first = torch.full_like(old, -7.0)
        ba.ba_paged_key_weights(heads, pool.cache, q, lse, None, first, 1.0, ints(lens), pool.max_len, None, None, nq, ws)
        assert torch.equal(first, out)


@pytest.mark.parametrize("hq,hkv,d,rows,nq,members,prefix,behind", [
    (32, 8, 128, 16, 1, [3], [160], [5, 1, 300]), (8, 2, 64, 7, 2, [2, 3], [30, 100], [9, 2, 40, 2, 3]), (6, 2, 128, 64, 1, [1, 4, 0, 2], [20, 129, 5, 0], [3, 1, 70, 5, 2, 9, 4]),
    (16, 2, 64, 16, 3, [9], [500], [3, 4, 5, 6, 7, 8, 9, 10, 300])])
def test_key_weights_over_shared_prefixes(ba, hq, hkv, d, rows, nq, members, prefix, behind):
    import torch
    before = np.repeat(prefix, members)
    lens = [int(a + b) for a, b in zip(before, behind)]
    pool, heads = Pool(ba, 11, lens, hkv, d, rows), ba.Heads(hq, hkv, d, softmax_scale=0.2)
    first = np.repeat(np.concatenate([[0], np.cumsum(members)])[:-1], members)
    for s, n in enumerate(before):  # the same tokens; the group's first sequence has them, the others' copies are not looked at
        pool.k[s, :n] = pool.k[first[s], :n]
        for i in range(n // rows):
            if first[s] != s:
                pool.table[s, i] = -5
        if n % rows and first[s] != s:
            pool.kp[pool.table[s, n // rows], : n % rows] = float("nan")
    cache = ba.PagedCache(pool.kp, pool.vp, ints(pool.table))
    q = rand(12, len(lens) * nq, hq, d, scale=2.0)
    lse = torch.from_numpy(lse64(pool, f64(q), nq, 0.2)).float().cuda()
    out = torch.full((len(lens), hkv, pool.max_len), -7.0, device="cuda")
    cu = np.concatenate([[0], np.cumsum(members)]).astype(np.int32)
    ws = torch.empty(max(256, ba.ba_paged_key_weights_workspace_bytes(heads, len(lens), nq, pool.max_len, cu, prefix)), dtype=torch.uint8, device="cuda")
    ba.ba_paged_key_weights(heads, cache, q, lse, None, out, 0.0, ints(lens), pool.max_len, cu, prefix, nq, ws)
    w, err = weights64(pool, f64(q), f64(lse), nq, 0.2)
    for s, n in enumerate(lens):
        assert (np.abs(f64(out)[s, :, :n] - w[s, :, :n]) <= err[s, :, :n] + 1e-37).all(), s
        assert (f64(out)[s, :, n:] == -7.0).all()


def test_key_weights_where_rows_see_nothing_and_pages_are_missing(ba):
    import torch
    lens, nq, rows = [40, 3, 100], 4, 16
    pool, heads = Pool(ba, 21, lens, 2, 64, rows), ba.Heads(8, 2, 64)
    q = rand(22, 12, 8, 64)
    lse = lse64(pool, f64(q), nq, 0.125)
    lse[1], lse[9, 3] = -np.inf, -np.inf  # (and token 0 of sequence 1 lies before its beginning)
    pool.table[2, 1], pool.table[0, 0] = 10 ** 9, -1
    cache = ba.PagedCache(pool.kp, pool.vp, ints(pool.table))
    lse_d = torch.from_numpy(lse).float().cuda()
    out = torch.full((3, 2, 100), -7.0, device="cuda")
    ba.ba_paged_key_weights(heads, cache, q, lse_d, None, out, 0.0, ints(lens), 100, None, None, nq)
    w, err = weights64(pool, f64(q), f64(lse_d), nq, 0.125, holes=[(2, 1), (0, 0)])
    for s, n in enumerate(lens):
        assert (np.abs(f64(out)[s, :, :n] - w[s, :, :n]) <= err[s, :, :n] + 1e-37).all(), s
    # a NaN or an infinity in one key is that key's alone
    pool.kp[pool.table[2, 3], 5, 1, 7], pool.kp[pool.table[2, 4], 0, 1, 0] = float("nan"), float("inf")
    bad = torch.full_like(out, -7.0)
    ba.ba_paged_key_weights(heads, cache, q, lse_d, None, bad, 0.0, ints(lens), 100, None, None, nq)
    same = torch.ones_like(out, dtype=torch.bool)
    same[2, 1, [53, 64]] = False
    assert torch.equal(bad[same], out[same]) and bool(bad[2, 1, 53].isnan())


# ---- eviction -------------------------------------------------------------------------------------------------------
def kept64(w, n, keep, first, last):
    """Places of the kept tokens of one list of weights."""
    if n <= keep:
        return list(range(n))
    tie = np.isnan(w[:n])
    w = np.where(tie, -np.inf, w[:n] + 0.0)
    always = list(range(first)) + list(range(n - last, n))
    middle = sorted(range(first, n - last), key=lambda i: (-w[i], tie[i], i))[: keep - len(always)]
    return sorted(always + middle)


@pytest.mark.parametrize("hkv,d,rows,to_rows,lens,keep,first,last", [
    (1, 64, 16, 16, [1], 1, 0, 0), (8, 128, 16, 16, [2064], 512, 4, 64), (2, 64, 7, 5, [0, 1, 50, 49, 200], 49, 3, 10), (3, 128, 64, 16, [1500, 20], 33, 0, 33),
    (2, 64, 16, 64, [3000, 1100, 5], 1024, 1, 0), (2, 64, 1, 3, [40, 30], 7, 7, 0), (1, 128, 128, 128, [5000], 1, 0, 0)])
@pytest.mark.parametrize("kind", ["plain", "ties", "odd"])
def test_evict(ba, hkv, d, rows, to_rows, lens, keep, first, last, kind):
    import torch
    pool, heads = Pool(ba, 31, lens, hkv, d, rows, padded=rows == 7), ba.Heads(hkv, hkv, d)
    w = np.random.default_rng(32).standard_normal((len(lens), hkv, pool.max_len + 5)).astype(np.float32)
    if kind == "ties":
        w = np.round(w)
        w[w == 0] = np.where(np.random.default_rng(33).random((w == 0).sum()) < 0.5, 0.0, -0.0)
    elif kind == "odd":
        u = np.random.default_rng(34).random(w.shape)
        w[u < 0.5], w[u < 0.1], w[u < 0.05], w[u < 0.02] = np.nan, np.inf, -np.inf, 1e-42
        w = np.where(np.isnan(w), np.float32(np.nan), w)
    wt = torch.from_numpy(w).cuda()
    to = Pool(ba, 35, [min(keep, n) for n in lens], hkv, d, to_rows, extra=3, padded=rows == 7)
    kp, vp = to.kp.clone(), to.vp.clone()  # what lay there before
    kept = torch.full((len(lens), hkv, keep), 99, dtype=torch.int32, device="cuda")
    w_out = torch.full((len(lens), hkv, keep + 2), -7.0, device="cuda")
    len_out = torch.full((len(lens),), 99, dtype=torch.int32, device="cuda")
    ws = torch.empty(max(256, ba.ba_paged_evict_workspace_bytes(heads, len(lens), pool.max_len, keep)), dtype=torch.uint8, device="cuda")
    ba.ba_paged_evict(heads, pool.cache, to.cache, wt, ints(lens), pool.max_len, keep, first, last, kept, w_out, len_out, ws)
    assert len_out.tolist() == [min(keep, n) for n in lens]
    kept, w_out = kept.cpu().numpy(), w_out.cpu().numpy()
    touched = torch.zeros(to.kp.shape[:2], dtype=torch.bool)
    for s, n in enumerate(lens):
        for h in range(hkv):
            want = kept64(w[s, h], n, keep, first, last)
            m = len(want)
            assert kept[s, h, :m].tolist() == want and (kept[s, h, m:] == -1).all(), (s, h)
            assert np.array_equal(w_out[s, h, :m], w[s, h, want], equal_nan=True) and (w_out[s, h, m:] == -7.0).all()
            j = np.arange(m)
            page, row = torch.from_numpy(to.table[s, j // to_rows]), torch.from_numpy(j % to_rows)
            touched[page, row] = True
            for got, src in ((to.kp, pool.k), (to.vp, pool.v)):
                assert np.array_equal(f64(got[page, row, h]), src[s, want, h]), (s, h)
    for got, before in ((to.kp, kp), (to.vp, vp)):  # nothing else has changed
        assert torch.equal(got.cpu()[~touched].nan_to_num(5.0), before.cpu()[~touched].nan_to_num(5.0))


def test_evict_within_one_pool(ba):
    """Old and new pages in the same tensor, sequences that share their old ones."""
    import torch
    hkv, d, rows, lens, keep = 2, 64, 16, [100, 90], 40
    heads, kp, vp = ba.Heads(2, 2, 64), rand(41, 20, rows, hkv, d), rand(42, 20, rows, hkv, d)
    old = ints([[3, 5, 1, 7, 0, 2, 9], [3, 5, 1, 7, 0, 8, -1]])
    new = ints([[10, 11, 12], [13, 14, 19]])
    w = torch.rand((2, hkv, 100), generator=torch.Generator().manual_seed(43)).cuda()
    kb, vb = kp.clone(), vp.clone()
    kept = torch.empty((2, hkv, keep), dtype=torch.int32, device="cuda")
    ba.ba_paged_evict(heads, ba.PagedCache(kp, vp, old), ba.PagedCache(kp, vp, new), w, ints(lens), 100, keep, 2, 5, kept)
    for s, n in enumerate(lens):
        for h in range(hkv):
            i = torch.tensor(kept64(f64(w)[s, h], n, keep, 2, 5)).cuda()
            assert torch.equal(kept[s, h].long(), i)
            j = torch.arange(keep).cuda()
            for pool, before in ((kp, kb), (vp, vb)):
                assert torch.equal(pool[new[s][j // rows].long(), j % rows, h], before[old[s][i // rows].long(), i % rows, h])
    assert torch.equal(kp[:10], kb[:10]) and torch.equal(vp[15:19], vb[15:19])


def test_evict_where_pages_are_missing(ba):
    import torch
    lens, keep, rows = [64], 32, 16
    pool, to, heads = Pool(ba, 51, lens, 1, 64, rows), Pool(ba, 52, [32], 1, 64, rows), ba.Heads(1, 1, 64)
    w = torch.arange(64.0).cuda().view(1, 1, 64).clone()
    w[0, 0, :16] += 100  # kept: 0 .. 15, 48 .. 63
    pool.table[0, 3], to.table[0, 0] = 77, -1
    before = to.kp.clone()
    kept = torch.empty((1, 1, keep), dtype=torch.int32, device="cuda")
    ba.ba_paged_evict(heads, ba.PagedCache(pool.kp, pool.vp, ints(pool.table)), ba.PagedCache(to.kp, to.vp, ints(to.table)), w, ints(lens), 64, keep, 0, 0, kept)
    assert kept[0, 0].tolist() == list(range(16)) + list(range(48, 64))
    assert torch.equal(to.kp.nan_to_num(5.0), before.nan_to_num(5.0))


# ---- bounds of pages ------------------------------------------------------------------------------------------------
def exponent(top):
    e = -60
    while top > 127 * 2.0 ** e and e < 40:  # (an infinity's is the largest)
        e += 1
    return e


def codes64(k):
    """Keys [rows, D] of one page and head: exponent, codes."""
    k = np.where(np.isnan(k), 0.0, k)
    e = exponent(np.abs(k).max())
    with np.errstate(invalid="ignore"):
        return e, np.clip(np.ceil(k.max(0) / 2.0 ** e), -127, 127), np.clip(np.floor(k.min(0) / 2.0 ** e), -127, 127)


@pytest.mark.parametrize("hkv,d,rows,lens,since", [
    (1, 64, 16, [1], [0]), (8, 128, 16, [2064], [0]), (2, 64, 7, [0, 1, 50, 49, 200], [0, 0, 20, 48, 100]), (3, 128, 64, [1500, 20, 64], [1499, 20, 63]),
    (2, 64, 128, [130, 128, 5], [127, 129, 2]), (2, 128, 1, [40, 3], [10, 0]), (1, 64, 100, [1000], [950])])
def test_page_bounds(ba, hkv, d, rows, lens, since):
    """In two steps: up to `since`, then the rest; pages of keys of very different size."""
    import torch
    pool, heads = Pool(ba, 61, lens, hkv, d, rows, padded=rows == 7), ba.Heads(hkv, hkv, d)
    rng = np.random.default_rng(62)
    for s, n in enumerate(lens):  # larger and smaller as they come, some odd ones
        size = 2.0 ** rng.integers(-70, 50, (pool.k.shape[1], hkv, 1))
        size[rng.random(size.shape) < 0.5] = 1.0
        k = pool.k[s] * size
        k[rng.random(k.shape) < 0.01], k[rng.random(k.shape) < 0.003], k[rng.random(k.shape) < 0.003] = 0.0, np.nan, -np.inf
        k = torch.from_numpy(k).bfloat16()
        pool.k[s] = k.double().numpy()
        for i in range(-(-n // rows)):
            m = min(rows, n - i * rows)
            pool.kp[pool.table[s, i], :m] = k[i * rows:i * rows + m].cuda()
    n_pages = pool.kp.shape[0]
    codes = torch.full((n_pages, hkv, 2, d), 55, dtype=torch.int8, device="cuda")
    exps = torch.full((n_pages, hkv), 5, dtype=torch.int8, device="cuda")
    bounds = ba.PageBounds(codes, exps)
    ba.ba_page_bounds(heads, pool.cache, bounds, None, ints(np.minimum(lens, since)), pool.max_len)
    ba.ba_page_bounds(heads, pool.cache, bounds, ints(since), ints(lens), pool.max_len)
    want_c, want_e = np.full(codes.shape, 55), np.full(exps.shape, 5)
    for s, n in enumerate(lens):
        for i in range(-(-n // rows)):
            for h in range(hkv):
                e, hi, lo = codes64(pool.k[s, i * rows:min(n, (i + 1) * rows), h])
                page = pool.table[s, i]
                want_e[page, h], want_c[page, h, 0], want_c[page, h, 1] = e, hi, lo
    assert np.argwhere(exps.cpu().numpy() != want_e).tolist() == []
    assert np.argwhere(codes.cpu().numpy() != want_c)[:9].tolist() == []


# ---- selection ------------------------------------------------------------------------------------------------------
def select64(pool, codes, exps, q, nq, n_select, first, last, table):
    hkv, hq = pool.hkv, q.shape[1]
    g = hq // hkv
    sel = np.full((len(pool.lens), hkv, n_select), -1)
    scores = np.full(sel.shape, -np.inf)
    for s, n in enumerate(pool.lens):
        held = -(-n // pool.rows)
        newest = max(0, n - nq) // pool.rows
        for h in range(hkv):
            x = np.full(held, -np.inf)
            for i in range(nq):
                for j in range(g):
                    r = q[s * nq + i, h * g + j]
                    r = np.where(np.isnan(r), 0.0, r)
                    e = exponent(np.abs(r).max())
                    c = np.clip(np.round(r / 2.0 ** e), -127, 127)
                    for p in range(held):
                        if 0 <= table[s, p] < len(codes):
                            both = codes[table[s, p], h].astype(np.float64)
                            x[p] = max(x[p], np.maximum(c * both[0], c * both[1]).sum() * 2.0 ** e * 2.0 ** float(exps[table[s, p], h]))
            there = [p for p in range(held) if 0 <= table[s, p] < len(codes)]
            always = [p for p in there if p < first or p >= min(held - last, newest)]
            rest = sorted((p for p in there if p not in always), key=lambda p: (-x[p], p))
            mine = sorted((always + rest)[:n_select])
            sel[s, h, :len(mine)], scores[s, h, :len(mine)] = mine, x[mine]
    return sel, scores


@pytest.mark.parametrize("hq,hkv,d,rows,lens,nq,n_select,first,last", [
    (4, 4, 64, 16, [1], 1, 1, 0, 1), (32, 8, 128, 16, [2064], 1, 20, 1, 4), (8, 2, 64, 7, [0, 1, 50, 49, 500], 1, 8, 0, 0), (6, 2, 128, 64, [1500, 20], 3, 5, 2, 2),
    (16, 2, 64, 16, [3000, 1100, 5], 5, 33, 1, 0), (40, 1, 128, 1, [140, 30], 2, 12, 0, 3), (8, 8, 64, 16, [4000, 700], 40, 64, 5, 0), (4, 1, 64, 100, [513], 1, 300, 0, 0)])
def test_page_select(ba, hq, hkv, d, rows, lens, nq, n_select, first, last):
    import torch
    pool, heads = Pool(ba, 71, lens, hkv, d, rows), ba.Heads(hq, hkv, d)
    rng = np.random.default_rng(72)
    n_pages = pool.kp.shape[0]
    codes = rng.integers(-127, 128, (n_pages, hkv, 2, d)).astype(np.int8)
    codes = np.stack([codes.max(2), codes.min(2)], 2)
    exps = rng.integers(-8, -5, (n_pages, hkv)).astype(np.int8)
    for _ in range(n_pages // 2):  # pages that are alike: ties
        codes[rng.integers(n_pages)], exps[rng.integers(n_pages)] = codes[0], exps[0]
    q = rand(73, len(lens) * nq, hq, d, scale=3.0)
    q[0, 0] = 0.0
    q[-1, -1, 3], q[-1, 0, 5] = float("nan"), float("inf")
    if len(lens) > 1:
        q[nq:2 * nq] *= 1e-30
    if n_pages > 20:
        pool.table[-1, 2], pool.table[-1, 0] = -3, n_pages
    cache = ba.PagedCache(pool.kp, pool.vp, ints(pool.table))
    bounds = ba.PageBounds(torch.from_numpy(codes).cuda(), torch.from_numpy(exps).cuda())
    sel = torch.full((len(lens), hkv, n_select), 99, dtype=torch.int32, device="cuda")
    scores = torch.full(sel.shape, 99.0, device="cuda")
    ws = torch.empty(max(256, ba.ba_page_select_workspace_bytes(heads, len(lens), rows, pool.max_len)), dtype=torch.uint8, device="cuda")
    ba.ba_page_select(heads, cache, bounds, q, ints(lens), pool.max_len, sel, scores, first, last, nq, ws)
    want, x = select64(pool, codes, exps, f64(q), nq, n_select, first, last, pool.table)
    assert np.argwhere(sel.cpu().numpy() != want)[:9].tolist() == []
    assert np.argwhere(f64(scores) != x)[:9].tolist() == []
    alone = torch.full_like(sel, 99)
    ba.ba_page_select(heads, cache, bounds, q, ints(lens), pool.max_len, alone, None, first, last, nq, ws)
    assert torch.equal(alone, sel)


# ---- attention over the selected pages ------------------------------------------------------------------------------
def attend64(pool, q, nq, sel, scale, table):
    """Outputs, log-sum-exps, sum p |v|, and how far the log-sum-exps may be off."""
    hq, d = q.shape[1], pool.d
    g = hq // pool.hkv
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    lse, off = np.full(q.shape[:2], -np.inf), np.zeros(q.shape[:2])
    for s in range(len(pool.lens)):
        for h in range(hq):
            t = []
            for j, page in enumerate(sel[s, h // g]):
                if page < 0 or (j and page <= sel[s, h // g][j - 1]):
                    break
                if page < table.shape[1] and 0 <= table[s, page] < pool.kp.shape[0]:
                    t += range(page * pool.rows, (page + 1) * pool.rows)
            t = np.array(t, dtype=np.int64)
            for i in range(nq):
                mine = t[t <= p_of(pool, s, nq, i)]
                if not len(mine):
                    continue
                k, v, r = pool.k[s, mine, h // g], pool.v[s, mine, h // g], q[s * nq + i, h]
                sc = k @ r * scale
                m = sc.max()
                p = np.exp(sc - m)
                lse[s * nq + i, h] = m + np.log(p.sum())
                off[s * nq + i, h] = d * U * (np.abs(k) @ np.abs(r) * scale).max() + (np.abs(sc).max() + abs(m) + len(mine) + 8) * U
                p /= p.sum()
                out[s * nq + i, h], size[s * nq + i, h] = p @ v, p @ np.abs(v)
    return out, lse, size, off


@pytest.mark.parametrize("hq,hkv,d,rows,lens,nq,n_select", [
    (4, 4, 64, 16, [1], 1, 1), (32, 8, 128, 16, [2064], 1, 40), (8, 2, 64, 7, [0, 1, 50, 49, 500], 1, 20), (6, 2, 128, 64, [1500, 20], 3, 9),
    (16, 2, 64, 16, [3000, 1100, 5], 5, 90), (40, 1, 128, 1, [140, 30], 2, 33), (8, 2, 128, 16, [1700, 300], 20, 64), (4, 1, 64, 100, [5130], 1, 30),
    (32, 8, 128, 32, [900] * 24, 1, 8), (8, 2, 128, 48, [700, 650], 12, 6)])
def test_attention_over_selected_pages(ba, hq, hkv, d, rows, lens, nq, n_select):
    import torch
    pool, heads = Pool(ba, 81, lens, hkv, d, rows, padded=rows == 7), ba.Heads(hq, hkv, d)
    rng = np.random.default_rng(82)
    q = rand(83, len(lens) * nq, hq, d, scale=2.0)
    sel = np.full((len(lens), hkv, n_select), -1)
    for s, n in enumerate(lens):
        held = -(-n // rows)
        for h in range(hkv):
            mine = np.sort(rng.permutation(held)[:n_select])
            if h % 3 == 0 and held and held - 1 not in mine:
                mine[-1] = held - 1
            sel[s, h, :len(mine)] = mine
    if rows == 7:
        pool.table[4, 3] = pool.kp.shape[0] + 5
        sel[4, 0, :4], sel[4, 1, 10] = [1, 2, 3, 30], 2  # a page that is not there; entries behind one that is no larger than the last
    if rows == 48:
        sel[0, 0], sel[1, 1] = -1, [13, 14, 15, 16, 1000, 2 ** 31 - 1]  # no page; pages that no token has
    cache = ba.PagedCache(pool.kp, pool.vp, ints(pool.table))
    o, lse = torch.full_like(q, float("nan")), torch.full(q.shape[:2], float("nan"), device="cuda")
    ws = torch.full((max(256, ba.ba_paged_attention_selected_workspace_bytes(heads, len(lens), nq, rows, pool.max_len, n_select)),), 255, dtype=torch.uint8, device="cuda")
    ba.ba_paged_attention_selected(heads, cache, q, o, lse, ints(lens), pool.max_len, ints(sel), nq, ws)
    out, l64, size, off = attend64(pool, f64(q), nq, sel, 1 / math.sqrt(d), pool.table)
    # probabilities to bf16 (half a step each), parts to fp16, the result to bf16; the exponentials' own errors twice (above and below)
    tol = (BF16_STEP + 2.0 ** -11 + 2 * off[..., None]) * size + BF16_STEP * (np.abs(out) + (BF16_STEP + 2.0 ** -11) * size) + 1e-30
    assert (np.abs(f64(o) - out) <= tol).all(), float((np.abs(f64(o) - out) / tol).max())
    got = f64(lse)
    assert np.array_equal(np.isinf(got), np.isinf(l64))
    fine = np.isfinite(l64)
    assert (np.abs(got[fine] - l64[fine]) <= off[fine]).all()
    in_place = q.clone()
    ba.ba_paged_attention_selected(heads, cache, in_place, in_place, None, ints(lens), pool.max_len, ints(sel), nq, ws)
    assert torch.equal(in_place, o)


def test_all_pages_selected_is_paged_attention(ba):
    """The same keys in the same order and parts: the same result, up to the parts' rounding."""
    import torch
    lens, rows, nq = [777, 64, 1000], 16, 2
    pool, heads = Pool(ba, 91, lens, 2, 128, rows), ba.Heads(8, 2, 128)
    q = rand(92, 6, 8, 128)
    n = -(-1000 // rows)
    sel = torch.arange(n).int().cuda().expand(3, 2, n).contiguous()
    outs = []
    for call, nbytes in ((lambda *a: ba.ba_paged_attention(heads, pool.cache, q, *a[:2], ints(lens), 1000, None, None, nq, a[2]),
                          ba.ba_paged_attention_workspace_bytes(heads, 3, nq, 1000)),
                         (lambda *a: ba.ba_paged_attention_selected(heads, pool.cache, q, *a[:2], ints(lens), 1000, sel, nq, a[2]),
                          ba.ba_paged_attention_selected_workspace_bytes(heads, 3, nq, rows, 1000, n))):
        o, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
        call(o, lse, torch.empty(max(256, nbytes), dtype=torch.uint8, device="cuda"))
        outs.append((f64(o), f64(lse)))
    out, l64, size, off = attend64(pool, f64(q), nq, sel.cpu().numpy(), 128 ** -0.5, pool.table)
    tol = (BF16_STEP + 2.0 ** -11 + 2 * off[..., None]) * size + BF16_STEP * (np.abs(out) + 2 * BF16_STEP * size)
    assert (np.abs(outs[0][0] - outs[1][0]) <= 2 * tol).all() and (np.abs(outs[0][1] - outs[1][1]) <= 2 * off).all()
