"""Long paged caches at their edges: a run of the operators as a program makes it, captured and replayed, on a stream of its own; places beyond 32 bits;
lists longer than a workgroup keeps; waves that go through many pages.  Tolerances as in test_long_cache_gpu.py."""
import math

import numpy as np
import pytest

from test_long_cache_gpu import BF16_STEP, Pool, attend64, codes64, f64, ints, kept64, lse64, rand, select64, weights64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ba():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2409_15355_amd import binding
    binding.load()
    return binding


def room(nbytes):
    import torch
    return torch.empty(max(256, nbytes), dtype=torch.uint8, device="cuda")


def close_attention(o, lse, out, l64, size, off):
    tol = (BF16_STEP + 2.0 ** -11 + 2 * off[..., None]) * size + BF16_STEP * (np.abs(out) + (BF16_STEP + 2.0 ** -11) * size) + 1e-30
    assert (np.abs(f64(o) - out) <= tol).all(), float((np.abs(f64(o) - out) / tol).max())
    fine = np.isfinite(l64)
    assert np.array_equal(np.isfinite(f64(lse)), fine) and (np.abs(f64(lse)[fine] - l64[fine]) <= off[fine]).all()


class Answers:
    """A program's state: prompts in one pool, cut down to other pages of it after the question, answered from there token by token."""
    HQ, HKV, D, ROWS, KEEP, SELECT = 8, 2, 128, 16, 64, 4

    def __init__(self, ba, lens, nq, steps, seed=1):
        import torch
        self.ba, self.lens, self.nq = ba, lens, nq
        self.heads = ba.Heads(self.HQ, self.HKV, self.D, 10000.0)
        n, rows = len(lens), self.ROWS
        pages, new_pages = -(-max(lens) // rows), -(-(self.KEEP + steps) // rows)
        total = n * (pages + new_pages)
        order = np.random.default_rng(seed).permutation(total)
        self.old, self.new = order[: n * pages].reshape(n, pages), order[n * pages:].reshape(n, new_pages)
        self.kp, self.vp = (torch.full((total, rows, self.HKV, self.D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.before, self.after = ba.PagedCache(self.kp, self.vp, ints(self.old)), ba.PagedCache(self.kp, self.vp, ints(self.new))
        self.bounds = ba.PageBounds(torch.zeros((total, self.HKV, 2, self.D), dtype=torch.int8, device="cuda"), torch.zeros((total, self.HKV), dtype=torch.int8, device="cuda"))
        self.max_new = self.KEEP + steps
        self.weights = torch.zeros((n, self.HKV, max(max(lens), self.max_new)), device="cuda")
        self.kept_weights = torch.zeros((n, self.HKV, self.max_new), device="cuda")
        self.kept = torch.empty((n, self.HKV, self.KEEP), dtype=torch.int32, device="cuda")
        self.len, self.since = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
        self.selected, self.scores = torch.empty((n, self.HKV, self.SELECT), dtype=torch.int32, device="cuda"), torch.empty((n, self.HKV, self.SELECT), device="cuda")
        h = self.heads
        self.ws = room(max(ba.ba_paged_attention_workspace_bytes(h, n, nq, max(lens)), ba.ba_paged_key_weights_workspace_bytes(h, n, nq, max(lens)),
                           ba.ba_paged_key_weights_workspace_bytes(h, n, 1, self.max_new), ba.ba_paged_evict_workspace_bytes(h, n, max(lens), self.KEEP),
                           ba.ba_page_select_workspace_bytes(h, n, rows, self.max_new),
                           ba.ba_paged_attention_selected_workspace_bytes(h, n, 1, rows, self.max_new, self.SELECT),
                           ba.ba_paged_attention_workspace_bytes(h, n, 1, self.max_new)))
        # a step's buffers
        self.q, self.k, self.v = (torch.empty((n, x, self.D), dtype=torch.bfloat16, device="cuda") for x in (self.HQ, self.HKV, self.HKV))
        self.o, self.o_all = torch.empty_like(self.q), torch.empty_like(self.q)
        self.lse, self.lse_all = (torch.empty((n, self.HQ), device="cuda") for _ in range(2))

    def prompt(self):
        import torch
        ba, h, n = self.ba, self.heads, len(self.lens)
        k, v = rand(11, sum(self.lens), self.HKV, self.D), rand(12, sum(self.lens), self.HKV, self.D)
        seq = np.repeat(np.arange(n), self.lens)
        at = np.concatenate([np.arange(x) for x in self.lens])
        ba.ba_paged_append(h, None, self.before, None, k, v, None, ints(at), ints(seq), None, ba.ROPE_APPLY)
        q = rand(13, n * self.nq, self.HQ, self.D, scale=2.0)
        o, lse, lens = torch.empty_like(q), torch.empty((n * self.nq, self.HQ), device="cuda"), ints(self.lens)
        ba.ba_paged_attention(h, self.before, q, o, lse, lens, max(self.lens), None, None, self.nq, self.ws)
        ba.ba_paged_key_weights(h, self.before, q, lse, None, self.weights, 0.0, lens, max(self.lens), None, None, self.nq, self.ws)
        ba.ba_paged_evict(h, self.before, self.after, self.weights, lens, max(self.lens), self.KEEP, 2, 8, self.kept, self.kept_weights, self.len, self.ws)
        ba.ba_page_bounds(h, self.after, self.bounds, None, self.len, self.max_new)
        return q, lse

    def step(self):
        """One token of every sequence: the new length, then everything that reads it."""
        ba, h = self.ba, self.heads
        self.since.copy_(self.len)
        ba.ba_paged_append(h, None, self.after, None, self.k, self.v, None, self.since, None, None, ba.ROPE_NONE)
        self.len += 1
        ba.ba_page_bounds(h, self.after, self.bounds, self.since, self.len, self.max_new)
        ba.ba_page_select(h, self.after, self.bounds, self.q, self.len, self.max_new, self.selected, self.scores, 1, 1, 1, self.ws)
        ba.ba_paged_attention_selected(h, self.after, self.q, self.o, self.lse, self.len, self.max_new, self.selected, 1, self.ws)
        ba.ba_paged_attention(h, self.after, self.q, self.o_all, self.lse_all, self.len, self.max_new, None, None, 1, self.ws)
        ba.ba_paged_key_weights(h, self.after, self.q, self.lse_all, self.kept_weights, self.kept_weights, 0.5, self.len, self.max_new, None, None, 1, self.ws)

    def token(self, i):
        n = len(self.lens)
        self.q.copy_(rand(100 + i, n, self.HQ, self.D, scale=2.0))
        self.k.copy_(rand(200 + i, n, self.HKV, self.D))
        self.v.copy_(rand(300 + i, n, self.HKV, self.D))

    def results(self):
        return [x.clone() for x in (self.o, self.lse, self.selected, self.scores, self.kept_weights, self.len, self.kp, self.vp, self.bounds.codes, self.bounds.exponents)]


def in_pages(pool, pages, n):
    return f64(pool)[pages].reshape(-1, *pool.shape[2:])[:n]


class Seen:
    """What the 64-bit forms want to know of sequences in pages."""

    def __init__(self, a, table, lens):
        self.lens, self.rows, self.hkv, self.d, self.kp, self.max_len = lens, a.ROWS, a.HKV, a.D, a.kp, max(lens)
        self.k, self.v = ([in_pages(pool, table[s], n) for s, n in enumerate(lens)] for pool in (a.kp, a.vp))
        width = table.shape[1] * a.ROWS
        pad = lambda xs: np.stack([np.pad(x, ((0, width - len(x)), (0, 0), (0, 0))) for x in xs])  # noqa: E731
        self.k, self.v = pad(self.k), pad(self.v)


def test_a_run_of_them(ba):
    """Prompt, question, eviction, then tokens from selected pages: every output against what the ones before it have left."""
    steps, lens, nq = 20, [200, 37, 130], 6
    a = Answers(ba, lens, nq, steps)
    q, lse = a.prompt()
    seen = Seen(a, a.old, lens)
    scale = a.D ** -0.5
    w, err = weights64(seen, f64(q), f64(lse), nq, scale)
    new = [min(n, a.KEEP) for n in lens]
    assert a.len.tolist() == new
    got_w, kept = f64(a.weights), a.kept.cpu().numpy()
    for s, n in enumerate(lens):
        assert (np.abs(got_w[s, :, :n] - w[s, :, :n]) <= err[s, :, :n] + 1e-37).all()
        for h in range(a.HKV):
            want = kept64(got_w[s, h], n, a.KEEP, 2, 8)
            assert kept[s, h, :new[s]].tolist() == want
            for pool, x in ((a.kp, seen.k), (a.vp, seen.v)):
                assert np.array_equal(in_pages(pool, a.new[s], new[s])[:, h], x[s, want, h])
    old_w = f64(a.kept_weights)
    for i in range(steps):
        a.token(i)
        a.step()
        now = [n + i + 1 for n in new]
        assert a.len.tolist() == now
        seen = Seen(a, a.new, now)
        for s, n in enumerate(now):
            assert np.array_equal(seen.k[s, n - 1], f64(a.k)[s])
            for p in range(-(-n // a.ROWS)):
                for h in range(a.HKV):
                    e, hi, lo = codes64(seen.k[s, p * a.ROWS:min(n, (p + 1) * a.ROWS), h])
                    page = a.new[s, p]
                    assert int(a.bounds.exponents[page, h]) == e and np.array_equal(f64(a.bounds.codes[page, h]), [hi, lo])
        codes, exps = a.bounds.codes.cpu().numpy(), a.bounds.exponents.cpu().numpy()
        sel, scores = select64(seen, codes, exps, f64(a.q), 1, a.SELECT, 1, 1, a.new)
        assert np.array_equal(a.selected.cpu().numpy(), sel) and np.array_equal(f64(a.scores), scores)
        close_attention(a.o, a.lse, *attend64(seen, f64(a.q), 1, sel, scale, a.new))
        w, err = weights64(seen, f64(a.q), f64(a.lse_all), 1, scale)
        got = f64(a.kept_weights)
        for s, n in enumerate(now):
            want = w[s, :, :n].copy()
            want[:, :n - 1] += 0.5 * old_w[s, :, :n - 1]
            assert (np.abs(got[s, :, :n] - want) <= err[s, :, :n] + 2.0 ** -23 * np.abs(want) + 1e-37).all()
        old_w = got


@pytest.mark.parametrize("how", ["stream", "graph"])
def test_a_run_on_a_stream_of_its_own_and_replayed(ba, how):
    import torch
    steps, lens, nq = 8, [100, 250], 40
    plain, other = Answers(ba, lens, nq, steps), Answers(ba, lens, nq, steps)
    plain.prompt()
    want = []
    for i in range(steps):
        plain.token(i)
        plain.step()
        want.append(plain.results())
    other.prompt()
    torch.cuda.synchronize()
    if how == "stream":
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for i in range(steps):
                other.token(i)
                other.step()
                got = other.results()
                stream.synchronize()
                assert all(torch.equal(x.nan_to_num(3.0), y.nan_to_num(3.0)) for x, y in zip(got, want[i])), i
        return
    other.token(0)
    other.step()  # (ahead of the capture, as programs warm up)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        other.step()
    for i in range(1, steps):
        other.token(i)
        graph.replay()
        torch.cuda.synchronize()
        got = other.results()
        assert all(torch.equal(x.nan_to_num(3.0), y.nan_to_num(3.0)) for x, y in zip(got, want[i])), i
        plain.o.add_(1)  # (eager work between the replays)


def test_places_beyond_32_bits(ba):
    """Pages 4 GB and more apart, weights of heads 2 GB apart."""
    import torch
    hkv, d, rows, n = 2, 64, 16, 40
    stride = (1 << 31) + 64  # elements
    whole = [torch.empty(2 * stride + rows * hkv * d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    kp, vp = (x.as_strided((3, rows, hkv, d), (stride, hkv * d, d, 1)) for x in whole)
    k, v = rand(1, n, hkv, d), rand(2, n, hkv, d)
    for pool, x in ((kp, k), (vp, v)):
        for i, page in enumerate((2, 0, 1)):
            pool[page] = float("nan")
            part = x[i * rows:(i + 1) * rows]
            pool[page, :len(part)] = part
    heads, cache = ba.Heads(4, hkv, d), ba.PagedCache(kp, vp, ints([[2, 0, 1]]))

    class Near:
        pass
    Near.lens, Near.k, Near.v, Near.max_len = [n], f64(k)[None], f64(v)[None], n
    Near.rows, Near.hkv, Near.d, Near.kp = rows, hkv, d, kp
    q = rand(3, 1, 4, d, scale=2.0)
    lse = torch.from_numpy(lse64(Near, f64(q), 1, 0.125)).float().cuda()
    far = torch.empty((1 << 29) + n, dtype=torch.float32, device="cuda")
    weights = far.as_strided((1, hkv, n), (hkv << 29, 1 << 29, 1))
    ba.ba_paged_key_weights(heads, cache, q, lse, None, weights, 0.0, ints([n]), n)
    w, err = weights64(Near, f64(q), f64(lse), 1, 0.125)
    assert (np.abs(f64(weights) - w) <= err + 1e-37).all()
    kept = torch.empty((1, hkv, 20), dtype=torch.int32, device="cuda")
    to_k, to_v = (torch.empty((2, rows, hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ba.ba_paged_evict(heads, cache, ba.PagedCache(to_k, to_v, ints([[1, 0]])), weights, ints([n]), n, 20, 0, 3, kept)
    for h in range(hkv):
        i = kept64(f64(weights)[0, h], n, 20, 0, 3)
        assert kept[0, h].tolist() == i
        assert torch.equal(torch.cat([to_k[1], to_k[0]])[:20, h], k[i, h]) and torch.equal(torch.cat([to_v[1], to_v[0]])[:20, h], v[i, h])
    # and into pages that far apart
    back = ba.PagedCache(to_k, to_v, ints([[1, 0]]))
    kp[:, :, :, :], vp[:, :, :, :] = 0, 0
    ba.ba_paged_evict(heads, back, cache, weights, ints([20]), 20, 20, 0, 0, kept)
    assert torch.equal(kp[0, :4], to_k[0, :4]) and torch.equal(vp[2], to_v[1]) and not kp[1].any()
    bounds = ba.PageBounds(torch.zeros((3, hkv, 2, d), dtype=torch.int8, device="cuda"), torch.zeros((3, hkv), dtype=torch.int8, device="cuda"))
    ba.ba_page_bounds(heads, cache, bounds, None, ints([20]), n)
    for page, m in ((2, 16), (0, 4)):
        for h in range(hkv):
            e, hi, lo = codes64(f64(kp[page, :m, h]))
            assert int(bounds.exponents[page, h]) == e and np.array_equal(f64(bounds.codes[page, h]), [hi, lo])
    Near.k, Near.v, Near.lens = np.concatenate([f64(kp[2]), f64(kp[0]), f64(kp[1])])[None], np.concatenate([f64(vp[2]), f64(vp[0]), f64(vp[1])])[None], [20]
    o, lse_out = torch.empty_like(q), torch.empty((1, 4), device="cuda")
    sel = np.array([[[1], [0]]])
    ba.ba_paged_attention_selected(heads, cache, q, o, lse_out, ints([20]), n, ints(sel), 1, room(ba.ba_paged_attention_selected_workspace_bytes(heads, 1, 1, rows, n, 1)))
    close_attention(o, lse_out, *attend64(Near, f64(q), 1, sel, 0.125, np.array([[2, 0, 1]])))


@pytest.mark.parametrize("n,keep", [(4097, 1000), (9000, 4000), (40000, 5000), (32768, 1), (70000, 69000)])
@pytest.mark.parametrize("kind", ["plain", "few values", "one value", "denormal"])
def test_long_lists(ba, n, keep, kind):
    """Lists that a workgroup keeps in registers, and longer ones; keys that take several digits to tell apart, or none."""
    import torch
    rng = np.random.default_rng(n)
    w = rng.standard_normal((1, 2, n)).astype(np.float32)
    if kind == "few values":
        w = rng.integers(0, 3, w.shape).astype(np.float32)
    elif kind == "one value":
        w[:] = 0.25
    elif kind == "denormal":  # neighbours: every bit counts
        w = (np.float32(1.0).view(np.int32) + rng.integers(0, 2 * n, w.shape).astype(np.int32)).view(np.float32)
        w[0, 1] = rng.integers(0, 1 << 20, n).astype(np.int32).view(np.float32)
    heads, rows = ba.Heads(2, 2, 64), 64
    pages = -(-n // rows)
    kp = torch.zeros((1, rows, 2, 64), dtype=torch.bfloat16, device="cuda")
    to = torch.zeros((1, rows, 2, 64), dtype=torch.bfloat16, device="cuda")
    none = ba.PagedCache(kp, kp.clone(), torch.full((1, pages), -1, dtype=torch.int32, device="cuda"))  # (no page is there: only the lists count)
    new = ba.PagedCache(to, to.clone(), torch.full((1, pages), -1, dtype=torch.int32, device="cuda"))
    kept = torch.empty((1, 2, keep), dtype=torch.int32, device="cuda")
    out = torch.empty((1, 2, keep), device="cuda")
    for first, last in ((0, 0), (min(3, keep), min(100, keep - min(3, keep)))):
        ba.ba_paged_evict(heads, none, new, torch.from_numpy(w).cuda(), ints([n]), n, keep, first, last, kept, out)
        for h in range(2):
            order = np.argsort(-w[0, h, first:n - last], kind="stable")[: keep - first - last] + first
            want = np.sort(np.concatenate([np.arange(first), order, np.arange(n - last, n)]))
            assert np.array_equal(kept[0, h].cpu().numpy(), want)
            assert np.array_equal(out[0, h].cpu().numpy(), w[0, h, want])


def test_many_pages(ba):
    """Waves that bound more pages than they have lanes; selections out of more pages than a workgroup keeps."""
    import torch
    hkv, d, n_seqs, n = 8, 64, 256, 130
    heads = ba.Heads(hkv, hkv, d)
    k = rand(1, n_seqs * n, 1, hkv, d)
    table = torch.randperm(n_seqs * n, generator=torch.Generator().manual_seed(2)).view(n_seqs, n)
    cache = ba.PagedCache(k, k, table.int().cuda())
    bounds = ba.PageBounds(torch.zeros((n_seqs * n, hkv, 2, d), dtype=torch.int8, device="cuda"), torch.zeros((n_seqs * n, hkv), dtype=torch.int8, device="cuda"))
    ba.ba_page_bounds(heads, cache, bounds, None, ints([n] * n_seqs), n)
    x = f64(k[:, 0])  # (powers of two on the CPU: exact)
    e = np.ceil(np.log2(np.abs(x).max(-1) / 127) - 1e-6)
    scale = np.ldexp(1.0, e.astype(int))[..., None]
    codes = f64(bounds.codes)
    assert np.array_equal(f64(bounds.exponents), e)
    assert np.array_equal(codes[:, :, 0], np.ceil(x / scale)) and np.array_equal(codes[:, :, 1], np.floor(x / scale))
    long = ba.PagedCache(k, k, table.view(1, -1)[:, :33000].contiguous().int().cuda())
    q = rand(3, 1, hkv, d)
    sel = torch.empty((1, hkv, 700), dtype=torch.int32, device="cuda")
    ba.ba_page_select(heads, long, bounds, q, ints([32990]), 33000, sel, None, 2, 3, 1, room(ba.ba_page_select_workspace_bytes(heads, 1, 1, 33000)))
    qe = np.ceil(np.log2(np.abs(f64(q[0])).max(-1) / 127) - 1e-6)
    c = np.round(np.ldexp(f64(q[0]), -qe.astype(int)[:, None]))
    pages = table.view(-1)[:32990].numpy()
    both = codes[pages] * scale[pages][..., None, :]  # [pages, heads, 2, D]
    score = np.maximum(c * both[:, :, 0], c * both[:, :, 1]).sum(-1).T  # (2^qe: the same for all of a head's)
    for h in range(hkv):
        rest = np.argsort(-score[h, 2:32987], kind="stable")[:695] + 2
        assert np.array_equal(sel[0, h].cpu().numpy(), np.sort(np.concatenate([[0, 1], rest, [32987, 32988, 32989]])))


def test_a_padded_batch(ba):
    """Sequences that are not there yet (length 0, no pages), lengths beyond the bound and below zero."""
    import torch
    lens = [100, 0, 300, -5, 37]
    real = [100, 0, 64, 0, 37]
    pool = Pool(ba, 5, real, 2, 64, 16)
    heads, max_len = ba.Heads(4, 2, 64), 100
    pool.max_len = max_len
    pool.lens = [min(max(n, 0), max_len) for n in lens]
    pool.table[1], pool.table[3] = -1, -1
    cache = ba.PagedCache(pool.kp, pool.vp, ints(pool.table))
    pad = lambda x: np.pad(x, ((0, 0), (0, max(0, max_len - x.shape[1])), (0, 0), (0, 0)))  # noqa: E731
    pool.k, pool.v = pad(pool.k), pad(pool.v)
    q = rand(6, 5, 4, 64, scale=2.0)
    lse = torch.zeros((5, 4), device="cuda")
    w = torch.full((5, 2, max_len), -7.0, device="cuda")
    ba.ba_paged_key_weights(heads, cache, q, lse, None, w, 0.0, ints(lens), max_len)
    want, err = weights64(pool, f64(q), np.zeros((5, 4)), 1, 0.125, holes=[(2, i) for i in range(4, 7)])
    for s, n in enumerate(pool.lens):
        m = min(n, real[s]) if s == 2 else n
        assert (np.abs(f64(w)[s, :, :m] - want[s, :, :m]) <= err[s, :, :m] + 1e-37).all() and (f64(w)[s, :, n:] == -7.0).all()
        assert (f64(w)[s, :, m:n] == 0).all()  # (pages that are not there)
    sel = torch.full((5, 2, 3), 9, dtype=torch.int32, device="cuda")
    n_pages = pool.kp.shape[0]
    bounds = ba.PageBounds(torch.zeros((n_pages, 2, 2, 64), dtype=torch.int8, device="cuda"), torch.zeros((n_pages, 2), dtype=torch.int8, device="cuda"))
    ba.ba_page_bounds(heads, cache, bounds, None, ints(lens), max_len)
    ba.ba_page_select(heads, cache, bounds, q, ints(lens), max_len, sel, None, 1, 1, 1, room(ba.ba_page_select_workspace_bytes(heads, 5, 16, max_len)))
    assert (sel[[1, 3]] == -1).all() and sel[2].max() <= 3 and sel[4, 0].tolist() == [0, 1, 2]
    o, l = torch.full_like(q, 5.0), torch.full((5, 4), 5.0, device="cuda")
    ba.ba_paged_attention_selected(heads, cache, q, o, l, ints(lens), max_len, sel, 1, room(ba.ba_paged_attention_selected_workspace_bytes(heads, 5, 1, 16, max_len, 3)))
    assert not o[[1, 3]].any() and (l[[1, 3]] == -math.inf).all()
    close_attention(o, l, *attend64(pool, f64(q), 1, sel.cpu().numpy(), 0.125, pool.table))


@pytest.mark.parametrize("keep,pages", [(0, 0), (48, 0), (0, 6), (64, 3)])
def test_the_example(keep, pages):
    """examples/long_answers.py at a small size: what its last step leaves against 64 bits."""
    import importlib.util
    import os

    from paper_2409_15355_amd import binding
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "long_answers.py")
    spec = importlib.util.spec_from_file_location("long_answers", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    run = example.LongAnswers(binding.Heads(8, 2, 64, 10000.0), 3, 200, 9, 5, 16, keep, pages, seed=4)
    for _ in range(4):
        o = run.step()
    n = (keep or 209) + 4
    assert run.len.tolist() == [n] * 3 and run.position.tolist() == [213] * 3

    class Now:
        pass
    table = run.cache.page_table.cpu().numpy()
    Now.lens, Now.rows, Now.hkv, Now.d, Now.kp, Now.max_len = [n] * 3, 16, 2, 64, run.cache.k_pages, n
    Now.k, Now.v = (np.nan_to_num(np.stack([f64(pool)[table[s]].reshape(-1, 2, 64) for s in range(3)])) for pool in (run.cache.k_pages, run.cache.v_pages))
    held = -(-n // 16)
    sel = run.selected.cpu().numpy() if pages else np.tile(np.arange(held), (3, 2, 1))
    if pages:
        sel64, _ = select64(Now, run.bounds.codes.cpu().numpy(), run.bounds.exponents.cpu().numpy(), f64(run.q_rot), 1, pages, 1, 1, table)
        assert np.array_equal(sel, sel64)
    out, _, size, off = attend64(Now, f64(run.q_rot), 1, sel, 0.125, table)
    tol = (BF16_STEP + 2.0 ** -11 + 2 * off[..., None]) * size + BF16_STEP * (np.abs(out) + (BF16_STEP + 2.0 ** -11) * size) + 1e-30
    assert (np.abs(f64(o) - out) <= tol).all()
