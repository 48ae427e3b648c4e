"""Head norms with rotation and their backward, appending to a paged cache and attention over its pages, against plain
implementations in 64 bits.  Tolerances follow from the arithmetic and are set ahead of any run: a bf16 result may be off by
its rounding (2^-8 of the value at most), probabilities are rounded once to bf16 as well (2^-8 of sum p |v|), everything
else is 32-bit (some 2^-24 an operation, relative to what is added up)."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

BF16_STEP = 2.0 ** -8


@pytest.fixture(scope="module")
def ba():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2409_15355_amd import binding
    binding.load()
    return binding


def rand(seed, *shape, scale=1.0, dtype="bf16"):
    import torch
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=gen) * scale
    return (x.bfloat16() if dtype == "bf16" else x).cuda()


def f64(t):
    return t.detach().double().cpu().numpy()


def ints(x):
    import torch
    return torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


# ---- in 64 bits -------------------------------------------------------------------------------------------------
def rotate64(x, pos, base, layout):
    """x [tokens, heads, D] turned by R(pos)."""
    d = x.shape[-1]
    th = np.array([base ** (-2.0 * j / d) for j in range(d // 2)])
    ang = np.asarray(pos, dtype=np.float64)[:, None, None] * th
    c, s = np.cos(ang), np.sin(ang)
    y = np.empty_like(x)
    a, b = (np.s_[..., 0::2], np.s_[..., 1::2]) if layout == 0 else (np.s_[..., : d // 2], np.s_[..., d // 2:])
    y[a] = c * x[a] - s * x[b]
    y[b] = s * x[a] + c * x[b]
    return y


def pair_size(x, layout):
    """Length of the pair that each element belongs to."""
    d = x.shape[-1]
    if layout == 0:
        return np.repeat(np.hypot(x[..., 0::2], x[..., 1::2]), 2, axis=-1)
    n = np.hypot(x[..., : d // 2], x[..., d // 2:])
    return np.concatenate([n, n], axis=-1)


def norm64(x, w, eps):
    y = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps)
    return y if w is None else y * w


def norm_back64(x, w, eps, g):
    r = 1.0 / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps)
    n, b = x * r, (g if w is None else g * w)
    m = (b * n).mean(-1, keepdims=True)
    size = r * (np.abs(b).max(-1, keepdims=True) + np.abs(n).max(-1, keepdims=True) * np.abs(b * n).mean(-1, keepdims=True))
    return r * (b - n * m), (g * n).sum((0, 1)), size, np.abs(g * n).sum((0, 1))


def attend64(q, k, v, scale):
    """Rows q [heads, D] over keys k, v [keys, KV heads, D], all of them seen: outputs, lse, sum p |v|."""
    hq, d = q.shape
    if len(k) == 0:
        return np.zeros_like(q), np.full(hq, -np.inf), np.zeros_like(q)
    g = hq // k.shape[1]
    kk, vv = np.repeat(k, g, axis=1), np.repeat(v, g, axis=1)
    s = np.einsum("hd,khd->hk", q, kk) * scale
    m = s.max(1, keepdims=True)
    p = np.exp(s - m)
    lse = m[:, 0] + np.log(p.sum(1))
    p /= p.sum(1, keepdims=True)
    return np.einsum("hk,khd->hd", p, vv), lse, np.einsum("hk,khd->hd", p, np.abs(vv))


# ---- head norms ---------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("hq,hkv,d,tokens", [(4, 4, 64, 1), (8, 2, 64, 77), (32, 8, 128, 33), (5, 1, 128, 2049), (3, 3, 64, 4097)])
def test_norm_rotate(ba, hq, hkv, d, tokens, layout, dtype):
    import torch
    heads = ba.Heads(hq, hkv, d, 500000.0, rope_layout=layout)
    q, k = rand(1, tokens, hq, d, scale=3.0, dtype=dtype), rand(2, tokens, hkv, d, scale=0.01, dtype=dtype)
    if tokens > 3:
        q[2] = 0.0
    wq, wk = (rand(s, d, scale=0.3, dtype=dtype) + 1 for s in (3, 4))
    pos = np.random.default_rng(5).integers(-1000, 200000, tokens)
    for mode in (ba.ROPE_APPLY, ba.ROPE_NONE):
        qo, ko = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
        ba.ba_norm_rotate(heads, ba.HeadNorm(wq, wk, 1e-5), q, k, qo, ko, ints(pos), mode)
        for x, w, y in ((q, wq, qo), (k, wk, ko)):
            ref = norm64(f64(x), f64(w), 1e-5)
            if mode == ba.ROPE_APPLY:
                ref = rotate64(ref, pos, 500000.0, layout)
            size = pair_size(ref, layout)
            tol = 2e-6 * size + (BF16_STEP * np.abs(ref) if dtype == "bf16" else 0.0) + 1e-30
            err = np.abs(f64(y) - ref)
            assert (err <= tol).all(), float((err / np.maximum(size, 1e-30)).max())
    # in place, without gains, one tensor only, positions by number
    q2 = q.clone()
    ba.ba_norm_rotate(heads, ba.HeadNorm(None, wk, 1e-5), q2, None, q2, None, None)
    ref = rotate64(norm64(f64(q), None, 1e-5), np.arange(tokens), 500000.0, layout)
    tol = 2e-6 * pair_size(ref, layout) + (BF16_STEP * np.abs(ref) if dtype == "bf16" else 0.0) + 1e-30
    assert (np.abs(f64(q2) - ref) <= tol).all()


def test_norm_rotate_of_one_projection_in_place(ba):
    """Query and key heads lie side by side in the rows of one projection; values between them stay as they are."""
    import torch
    hq, hkv, d, tokens = 8, 2, 64, 50
    heads = ba.Heads(hq, hkv, d, 10000.0)
    qkv = rand(11, tokens, hq + 2 * hkv, d)
    before = qkv.clone()
    w = rand(12, d, dtype="f32") + 1
    norm = ba.HeadNorm(w, w)
    q, k = qkv[:, :hq], qkv[:, hq:hq + hkv]
    ba.ba_norm_rotate(heads, norm, q, k, q, k)
    qo, ko = torch.empty_like(before[:, :hq]), torch.empty_like(before[:, hq:hq + hkv])
    ba.ba_norm_rotate(heads, norm, before[:, :hq], before[:, hq:hq + hkv], qo, ko)
    assert torch.equal(qkv[:, :hq], qo) and torch.equal(qkv[:, hq:hq + hkv], ko) and torch.equal(qkv[:, hq + hkv:], before[:, hq + hkv:])


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_norm_rotate_keeps_a_bad_head_to_itself(ba, bad):
    import torch
    heads = ba.Heads(8, 2, 128, 10000.0)
    q, k = rand(21, 40, 8, 128), rand(22, 40, 2, 128)
    norm = ba.HeadNorm(None, None)
    clean = torch.empty_like(q)
    ba.ba_norm_rotate(heads, norm, q, None, clean, None)
    q[7, 3, 5] = bad
    out = torch.empty_like(q)
    ba.ba_norm_rotate(heads, norm, q, k, out, torch.empty_like(k))
    same = torch.ones(40, 8, dtype=torch.bool)
    same[7, 3] = False
    assert torch.equal(out.cpu()[same], clean.cpu()[same]) and torch.isnan(out[7, 3]).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout,mode", [(0, 1), (1, 1), (0, 0)])
@pytest.mark.parametrize("hq,hkv,d,tokens", [(4, 4, 64, 1), (8, 2, 64, 77), (32, 8, 128, 33), (5, 1, 128, 300)])
def test_norm_rotate_backward(ba, hq, hkv, d, tokens, layout, mode, dtype):
    import torch
    heads = ba.Heads(hq, hkv, d, 10000.0, rope_layout=layout)
    q, k = rand(31, tokens, hq, d, scale=2.0, dtype=dtype), rand(32, tokens, hkv, d, scale=0.2, dtype=dtype)
    gq, gk = rand(33, tokens, hq, d, scale=0.1, dtype=dtype), rand(34, tokens, hkv, d, dtype=dtype)
    wq, wk = (rand(s, d, scale=0.3, dtype="f32") + 1 for s in (35, 36))
    pos = np.random.default_rng(37).integers(0, 30000, tokens)
    dq, dk = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    dwq, dwk = torch.full((d,), float("nan"), device="cuda"), torch.full((d,), float("nan"), device="cuda")
    ws = torch.empty(ba.ba_norm_rotate_backward_workspace_bytes(heads, tokens), dtype=torch.uint8, device="cuda")
    norm = ba.HeadNorm(wq, wk, 1e-6)
    ba.ba_norm_rotate_backward(heads, norm, q, k, gq, gk, dq, dk, dwq, dwk, ints(pos), mode, ws)
    for x, w, g, dx, dw in ((q, wq, gq, dq, dwq), (k, wk, gk, dk, dwk)):
        g64 = rotate64(f64(g), -pos, 10000.0, layout) if mode else f64(g)
        ref, ref_w, size, size_w = norm_back64(f64(x), f64(w), 1e-6, g64)
        tol = 8e-6 * size + (BF16_STEP * np.abs(ref) if dtype == "bf16" else 0.0)
        assert (np.abs(f64(dx) - ref) <= tol).all()
        assert (np.abs(f64(dw) - ref_w) <= 4e-6 * size_w).all()
    # again, into the gradients' own memory and without the gains' gradients: the same bits
    dq2, dk2 = gq.clone(), gk.clone()
    ba.ba_norm_rotate_backward(heads, norm, q, k, dq2, dk2, dq2, dk2, None, None, ints(pos), mode, ws)
    assert torch.equal(dq2, dq) and torch.equal(dk2, dk)
    dwk2 = torch.empty_like(dwk)
    ba.ba_norm_rotate_backward(heads, norm, None, k, None, gk, None, dk2, None, dwk2, ints(pos), mode, ws)
    assert torch.equal(dwk2, dwk) and torch.equal(dk2, dk)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,tokens", [(32, 8, 128, 2), (32, 8, 128, 3), (32, 8, 128, 4), (32, 8, 128, 5), (8, 2, 64, 16), (8, 2, 64, 17),
                                             (8, 2, 64, 33), (7, 7, 64, 11), (16, 1, 128, 1), (1, 1, 64, 256), (1, 1, 64, 257), (40, 2, 128, 1),
                                             (32, 8, 128, 300)])
def test_norm_rotate_backward_of_few_tokens(ba, hq, hkv, d, tokens, dtype):
    """Around the size from which the gains' gradients take a launch of their own.  Few terms: a rotation's error goes with its pair's
    length, however small the element that comes out."""
    import torch
    heads = ba.Heads(hq, hkv, d, 10000.0, rope_layout=0)
    q, k = rand(31, tokens, hq, d, scale=2.0, dtype=dtype), rand(32, tokens, hkv, d, scale=0.2, dtype=dtype)
    gq, gk = rand(33, tokens, hq, d, scale=0.1, dtype=dtype), rand(34, tokens, hkv, d, dtype=dtype)
    wq, wk = (rand(s, d, scale=0.3, dtype="f32") + 1 for s in (35, 36))
    pos = np.random.default_rng(37).integers(0, 30000, tokens)
    dq, dk = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    dwq, dwk = torch.full((d,), float("nan"), device="cuda"), torch.full((d,), float("nan"), device="cuda")
    ws = torch.empty(ba.ba_norm_rotate_backward_workspace_bytes(heads, tokens), dtype=torch.uint8, device="cuda")
    norm = ba.HeadNorm(wq, wk, 1e-6)
    ba.ba_norm_rotate_backward(heads, norm, q, k, gq, gk, dq, dk, dwq, dwk, ints(pos), ba.ROPE_APPLY, ws)
    for x, w, g, dx, dw in ((q, wq, gq, dq, dwq), (k, wk, gk, dk, dwk)):
        g64 = rotate64(f64(g), -pos, 10000.0, 0)
        ref, ref_w, size, _ = norm_back64(f64(x), f64(w), 1e-6, g64)
        size_w = norm_back64(f64(x), f64(w), 1e-6, pair_size(f64(g), 0))[3]
        assert (np.abs(f64(dx) - ref) <= 8e-6 * size + (BF16_STEP * np.abs(ref) if dtype == "bf16" else 0.0)).all()
        assert (np.abs(f64(dw) - ref_w) <= 4e-6 * size_w).all()
    dq2, dk2, dwk2 = gq.clone(), gk.clone(), torch.empty_like(dwk)
    ba.ba_norm_rotate_backward(heads, norm, q, k, dq2, dk2, dq2, dk2, None, None, ints(pos), ba.ROPE_APPLY, ws)
    assert torch.equal(dq2, dq) and torch.equal(dk2, dk)
    ba.ba_norm_rotate_backward(heads, norm, None, k, None, gk, None, dk2, None, dwk2, ints(pos), ba.ROPE_APPLY, ws)
    assert torch.equal(dwk2, dwk) and torch.equal(dk2, dk)


def test_norm_rotate_backward_against_differences(ba):
    """Directional differences of the 32-bit forward pass, step 2^-8: their own error is some h^2 of the gradient's size
    (curvature of the norm) and 2^-24 / h of the outputs' (rounding), below 1e-3 of it together."""
    import torch
    hq, hkv, d, tokens, h = 4, 2, 64, 19, 2.0 ** -8
    heads = ba.Heads(hq, hkv, d, 10000.0, rope_layout=1)
    q, k = rand(41, tokens, hq, d, dtype="f32"), rand(42, tokens, hkv, d, dtype="f32")
    gq, gk = rand(43, tokens, hq, d, dtype="f32"), rand(44, tokens, hkv, d, dtype="f32")
    wq, wk = (rand(s, d, scale=0.3, dtype="f32") + 1 for s in (45, 46))
    pos = ints(np.arange(tokens) * 37)

    def loss(q_, k_, wq_, wk_):
        qo, ko = torch.empty_like(q), torch.empty_like(k)
        ba.ba_norm_rotate(heads, ba.HeadNorm(wq_, wk_, 1e-6), q_, k_, qo, ko, pos)
        return float((f64(qo) * f64(gq)).sum() + (f64(ko) * f64(gk)).sum())

    dq, dk, dwq, dwk = torch.empty_like(q), torch.empty_like(k), torch.empty_like(wq), torch.empty_like(wk)
    ws = torch.empty(ba.ba_norm_rotate_backward_workspace_bytes(heads, tokens), dtype=torch.uint8, device="cuda")
    ba.ba_norm_rotate_backward(heads, ba.HeadNorm(wq, wk, 1e-6), q, k, gq, gk, dq, dk, dwq, dwk, pos, ba.ROPE_APPLY, ws)
    args = [q, k, wq, wk]
    for i, grad in enumerate((dq, dk, dwq, dwk)):
        step = rand(50 + i, *grad.shape, dtype="f32")
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + h * step, args[i] - h * step
        got = (loss(*up) - loss(*down)) / (2 * h)
        assert abs(got - (f64(grad) * f64(step)).sum()) <= 1e-3 * np.linalg.norm(f64(grad)) * max(1.0, np.linalg.norm(f64(step)) / math.sqrt(step.numel()))


def test_norm_rotate_backward_without_tokens(ba):
    import torch
    heads = ba.Heads(4, 2, 64)
    q, k = torch.empty(0, 4, 64, device="cuda"), torch.empty(0, 2, 64, device="cuda")
    dw = torch.full((64,), 7.0, device="cuda")
    ba.ba_norm_rotate(heads, ba.HeadNorm(), q, k, q, k)
    ba.ba_norm_rotate_backward(heads, ba.HeadNorm(), q, k, q, k, q, k, dw, None)
    assert (dw == 0).all()


# ---- the cache ------------------------------------------------------------------------------------------------------
def pools(seed, n_pages, rows, hkv, d, form="plain"):
    """k and v pages, filled with NaN."""
    import torch
    shape = {"plain": (n_pages, rows, hkv, d), "heads_first": (n_pages, hkv, rows, d), "together": (n_pages, 2, rows, hkv, d)}[form]
    if form == "together":
        kv = torch.full(shape, float("nan"), dtype=torch.bfloat16, device="cuda")
        return kv[:, 0], kv[:, 1]
    k, v = (torch.full(shape, float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    return (k.transpose(1, 2), v.transpose(1, 2)) if form == "heads_first" else (k, v)


def paged(rng, lens, rows, max_pages, spare=2, first_of=None, prefix=None):
    """A page table that gives every sequence the pages of its tokens, in any order, whole pages of a prefix to all of its
    group; entries that nothing names are no pages at all."""
    need = [-(-n // rows) for n in lens]
    total = sum(need) + spare
    ids = list(rng.permutation(total))
    table = np.full((len(lens), max_pages), 10 ** 9, dtype=np.int64)
    for s, n in enumerate(need):
        shared = 0
        if first_of is not None and first_of[s] != s:
            shared = min(prefix[s] // rows, n, need[first_of[s]])
            table[s, :shared] = table[first_of[s], :shared]
        for j in range(shared, n):
            table[s, j] = ids.pop()
    table[:, 1::2][table[:, 1::2] == 10 ** 9] = -1
    return table, total


def put(pages, table, s, at, x):
    """Rows x of sequence s, tokens `at` on, into the pages."""
    import torch
    rows = pages.shape[1]
    t = at + np.arange(len(x))
    pages[torch.tensor(table[s, t // rows]).cuda(), torch.tensor(t % rows).cuda()] = x


@pytest.mark.parametrize("form", ["plain", "heads_first", "together"])
@pytest.mark.parametrize("hq,hkv,d,rows,layout", [(32, 8, 128, 16, 0), (4, 4, 64, 5, 1), (6, 2, 128, 64, 1), (8, 1, 64, 1, 0)])
@pytest.mark.parametrize("tokens", [1, 37])
def test_paged_append(ba, hq, hkv, d, rows, layout, form, tokens):
    import torch
    rng = np.random.default_rng(tokens + rows)
    heads = ba.Heads(hq, hkv, d, 500000.0, rope_layout=layout)
    n_seqs, max_pages = 5, 12
    lens = [max_pages * rows] * n_seqs
    table, n_pages = paged(rng, lens, rows, max_pages)
    kp, vp = pools(1, n_pages, rows, hkv, d, form)
    k_before, v_before = rand(61, *kp.shape), rand(62, *vp.shape)
    kp.copy_(k_before), vp.copy_(v_before)
    # every token a place of its own; some without a place
    flat = rng.permutation(n_seqs * max_pages * rows)[:tokens]
    seq, at = flat // (max_pages * rows), flat % (max_pages * rows)
    nowhere = set()
    if tokens > 20:
        at[3], seq[5], seq[6], at[7] = -1, n_seqs, -2, max_pages * rows
        table[seq[9], at[9] // rows] = n_pages  # (and whoever else lies in that page)
        nowhere = {3, 5, 6, 7} | {t for t in range(tokens) if t not in (3, 5, 6, 7) and table[seq[t], at[t] // rows] == n_pages}
    pos = rng.integers(0, 100000, tokens)
    cache = ba.PagedCache(kp, vp, ints(table))
    q, k, v = rand(63, tokens, hq, d), rand(64, tokens, hkv, d), rand(65, tokens, hkv, d)
    wq, wk = (rand(s, d, scale=0.3) + 1 for s in (66, 67))
    qo = torch.full_like(q, float("nan"))
    ba.ba_paged_append(heads, ba.HeadNorm(wq, wk, 1e-6), cache, q, k, v, qo, ints(at), ints(seq), ints(pos))
    expect_k, expect_v = k_before.clone(), v_before.clone()
    ref = rotate64(norm64(f64(k), f64(wk), 1e-6), pos, 500000.0, layout)
    got = np.zeros_like(ref)
    for t in range(tokens):
        if t in nowhere:
            got[t] = ref[t]
            continue
        page, row = int(table[seq[t], at[t] // rows]), int(at[t] % rows)
        got[t] = f64(kp[page, row])
        expect_k[page, row], expect_v[page, row] = kp[page, row], v[t]
    assert (np.abs(got - ref) <= 2e-6 * pair_size(ref, layout) + BF16_STEP * np.abs(ref)).all()
    assert torch.equal(kp, expect_k) and torch.equal(vp, expect_v)  # (nothing else has changed)
    ref = rotate64(norm64(f64(q), f64(wq), 1e-6), pos, 500000.0, layout)
    assert (np.abs(f64(qo) - ref) <= 2e-6 * pair_size(ref, layout) + BF16_STEP * np.abs(ref)).all()
    # neither norm nor rotation nor queries: a copy.  Rotation alone.
    ba.ba_paged_append(heads, None, cache, None, k, v, None, ints(at), ints(seq), None, ba.ROPE_NONE)
    for t in set(range(tokens)) - nowhere:
        assert torch.equal(kp[int(table[seq[t], at[t] // rows]), int(at[t] % rows)], k[t])
    ba.ba_paged_append(heads, None, cache, None, k, v, None, ints(at), ints(seq), ints(pos))
    ref = rotate64(f64(k), pos, 500000.0, layout)
    for t in set(range(tokens)) - nowhere:
        err = np.abs(f64(kp[int(table[seq[t], at[t] // rows]), int(at[t] % rows)]) - ref[t])
        assert (err <= 2e-6 * pair_size(ref, layout)[t] + BF16_STEP * np.abs(ref[t])).all()


def test_paged_append_of_a_cached_passage_is_its_reencoding(ba):
    """rope_pos = the shift: the bits of ba_reencode_positions; the sequence is the token's number without seq_of_token."""
    import torch
    heads = ba.Heads(8, 8, 128, 500000.0)
    k, v = rand(71, 200, 8, 128), rand(72, 200, 8, 128)
    turned = torch.empty_like(k)
    ba.ba_reencode_positions(heads, k, turned, [0], [0], [200], None, [1234], ba.REENC_SHIFT)
    kp, vp = pools(1, 20, 16, 8, 128)
    table = ints(np.random.default_rng(0).permutation(20)[None, :13])
    at = torch.arange(200, dtype=torch.int32, device="cuda")
    ba.ba_paged_append(heads, None, ba.PagedCache(kp, vp, table), None, k, v, None, at, torch.zeros_like(at), torch.full_like(at, 1234))
    where = table[0].long()[at.long() // 16], at.long() % 16
    assert torch.equal(kp[where], turned) and torch.equal(vp[where], v)
    one = ints(np.arange(13)[:, None])
    kp.fill_(0)
    ba.ba_paged_append(heads, None, ba.PagedCache(kp, vp, one), None, k[:13], v[:13], None, ints([3] * 13), None, None, ba.ROPE_NONE)
    assert torch.equal(kp[:13, 3], k[:13])


def attention_case(ba, seed, hq, hkv, d, rows, lens, nq=1, groups=None, form="plain", q_scale=1.0, max_len=None, holes=0, scale=0.0):
    """Runs ba_paged_attention on a fresh cache and checks every row.  groups: (members, prefix) one after the other.  Rows of pages
    without a token are NaN, so are pages that nothing names.  holes: that many pages are not there."""
    import torch
    rng = np.random.default_rng(seed)
    n = len(lens)
    max_len = max(max(lens), 1) if max_len is None else max_len
    heads = ba.Heads(hq, hkv, d, 10000.0, softmax_scale=scale)
    cu = prefix = None
    first_of, pre = list(range(n)), [0] * n
    if groups is not None:
        cu = np.concatenate([[0], np.cumsum([m for m, _ in groups])]).astype(np.int32)
        prefix = np.array([p for _, p in groups], dtype=np.int32)
        for g, (m, p) in enumerate(groups):
            for s in range(cu[g], cu[g + 1]):
                first_of[s], pre[s] = int(cu[g]), p
    table, n_pages = paged(rng, lens, rows, -(-max_len // rows) + 1, first_of=first_of, prefix=pre)
    kp, vp = pools(seed, n_pages, rows, hkv, d, form)
    keys = []
    for s in range(n):
        k, v = rand(seed * 1000 + 2 * s, lens[s], hkv, d), rand(seed * 1000 + 2 * s + 1, lens[s], hkv, d)
        if first_of[s] != s:  # the prefix is that of the first
            c = min(pre[s], lens[s], lens[first_of[s]])
            k[:c], v[:c] = keys[first_of[s]][0][:c], keys[first_of[s]][1][:c]
        keys.append((k, v))
        put(kp, table, s, 0, k), put(vp, table, s, 0, v)
    seen = [np.ones(m, dtype=bool) for m in lens]
    for _ in range(holes):
        s = int(rng.integers(n))
        if lens[s] == 0:
            continue
        page = int(rng.integers(-(-lens[s] // rows)))
        if page * rows < pre[s]:
            continue  # (a prefix is read from the first sequence's pages; holes there: a test of its own)
        table[s, page] = [-1, n_pages, -2 ** 31, 2 ** 31 - 1][int(rng.integers(4))]
        seen[s][page * rows:(page + 1) * rows] = False
    q = rand(seed * 1000 + 999, n * nq, hq, d, scale=q_scale)
    o, lse = torch.full_like(q, float("nan")), torch.full((n * nq, hq), float("nan"), device="cuda")
    ws = torch.empty(max(256, ba.ba_paged_attention_workspace_bytes(heads, n, nq, max_len, cu, prefix)), dtype=torch.uint8, device="cuda")
    ws.fill_(255)  # (NaN whatever it is taken for)
    cache = ba.PagedCache(kp, vp, ints(table.clip(-2 ** 31, 2 ** 31 - 1)))
    ba.ba_paged_attention(heads, cache, q, o, lse, ints(lens), max_len, cu, prefix, nq, ws)
    got, got_lse, q64 = f64(o), f64(lse), f64(q)
    sc = scale if scale > 0 else 1.0 / math.sqrt(d)
    for s in range(n):
        k, v = f64(keys[s][0]), f64(keys[s][1])
        for i in range(nq):
            row, end = s * nq + i, max(0, min(lens[s], max_len) - nq + i + 1)
            ok = seen[s][:end]
            ref, ref_lse, size = attend64(q64[row], k[:end][ok], v[:end][ok], sc)
            assert np.isfinite(got[row]).all(), (s, i)
            assert (np.abs(got[row] - ref) <= BF16_STEP * (np.abs(ref) + size) + 1e-5).all(), (s, i, np.abs(got[row] - ref).max())
            empty = np.isinf(ref_lse)
            assert (got_lse[row][empty] == -np.inf).all() and (got[row][empty] == 0).all()
            assert (np.abs(got_lse[row][~empty] - ref_lse[~empty]) <= 2e-5 * (1 + np.abs(ref_lse[~empty]))).all()
    o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
    ba.ba_paged_attention(heads, cache, q, o2, lse2, ints(lens), max_len, cu, prefix, nq, ws)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)  # the same call, the same bits
    return heads, cache, q, o, lse, keys, ws


GEOMETRIES = [(32, 8, 128), (4, 4, 64), (8, 2, 64), (16, 8, 128), (5, 1, 128), (7, 7, 64), (40, 2, 128)]


@pytest.mark.parametrize("hq,hkv,d", GEOMETRIES)
@pytest.mark.parametrize("rows", [16, 7, 128])
def test_paged_attention_alone(ba, hq, hkv, d, rows):
    attention_case(ba, 1 + rows, hq, hkv, d, rows, [1, 2, 31, 32, 33, 0, 64, 129, 300, 5])


@pytest.mark.parametrize("hq,hkv,d", GEOMETRIES)
@pytest.mark.parametrize("nq", [2, 5])
def test_paged_attention_of_several_tokens(ba, hq, hkv, d, nq):
    """Lengths below the number of tokens leave rows that see nothing."""
    attention_case(ba, 10 + nq, hq, hkv, d, 16, [0, 1, 2, 3, 4, 5, 33, 64, 66, 161], nq=nq)


@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (4, 4, 64), (8, 2, 64), (5, 1, 128)])
@pytest.mark.parametrize("rows,form", [(16, "plain"), (1, "plain"), (33, "heads_first"), (64, "together")])
def test_paged_attention_with_shared_prefixes(ba, hq, hkv, d, rows, form):
    groups = [(3, 70), (1, 40), (2, 0), (4, 129), (2, 32)]
    lens = [71, 130, 90, 55, 3, 60, 129, 140, 200, 131, 33, 40]
    attention_case(ba, 20 + rows, hq, hkv, d, rows, lens, groups=groups, form=form)


@pytest.mark.parametrize("nq", [1, 4])
def test_paged_attention_of_members_shorter_than_their_prefix(ba, nq):
    """Some have not reached the prefix's end, one is empty; the keys behind their end are none of theirs."""
    attention_case(ba, 31, 8, 2, 128, 16, [200, 100, 0, 3, 199, 205], nq=nq, groups=[(6, 190)])


@pytest.mark.parametrize("members,nq", [(5, 8), (70, 1), (45, 3)])
def test_paged_attention_of_many_rows(ba, members, nq):
    """More rows than a row tile has."""
    rng = np.random.default_rng(members)
    attention_case(ba, 40 + members, 8, 2, 64, 16, [150 + int(x) for x in rng.integers(nq, 40, members)], nq=nq, groups=[(members, 150)])


def test_paged_attention_of_many_tokens(ba):
    attention_case(ba, 51, 8, 1, 128, 16, [40, 17, 300], nq=40)


@pytest.mark.parametrize("rows", [1, 16, 100])
def test_paged_attention_over_missing_pages(ba, rows):
    attention_case(ba, 60 + rows, 8, 2, 128, rows, [200, 64, 33, 90], nq=2, holes=6)


def test_paged_attention_without_any_page(ba):
    import torch
    heads = ba.Heads(8, 2, 64)
    kp, vp = pools(1, 4, 16, 2, 64)
    q = rand(1, 3, 8, 64)
    o, lse = torch.full_like(q, 3.0), torch.full((3, 8), 3.0, device="cuda")
    table = ints([[-1, 99], [7, -5], [4, 4]])
    for cu, pre in ((None, None), ([0, 3], [20])):
        ws = torch.empty(max(256, ba.ba_paged_attention_workspace_bytes(heads, 3, 1, 32, cu, pre)), dtype=torch.uint8, device="cuda")
        ba.ba_paged_attention(heads, ba.PagedCache(kp, vp, table), q, o, lse, ints([32, 10, 30]), 32, cu, pre, 1, ws)
        assert (o == 0).all() and (lse == -math.inf).all()


def test_paged_attention_long_and_cut_into_parts(ba):
    attention_case(ba, 71, 8, 2, 128, 16, [9001, 1, 4097, 5000])
    attention_case(ba, 72, 4, 4, 64, 32, [7003, 6500, 6400], groups=[(3, 6399)])


@pytest.mark.parametrize("n,nq,max_len", [(1, 1, 384), (1, 1, 385), (3, 2, 383), (1, 5, 300), (70, 1, 1000), (70, 1, 1024), (70, 1, 1025),
                                          (20, 9, 500), (20, 13, 512), (20, 13, 600), (2, 30, 2100)])
def test_paged_attention_in_one_part_or_several(ba, n, nq, max_len):
    """Lengths around those where a call is cut, one of them the bound itself."""
    rng = np.random.default_rng(max_len + nq)
    attention_case(ba, 80 + n, 8, 2, 64, 32, [max_len] + [int(x) for x in rng.integers(0, max_len + 1, n - 1)], nq=nq)


@pytest.mark.parametrize("nq,rows", [(5, 1), (5, 16), (13, 48)])
def test_paged_attention_in_the_longest_parts(ba, nq, rows):
    """Many sequences under a long bound, few of which come near it."""
    rng = np.random.default_rng(nq)
    attention_case(ba, 90 + nq, 8, 2, 64, rows, [8200, 4097, 2049] + [int(x) for x in rng.integers(0, 30, 130)], nq=nq)


@pytest.mark.parametrize("groups", [None, [(3, 0)]])
def test_paged_attention_of_a_bound_of_zero(ba, groups):
    attention_case(ba, 79, 8, 2, 64, 16, [5, 0, 1], nq=2, groups=groups, max_len=0)


def test_paged_attention_lengths_beyond_the_bound_count_as_the_bound(ba):
    attention_case(ba, 73, 8, 2, 64, 16, [50, 10, 80], max_len=50)


@pytest.mark.parametrize("q_scale", [30.0, 0.0])
def test_paged_attention_of_large_scores(ba, q_scale):
    """Scores of some hundreds: the reference moves; and all alike: the mean."""
    attention_case(ba, 81, 8, 2, 128, 16, [500, 90], q_scale=q_scale)


def test_paged_attention_of_rising_scores(ba):
    """Each tile's scores tower over those before it."""
    import torch
    heads = ba.Heads(4, 1, 64, softmax_scale=1.0)
    n = 400
    k = torch.zeros(n, 1, 64, device="cuda")
    k[:, 0, 0] = torch.arange(n, device="cuda") // 16 * 16.0
    v = rand(82, n, 1, 64)
    q = torch.zeros(1, 4, 64, device="cuda")
    q[0, :, 0] = torch.tensor([1.0, -1.0, 8.0, -8.0])
    kp, vp = k.bfloat16().view(25, 16, 1, 64), v.view(25, 16, 1, 64)
    o = torch.empty(1, 4, 64, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    ba.ba_paged_attention(heads, ba.PagedCache(kp, vp, ints(np.arange(25)[None])), q.bfloat16(), o, None, ints([n]), n, None, None, 1, ws)
    ref, _, size = attend64(f64(q)[0], f64(kp).reshape(n, 1, 64), f64(v), 1.0)
    assert (np.abs(f64(o)[0] - ref) <= BF16_STEP * (np.abs(ref) + size) + 1e-5).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("what", ["k", "v"])
def test_paged_attention_keeps_what_a_row_does_not_see_out(ba, bad, what):
    """A token's own key or value reaches the rows that see it, and no other: not the earlier tokens of its sequence, not the other
    sequences, not a member that has not come that far in the prefix."""
    heads, cache, q, o, lse, keys, ws = attention_case(ba, 91, 8, 2, 64, 16, [100, 70, 90, 40], nq=3, groups=[(4, 60)])
    import torch
    lens, table = [100, 70, 90, 40], cache.page_table.cpu().numpy()
    pages = cache.k_pages if what == "k" else cache.v_pages
    pages[int(table[0, 98 // 16]), 98 % 16] = bad  # token 98 of sequence 0: rows 0 (token 97) does not see it, rows 1 and 2 do
    pages[int(table[0, 45 // 16]), 45 % 16] = bad  # token 45 of the prefix: sequence 3 (tokens 37 .. 39) does not see it
    o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
    cu, pre = np.array([0, 4], np.int32), np.array([60], np.int32)
    ba.ba_paged_attention(heads, cache, q, o2, lse2, ints(lens), 100, cu, pre, 3, ws)
    assert torch.equal(o2[9:], o[9:]) and torch.equal(lse2[9:], lse[9:])  # sequence 3
    if what == "v" or not bad < 0:
        assert not torch.isfinite(o2[:9].float()).all(-1).all(-1).any()  # everybody else sees token 45
    pages[int(table[0, 45 // 16]), 45 % 16] = keys[0][0 if what == "k" else 1][45]
    ba.ba_paged_attention(heads, cache, q, o2, lse2, ints(lens), 100, cu, pre, 3, ws)
    assert torch.equal(o2[:1], o[:1]) and torch.equal(o2[3:], o[3:]) and torch.equal(lse2[3:], lse[3:])


def test_paged_attention_of_more_groups_than_a_launch_takes(ba):
    groups = [(2, 20)] * 130 + [(1, 0)] * 3
    lens = [21 + s % 9 for s in range(263)]
    attention_case(ba, 101, 4, 2, 64, 16, lens, groups=groups)


def test_paged_attention_beyond_32_bit_offsets(ba):
    """Pages that begin 4 GiB and more behind the first, rows far apart in them."""
    import torch
    heads = ba.Heads(8, 2, 128)
    n_pages, rows = 20, 16
    kp, vp = (torch.empty(n_pages, rows, 2, 128 * 128 * 256, dtype=torch.bfloat16, device="cuda")[..., :128] for _ in range(2))
    assert kp.stride(0) * 2 * (n_pages - 1) > 2 ** 32 and kp.stride(1) < 2 ** 24
    k, v = rand(111, 100, 2, 128), rand(112, 100, 2, 128)
    q = rand(113, 2, 8, 128)
    table = np.array([[19, 1, 18, 0, 16, 5, 2], [19, 1, 18, 0, 16, 5, 2]])
    cache = ba.PagedCache(kp, vp, ints(table))
    at = torch.arange(100, dtype=torch.int32, device="cuda")
    ba.ba_paged_append(heads, None, cache, None, k, v, None, at, torch.zeros_like(at), None, ba.ROPE_NONE)
    for cu, pre in ((None, None), ([0, 2], [64])):
        o = torch.empty_like(q)
        ws = torch.empty(max(256, ba.ba_paged_attention_workspace_bytes(heads, 2, 1, 100, cu, pre)), dtype=torch.uint8, device="cuda")
        ba.ba_paged_attention(heads, cache, q, o, None, ints([100, 77]), 100, cu, pre, 1, ws)
        for s, n in ((0, 100), (1, 77)):
            ref, _, size = attend64(f64(q)[s], f64(k)[:n], f64(v)[:n], 1 / math.sqrt(128))
            assert (np.abs(f64(o)[s] - ref) <= BF16_STEP * (np.abs(ref) + size) + 1e-5).all()


def test_strided_rows_and_another_stream(ba):
    """q and o as every second token and with heads apart, on a stream of their own."""
    import torch
    heads, cache, q, o, lse, _, _ = attention_case(ba, 121, 8, 2, 128, 16, [40, 170, 90], nq=2)
    wide_q = torch.zeros(12, 10, 128, dtype=torch.bfloat16, device="cuda")
    wide_o = torch.full((12, 8, 256), 5.0, dtype=torch.bfloat16, device="cuda")
    wide_q[::2, 1:9] = q
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ws = torch.empty(max(256, ba.ba_paged_attention_workspace_bytes(heads, 3, 2, 170)), dtype=torch.uint8, device="cuda")
        ba.ba_paged_attention(heads, cache, wide_q[::2, 1:9], wide_o[::2, :, :128], None, ints([40, 170, 90]), 170, None, None, 2, ws)
    stream.synchronize()
    assert torch.equal(wide_o[::2, :, :128], o) and (wide_o[1::2] == 5).all() and (wide_o[::2, :, 128:] == 5).all()


def test_a_captured_decoding_step(ba):
    """Norm, append and attention captured once and replayed with new tokens and lengths, against the same calls made eagerly."""
    import torch
    hq, hkv, d, rows, prefix, n_seqs = 8, 2, 64, 16, 100, 5
    heads = ba.Heads(hq, hkv, d, 10000.0)
    norm = ba.HeadNorm(rand(1, d) + 1, rand(2, d) + 1)
    max_len = 160
    rng = np.random.default_rng(3)
    table, n_pages = paged(rng, [max_len] * n_seqs, rows, 10, first_of=[0] * n_seqs, prefix=[prefix] * n_seqs)
    caches = []
    for _ in range(2):
        kp, vp = rand(4, n_pages, rows, hkv, d), rand(5, n_pages, rows, hkv, d)
        caches.append(ba.PagedCache(kp, vp, ints(table)))
    cu, pre = np.array([0, n_seqs], np.int32), np.array([prefix], np.int32)
    ws = torch.empty(ba.ba_paged_attention_workspace_bytes(heads, n_seqs, 1, max_len, cu, pre), dtype=torch.uint8, device="cuda")
    q, k, v = rand(6, n_seqs, hq, d), rand(7, n_seqs, hkv, d), rand(8, n_seqs, hkv, d)
    lens = ints([prefix + 1 + s for s in range(n_seqs)])
    at = lens - 1
    q_rot, o, lse = torch.empty_like(q), torch.empty_like(q), torch.empty(n_seqs, hq, device="cuda")

    def step(cache):
        ba.ba_paged_append(heads, norm, cache, q, k, v, q_rot, at)
        ba.ba_paged_attention(heads, cache, q_rot, o, lse, lens, max_len, cu, pre, 1, ws)

    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(caches[0])
    for turn in range(6):
        q.copy_(rand(100 + turn, n_seqs, hq, d)), k.copy_(rand(200 + turn, n_seqs, hkv, d)), v.copy_(rand(300 + turn, n_seqs, hkv, d))
        o.fill_(9), lse.fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        kept = o.clone(), lse.clone()
        step(caches[1])
        assert torch.equal(kept[0], o) and torch.equal(kept[1], lse)
        assert torch.equal(caches[0].k_pages, caches[1].k_pages) and torch.equal(caches[0].v_pages, caches[1].v_pages)
        lens += 1
        at += 1


@pytest.mark.parametrize("tokens", [6000, 12000])
def test_calls_larger_than_the_caches_give_the_bits_of_their_parts(ba, tokens):
    """From 96 MB on stores go past the caches, from 192 MB on loads as well; parts of 2,500 tokens lie below, of 700 in the
    kernel for few tokens."""
    import torch
    heads = ba.Heads(32, 8, 128, 500000.0)
    gen = torch.Generator(device="cuda").manual_seed(1)
    new = lambda h: torch.randn(tokens, h, 128, generator=gen, device="cuda").bfloat16()  # noqa: E731
    q, k, gq, gk = new(32), new(8), new(32), new(8)
    norm = ba.HeadNorm(rand(1, 128) + 1, rand(2, 128) + 1)
    pos = torch.arange(tokens, dtype=torch.int32, device="cuda") * 3
    whole = [torch.empty_like(x) for x in (q, k, q, k)]
    gains = torch.empty(2, 2, 128, device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    ba.ba_norm_rotate(heads, norm, q, k, whole[0], whole[1], pos)
    ba.ba_norm_rotate_backward(heads, norm, q, k, gq, gk, whole[2], whole[3], gains[0, 0], gains[0, 1], pos, ba.ROPE_APPLY, ws)
    for size in (2500, 700):
        sums = torch.zeros(2, 128, dtype=torch.float64, device="cuda")
        for a in range(0, tokens, size):
            s = slice(a, min(a + size, tokens))
            part = [torch.empty_like(x[s]) for x in (q, k, q, k)]
            ba.ba_norm_rotate(heads, norm, q[s], k[s], part[0], part[1], pos[s])
            ba.ba_norm_rotate_backward(heads, norm, q[s], k[s], gq[s], gk[s], part[2], part[3], gains[1, 0], gains[1, 1], pos[s], ba.ROPE_APPLY, ws)
            assert all(torch.equal(x, y[s]) for x, y in zip(part, whole))
            sums += gains[1].double()
        # (sums of 100,000 terms and more of random sign, in 32 bits within a workgroup: some hundreds of 2^-24 of their length)
        assert ((gains[0].double() - sums).norm(dim=1) <= 1e-5 * sums.norm(dim=1)).all()
    # keys and values of as many bytes into pages
    n = tokens * 40 // 16
    k, v = torch.randn(2, n, 8, 128, generator=gen, device="cuda").bfloat16()
    at = torch.arange(n, dtype=torch.int32, device="cuda")
    pools = torch.zeros(4, -(-n // 16), 16, 8, 128, dtype=torch.bfloat16, device="cuda")
    table = torch.arange(pools.shape[1], dtype=torch.int32, device="cuda")[None]
    ba.ba_paged_append(heads, norm, ba.PagedCache(pools[0], pools[1], table), None, k, v, None, at, torch.zeros_like(at))
    for a in range(0, n, 4000):
        s = slice(a, min(a + 4000, n))
        ba.ba_paged_append(heads, norm, ba.PagedCache(pools[2], pools[3], table), None, k[s], v[s], None, at[s], torch.zeros_like(at[s]))
    assert torch.equal(pools[0], pools[2]) and torch.equal(pools[1], pools[3])
