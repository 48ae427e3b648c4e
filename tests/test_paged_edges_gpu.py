"""What the paged attention and the head norms do at their edges: values that are not finite, outputs in place or among other tensors'
heads, and the forms of the walks that the other tests do not reach.  Tolerances as in test_paged_gpu.py: a result's rounding
to bf16, the rounding of the probabilities to bf16, that of the parts of a call to fp16 (2^-11 of sum p |v|, a small share of
what the probabilities are allowed)."""
import math

import numpy as np
import pytest

from test_paged_gpu import BF16_STEP, attend64, attention_case, f64, ints, paged, pools, put, rand

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ba():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2409_15355_amd import binding
    binding.load()
    return binding


def workspace(ba, heads, n, nq, max_len, cu=None, prefix=None):
    import torch
    return torch.empty(max(256, ba.ba_paged_attention_workspace_bytes(heads, n, nq, max_len, cu, prefix)), dtype=torch.uint8, device="cuda")


def close(got, ref, size):
    return (np.abs(got - ref) <= BF16_STEP * (np.abs(ref) + size) + 1e-5).all()


# ---- values that are not finite -----------------------------------------------------------------------------------
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("hq,hkv,d,nq", [(8, 2, 128, 1), (8, 2, 64, 5), (8, 2, 128, 12)])
@pytest.mark.parametrize("shared", [False, True])
def test_a_value_that_is_not_finite_stays_in_its_dimension(ba, hq, hkv, d, nq, bad, shared):
    """One element of one value row, in a call of many parts; the others are of a size that fp16 does not hold when it is brought to
    2^14 by mistake."""
    import torch
    n, lens, rows, at, dim = 2, [2000, 2000], 16, 500, 5
    heads = ba.Heads(hq, hkv, d, 10000.0)
    k, v = rand(1, 2000, hkv, d), rand(2, 2000, hkv, d) * 3 + 10
    q = rand(3, n * nq, hq, d)
    v[at, 0, dim] = bad
    kp, vp = k.view(125, rows, hkv, d), v.view(125, rows, hkv, d)
    cache = ba.PagedCache(kp, vp, ints(np.tile(np.arange(125), (n, 1))))
    cu, prefix = ([0, 2], [1900]) if shared else (None, None)
    o = torch.full_like(q, 7.0)
    ba.ba_paged_attention(heads, cache, q, o, None, ints(lens), 2000, cu, prefix, nq, workspace(ba, heads, n, nq, 2000, cu, prefix))
    v64 = f64(v)
    v64[at, 0, dim] = 0.0
    for row in range(n * nq):
        end = 2000 - nq + row % nq + 1
        ref, _, size = attend64(f64(q)[row], f64(k)[:end], v64[:end], 1 / math.sqrt(d))
        got = f64(o)[row]
        hit = np.zeros_like(got, dtype=bool)
        hit[: hq // hkv, dim] = True
        assert (np.isnan(got[hit]).all() if math.isnan(bad) else (got[hit] == bad).all())
        assert np.isfinite(got[~hit]).all() and close(got[~hit], ref[~hit], size[~hit])


# ---- one row's bits and another's scores ----------------------------------------------------------------------------
@pytest.mark.parametrize("hq", [4, 20, 40])
def test_no_score_changes_the_bits_of_another_row(ba, hq):
    """Row 0's exponentials come near the bound from which a row's reference is raised, lane by lane, and add up to more; row 1's pass it by
    far, or do not.  128 sequences and more: calls in one part, so that these keys are not the first of theirs."""
    import torch
    d, n, length = 64, 130, 96
    heads = ba.Heads(hq, 1, d, softmax_scale=1.0)
    k = torch.zeros(length, 1, d)
    if hq <= 32:
        k[[64, 68, 72, 76], 0, 0] = 27.5   # 2^39.7 in each of four lanes
    else:
        k[[64, 68], 0, 0] = 27.5           # ... of two
    k[65, 0, 1] = 60.0
    k, v = k.bfloat16().cuda(), rand(5, length, 1, d)
    kp, vp = k.view(6, 16, 1, d), v.view(6, 16, 1, d)
    cache = ba.PagedCache(kp, vp, ints(np.tile(np.arange(6), (n, 1))))
    assert ba.ba_paged_attention_workspace_bytes(heads, n, 1, length) == 0  # (one part)
    outs = []
    for other in (0.0, 1.0):
        q = torch.zeros(n, hq, d, device="cuda", dtype=torch.bfloat16)
        q[:, 0, 0] = 1.0
        q[:, 1, 1] = other
        o, lse = torch.empty_like(q), torch.empty(n, hq, device="cuda")
        ba.ba_paged_attention(heads, cache, q, o, lse, ints([length] * n), length)
        ref, _, size = attend64(f64(q)[0], f64(k), f64(v), 1.0)
        assert close(f64(o)[0], ref, size)
        outs.append((o[:, 0].clone(), lse[:, 0].clone()))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


# ---- where outputs lie ----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("nq,lens,groups", [(1, [200, 33, 90], None), (3, [9000, 1, 4097], None), (13, [300, 40, 77], None), (4, [310, 305, 400], [(3, 300)])])
def test_attention_in_place_of_its_queries(ba, nq, lens, groups):
    import torch
    heads, cache, q, o, lse, _, ws = attention_case(ba, 130 + nq, 8, 2, 128, 16, lens, nq=nq, groups=groups)
    cu, prefix = (None, None) if groups is None else ([0, 3], [groups[0][1]])
    same = q.clone()
    ba.ba_paged_attention(heads, cache, same, same, None, ints(lens), max(lens), cu, prefix, nq, ws)
    assert torch.equal(same, o)
    # heads of both side by side in one tensor
    both = torch.full((len(q), 8, 2, 128), 3.0, dtype=q.dtype, device="cuda")
    both[:, :, 0] = q
    ba.ba_paged_attention(heads, cache, both[:, :, 0], both[:, :, 1], None, ints(lens), max(lens), cu, prefix, nq, ws)
    assert torch.equal(both[:, :, 1], o) and torch.equal(both[:, :, 0], q)


def test_attention_does_not_write_over_what_it_reads(ba):
    import torch
    heads, cache, q, _, _, _, ws = attention_case(ba, 141, 8, 2, 128, 16, [100, 60], nq=2)
    room = torch.zeros(6, 8, 128, dtype=q.dtype, device="cuda")
    room[:4] = q
    for o in (room[1:5], cache.k_pages.view(-1)[: 4 * 8 * 128].view(4, 8, 128)):
        before = o.clone()
        with pytest.raises(ba.BaError, match="overlap"):
            ba.ba_paged_attention(heads, cache, room[:4], o, None, ints([100, 60]), 100, None, None, 2, ws)
        assert torch.equal(o.view(torch.int16), before.view(torch.int16))


@pytest.mark.parametrize("tokens", [1, 50, 3000])
def test_heads_of_query_key_and_value_one_after_the_other(ba, tokens):
    """A projection laid out [tokens, heads, 3, D]: the heads of one tensor lie between those of the others, and each can be normed
    where it lies, or appended."""
    import torch
    hq, d = 6, 64
    heads = ba.Heads(hq, hq, d, 10000.0)
    qkv = rand(151, tokens, hq, 3, d)
    before = qkv.clone()
    w = rand(152, d, dtype="f32") + 1
    norm = ba.HeadNorm(w, w)
    ref = [torch.empty(tokens, hq, d, dtype=qkv.dtype, device="cuda") for _ in range(2)]
    ba.ba_norm_rotate(heads, norm, before[:, :, 0], before[:, :, 1], *ref)
    ba.ba_norm_rotate(heads, norm, qkv[:, :, 0], qkv[:, :, 1], qkv[:, :, 0], qkv[:, :, 1])
    assert torch.equal(qkv[:, :, 0], ref[0]) and torch.equal(qkv[:, :, 1], ref[1]) and torch.equal(qkv[:, :, 2], before[:, :, 2])
    g = rand(153, tokens, hq, 3, d)
    got, back = g.clone(), [torch.empty_like(x) for x in ref]
    ws = torch.empty(ba.ba_norm_rotate_backward_workspace_bytes(heads, tokens), dtype=torch.uint8, device="cuda")
    ba.ba_norm_rotate_backward(heads, norm, before[:, :, 0], before[:, :, 1], g[:, :, 0], g[:, :, 1], *back, ws=ws)
    ba.ba_norm_rotate_backward(heads, norm, before[:, :, 0], before[:, :, 1], got[:, :, 0], got[:, :, 1], got[:, :, 0], got[:, :, 1], ws=ws)
    assert torch.equal(got[:, :, 0], back[0]) and torch.equal(got[:, :, 1], back[1]) and torch.equal(got[:, :, 2], g[:, :, 2])
    kp, vp = pools(1, -(-tokens // 16), 16, hq, d)
    cache = ba.PagedCache(kp, vp, torch.arange(len(kp), dtype=torch.int32, device="cuda")[None])
    at = torch.arange(tokens, dtype=torch.int32, device="cuda")
    qkv.copy_(before)
    ba.ba_paged_append(heads, norm, cache, qkv[:, :, 0], qkv[:, :, 1], qkv[:, :, 2], qkv[:, :, 0], at, torch.zeros_like(at))
    assert torch.equal(qkv[:, :, 0], ref[0]) and torch.equal(qkv[:, :, 1:], before[:, :, 1:])
    assert torch.equal(kp.reshape(-1, hq, d)[:tokens], ref[1]) and torch.equal(vp.reshape(-1, hq, d)[:tokens], before[:, :, 2])
    # a row further on the heads do meet
    if tokens > 1:
        flat = before.view(-1)
        moved = flat[3 * d * hq:].as_strided((tokens - 1, hq, d), (3 * d * hq, 3 * d, 1))
        with pytest.raises(ba.BaError, match="overlap"):
            ba.ba_norm_rotate(heads, norm, before[:-1, :, 0], None, moved, None)


@pytest.mark.parametrize("form", ["rows", "heads"])
def test_pages_with_keys_and_values_beside_each_other(ba, form):
    """[pages, rows, 2, heads, D] and [pages, rows, heads, 2, D]; attention may read one pool as both."""
    import torch
    hq, hkv, d, rows, n = 8, 2, 64, 16, 100
    heads = ba.Heads(hq, hkv, d, 10000.0)
    k, v, q = rand(171, n, hkv, d), rand(172, n, hkv, d), rand(173, 1, hq, d)
    at = torch.arange(n, dtype=torch.int32, device="cuda")
    table = ints(np.random.default_rng(2).permutation(7)[None])
    outs = []
    for together in (False, True):
        kv = torch.zeros((2, 7, rows, hkv, d) if not together else (7, rows, 2, hkv, d) if form == "rows" else (7, rows, hkv, 2, d), dtype=k.dtype, device="cuda")
        kp, vp = kv.unbind(0 if not together else 2 if form == "rows" else 3)
        ba.ba_paged_append(heads, None, ba.PagedCache(kp, vp, table), None, k, v, None, at, torch.zeros_like(at))
        for pair in ((kp, vp), (vp, vp)):
            o = torch.empty_like(q)
            ba.ba_paged_attention(heads, ba.PagedCache(*pair, table), q, o, None, ints([n]), n, ws=workspace(ba, heads, 1, 1, n))
            outs.append(o)
    assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[3])
    ref, _, size = attend64(f64(q)[0], f64(v), f64(v), 1 / math.sqrt(d))
    assert close(f64(outs[1])[0], ref, size)


def test_queries_and_keys_of_different_token_counts_are_refused(ba):
    import torch
    heads = ba.Heads(8, 2, 64)
    q, k = rand(161, 5, 8, 64), rand(162, 7, 2, 64)
    with pytest.raises(ValueError, match="tokens"):
        ba.ba_norm_rotate(heads, ba.HeadNorm(), q, k, torch.empty_like(q), torch.empty_like(k))
    with pytest.raises(ValueError, match="tokens"):
        ba.ba_norm_rotate_backward(heads, ba.HeadNorm(), q, k, q, k, torch.empty_like(q), torch.empty_like(k), ws=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))


# ---- forms of the walks ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("hq,hkv,d,nq", [(8, 2, 64, 13), (8, 1, 128, 40)])
@pytest.mark.parametrize("rows", [1, 7, 33, 100])
def test_many_rows_over_pages_of_any_length(ba, hq, hkv, d, nq, rows):
    attention_case(ba, 200 + rows, hq, hkv, d, rows, [40, 17, 300, 0, 5, 700], nq=nq)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows,form", [(7, "plain"), (48, "heads_first"), (33, "together")])
def test_many_rows_over_a_prefix_in_pages_of_any_length(ba, d, rows, form):
    attention_case(ba, 210 + rows, 8, 2, d, rows, [170, 163, 400, 151, 180, 90], nq=8, groups=[(5, 150), (1, 40)], form=form)


@pytest.mark.parametrize("nq", [5, 13])
@pytest.mark.parametrize("rows", [16, 7])
def test_missing_pages_of_many_rows(ba, nq, rows):
    attention_case(ba, 220 + rows, 8, 2, 128, rows, [200, 64, 33, 90, 700], nq=nq, holes=9)


@pytest.mark.parametrize("nq", [5, 13])
@pytest.mark.parametrize("q_scale", [30.0, 0.0])
def test_large_scores_of_many_rows(ba, nq, q_scale):
    attention_case(ba, 230 + nq, 8, 2, 128, 16, [500, 90], nq=nq, q_scale=q_scale)


@pytest.mark.parametrize("hq", [20, 40, 200])
def test_rising_scores_of_many_rows(ba, hq):
    """Each tile's scores tower over those before it, for some rows."""
    import torch
    heads = ba.Heads(hq, 1, 64, softmax_scale=1.0)
    n = 400
    k = torch.zeros(n, 1, 64, device="cuda")
    k[:, 0, 0] = torch.arange(n, device="cuda") // 16 * 16.0
    kp, v = k.bfloat16().view(25, 16, 1, 64), rand(240, n, 1, 64)
    q = torch.zeros(1, hq, 64, device="cuda")
    q[0, :, 0] = torch.tensor([1.0, -1.0, 8.0, -8.0, 0.0], device="cuda").repeat(hq // 5)
    o, lse = torch.empty(1, hq, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(1, hq, device="cuda")
    cache = ba.PagedCache(kp, v.view(25, 16, 1, 64), ints(np.arange(25)[None]))
    ba.ba_paged_attention(heads, cache, q.bfloat16(), o, lse, ints([n]), n, ws=workspace(ba, heads, 1, 1, n))
    ref, ref_lse, size = attend64(f64(q)[0], f64(k.bfloat16()), f64(v), 1.0)
    assert close(f64(o)[0], ref, size) and (np.abs(f64(lse)[0] - ref_lse) <= 2e-5 * (1 + np.abs(ref_lse))).all()


@pytest.mark.parametrize("nq", [1, 3, 9])
@pytest.mark.parametrize("rows", [16, 10])
def test_missing_pages_of_a_prefix(ba, nq, rows):
    """They are missing for every member; what another member's table has in their place does not matter."""
    import torch
    hq, hkv, d, prefix, lens = 8, 2, 128, 150, [190, 170, 100, 151]
    heads = ba.Heads(hq, hkv, d, 10000.0)
    table, n_pages = paged(np.random.default_rng(7), lens, rows, 20, first_of=[0] * 4, prefix=[prefix] * 4)
    kp, vp = pools(1, n_pages, rows, hkv, d)
    keys = []
    for s, n in enumerate(lens):
        k, v = rand(250 + s, n, hkv, d), rand(260 + s, n, hkv, d)
        if s:
            c = min(prefix, n)
            k[:c], v[:c] = keys[0][0][:c], keys[0][1][:c]
        keys.append((k, v))
        put(kp, table, s, 0, k), put(vp, table, s, 0, v)
    seen = np.ones(200, dtype=bool)
    for page, to in ((1, -1), (2, n_pages), (6, 2 ** 31 - 1)):
        table[0, page] = to
        seen[page * rows:(page + 1) * rows] = False
    q = rand(270, 4 * nq, hq, d)
    o, lse = torch.empty_like(q), torch.empty(4 * nq, hq, device="cuda")
    cache = ba.PagedCache(kp, vp, ints(table.clip(-2 ** 31, 2 ** 31 - 1)))
    ba.ba_paged_attention(heads, cache, q, o, lse, ints(lens), 200, [0, 4], [prefix], nq, workspace(ba, heads, 4, nq, 200, [0, 4], [prefix]))
    for s in range(4):
        for i in range(nq):
            row, end = s * nq + i, lens[s] - nq + i + 1
            ok = seen[:end]
            ref, ref_lse, size = attend64(f64(q)[row], f64(keys[s][0])[:end][ok], f64(keys[s][1])[:end][ok], 1 / math.sqrt(d))
            assert close(f64(o)[row], ref, size)
            assert (np.abs(f64(lse)[row] - ref_lse) <= 2e-5 * (1 + np.abs(ref_lse))).all()


@pytest.mark.parametrize("nq,rows,groups", [(1, 16, None), (7, 48, None), (9, 16, None), (9, 20, None), (4, 64, [(12, 60), (4, 0)])])
def test_calls_that_read_past_the_caches(ba, nq, rows, groups):
    """By the bound on their lengths: 96 MB of keys and values and more.  The sequences are short."""
    rng = np.random.default_rng(nq)
    low = 60 if groups else 0
    assert 16 * 3000 * 8 * 128 * 4 > 1.5 * 96 * 2 ** 20
    attention_case(ba, 280 + nq, 32, 8, 128, rows, [low + int(x) for x in rng.integers(0, 70, 15)] + [400], nq=nq, groups=groups, max_len=3000)


def test_the_python_half_of_the_face_makes_the_same_calls(ba, monkeypatch):
    """Norms, their backward, appends and attention without the native half that takes their arguments apart: the same bits."""
    import torch
    hq, hkv, d, tokens = 8, 2, 64, 40
    heads = ba.Heads(hq, hkv, d, 10000.0)
    norm = ba.HeadNorm(rand(301, d) + 1, rand(302, d) + 1, 1e-5)
    q, k, v = rand(303, tokens, hq, d), rand(304, tokens, hkv, d), rand(305, tokens, hkv, d)
    pos, at, seq = ints(np.arange(tokens) * 7), ints(np.arange(tokens) // 4), ints(np.arange(tokens) % 4)
    calls = []
    for native in (True, False):
        if not native:
            monkeypatch.setattr(ba, "_native", ba._NoNative())
        new = lambda x: torch.zeros_like(x)  # noqa: E731
        out = [new(q), new(k), new(q), new(k), torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda"), new(q)]
        ba.ba_norm_rotate(heads, norm, q, k, out[0], out[1], pos)
        ws = torch.empty(ba.ba_norm_rotate_backward_workspace_bytes(heads, tokens), dtype=torch.uint8, device="cuda")
        ba.ba_norm_rotate_backward(heads, norm, q, k, out[0], out[1], out[2], out[3], out[4], out[5], pos, ba.ROPE_APPLY, ws)
        kp, vp = torch.zeros(2, 8, 4, hkv, d, dtype=torch.bfloat16, device="cuda")
        cache = ba.PagedCache(kp, vp, ints(np.arange(8).reshape(4, 2)[:, ::-1].copy()))
        keep = at[:32], seq[:32], pos[:32]
        ba.ba_paged_append(heads, norm, cache, q[:32], k[:32], v[:32], out[6], *keep)
        o, lse = new(q[:8]), torch.zeros(8, hq, device="cuda")
        ba.ba_paged_attention(heads, cache, q[:8], o, lse, ints([8, 7, 3, 0]), 8, [0, 4], [3], 2, workspace(ba, heads, 4, 2, 8, [0, 4], [3]))
        calls.append(out + [kp, vp, o, lse])
        assert all(bool(x.any()) for x in calls[-1])
    assert all(torch.equal(a, b) for a, b in zip(*calls))
