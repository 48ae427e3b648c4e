"""examples/answer_questions.py at a small size against 64 bits: norm, append and attention as a program uses them together."""
import importlib.util
import math
import os

import numpy as np
import pytest

from test_paged_gpu import BF16_STEP, attend64, f64, norm64, norm_back64, pair_size, rotate64

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "answer_questions.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("answer_questions", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("heads,layout,lens,questions,question,steps,rows",
                         [((8, 2, 64), 0, [37, 80, 15], 5, 7, 6, 16), ((4, 4, 64), 1, [64, 64], 1, 1, 3, 32), ((16, 2, 128), 1, [50, 41, 9, 33], 12, 9, 4, 16)])
def test_answers(example, heads, layout, lens, questions, question, steps, rows):
    hq, hkv, d = heads
    layer = example.Layer(hq, hkv, d, 10000.0, layout, seed=3)
    got = example.answer(layer, lens, questions, question, steps, rows)
    cache, context = got["cache"], got["context"]
    table = cache.page_table.cpu().numpy()
    k_pages, v_pages = f64(cache.k_pages), f64(cache.v_pages)

    def rows_of(pages, s, n):
        t = np.arange(n)
        return pages[table[s, t // rows], t % rows]

    # the passages' keys in every question's pages: the cached ones turned by their passage's shift, rounded once more
    shift = np.repeat(np.concatenate([[0], np.cumsum(lens)[:-1]]), lens)
    ref = rotate64(f64(got["k_cached"]), shift, 10000.0, layout)
    for s in range(questions):
        err = np.abs(rows_of(k_pages, s, context) - ref)
        assert (err <= 2e-6 * pair_size(ref, layout) + BF16_STEP * np.abs(ref)).all()
    for q, o, lse, ends in got["done"]:
        q, o, lse, ends = f64(q), f64(o), f64(lse), ends.cpu().numpy()
        nq = len(q) // questions
        for s in range(questions):
            for i in range(nq):
                seen = ends[s] - nq + i + 1
                want, want_lse, size = attend64(q[s * nq + i], rows_of(k_pages, s, seen), rows_of(v_pages, s, seen), 1 / math.sqrt(d))
                assert (np.abs(o[s * nq + i] - want) <= BF16_STEP * (np.abs(want) + size) + 1e-5).all()
                assert (np.abs(lse[s * nq + i] - want_lse) <= 2e-5 * (1 + np.abs(want_lse))).all()


def test_a_fine_tune_step(example):
    """The gains' gradients against the formula on the gradients that Block-attention's backward pass returns, and against differences
    of the loss in 64 bits.  The bf16 roundings on the way (normed rows, probabilities, outputs, gradients: 2^-8 each at most, of
    random sign) bound the second: 3 % of the gradient's length."""
    import torch

    import oracle
    from paper_2409_15355_amd import binding as ba
    layer = example.Layer(4, 2, 64, 10000.0, seed=5)
    lens = [30, 41, 17]
    T = sum(lens)
    q, k, v = (x.contiguous() for x in layer.qkv(T))
    d_out = layer.randn(T, 4, 64)
    o, dq, dk, dv, gq, gk = example.tune(layer, lens, q, k, v, d_out)
    # the last pass alone
    offs, cu_blk = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32), np.array([0, 3], np.int32)
    q_n, k_n, lse = torch.empty_like(q), torch.empty_like(k), torch.empty(T, 4, device="cuda")
    ba.ba_norm_rotate(layer.heads, layer.norm, q, k, q_n, k_n, None, ba.ROPE_NONE)
    ws = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    o2 = torch.empty_like(o)
    ba.ba_block_attention_prompts(layer.heads, q_n, k_n, v, o2, None, lse, cu_blk, offs, ba.ROPE_APPLY, ws)
    assert torch.equal(o, o2)
    a, b, c = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    ba.ba_block_attention_prompts_backward(layer.heads, q_n, k_n, v, o, lse, d_out, a, b, c, cu_blk, offs, ws)
    for x, w, g, dx, dw in ((q, layer.q_gain, a, dq, gq), (k, layer.k_gain, b, dk, gk)):
        ref, ref_w, size, size_w = norm_back64(f64(x), f64(w), 1e-6, f64(g))
        assert (np.abs(f64(dx) - ref) <= 8e-6 * size + BF16_STEP * np.abs(ref)).all()
        assert (np.abs(f64(dw) - ref_w) <= 4e-6 * size_w).all()
    # differences, all in 64 bits
    th, t = oracle.theta(10000.0, 64), np.arange(T)
    blk = np.repeat(np.arange(3), lens)
    mask = (t[None, :] <= t[:, None]) & ((blk[None, :] == blk[:, None]) | (blk[:, None] == 2))
    assert np.allclose(th, 10000.0 ** (-2.0 * np.arange(32) / 64))

    def loss(wq, wk):
        qr, kr = (rotate64(norm64(f64(x), w, 1e-6), t, 10000.0, 0) for x, w in ((q, wq), (k, wk)))
        s = np.einsum("thd,shd->hts", qr, np.repeat(kr, 2, axis=1)) / 8.0
        p = np.exp(np.where(mask[None], s, -np.inf) - s.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        return float((np.einsum("hts,shd->thd", p, np.repeat(f64(v), 2, axis=1)) * f64(d_out)).sum())

    rng, wq, wk = np.random.default_rng(7), f64(layer.q_gain), f64(layer.k_gain)
    for _ in range(4):
        eq, ek = rng.standard_normal(64), rng.standard_normal(64)
        h = 1e-4
        got = (loss(wq + h * eq, wk + h * ek) - loss(wq - h * eq, wk - h * ek)) / (2 * h)
        want = (f64(gq) * eq).sum() + (f64(gk) * ek).sum()
        assert abs(got - want) <= 0.03 * math.hypot(np.linalg.norm(f64(gq)), np.linalg.norm(f64(gk)))
