"""The calls of long caches as a program may make them besides the plain one: without the native half of the Python face, on two streams at once, with heads far
apart.  Tolerances as in test_long_cache_gpu.py."""
import numpy as np
import pytest

import test_long_cache_gpu as forms
from test_long_cache_gpu import ba, f64, ints, kept64, lse64, rand, weights64  # noqa: F401

pytestmark = pytest.mark.gpu


class Step:
    """Weights, bounds, selection, attention over the selection and eviction of one batch, each into tensors of its own."""

    def __init__(self, ba, seed, hq, hkv, d, rows, lens, nq, n_select, keep):  # noqa: F811
        import torch
        self.ba, self.heads, self.nq, self.n_select, self.keep, self.rows = ba, ba.Heads(hq, hkv, d), nq, n_select, keep, rows
        self.pool, self.n, self.max_len = forms.Pool(ba, seed, lens, hkv, d, rows), len(lens), max(lens)
        self.to = forms.Pool(ba, seed + 1, [min(keep, m) for m in lens], hkv, d, rows)
        self.q, self.lens = rand(seed + 2, len(lens) * nq, hq, d, scale=2.0), ints(lens)
        self.lse = torch.from_numpy(lse64(self.pool, f64(self.q), nq, d ** -0.5)).float().cuda()
        self.old = torch.rand((self.n, hkv, self.max_len), generator=torch.Generator().manual_seed(seed)).cuda()
        n_pages = self.pool.kp.shape[0]
        new = lambda *shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype, device="cuda")  # noqa: E731
        self.w, self.codes, self.exps = new(self.n, hkv, self.max_len), new(n_pages, hkv, 2, d, dtype=torch.int8), new(n_pages, hkv, dtype=torch.int8)
        self.bounds = ba.PageBounds(self.codes, self.exps)
        self.sel, self.scores = new(self.n, hkv, n_select, dtype=torch.int32), new(self.n, hkv, n_select)
        self.o, self.o_lse = torch.zeros_like(self.q), new(len(lens) * nq, hq)
        self.kept, self.w_out, self.len_out = new(self.n, hkv, keep, dtype=torch.int32), new(self.n, hkv, keep), new(self.n, dtype=torch.int32)
        self.to.kp.zero_(), self.to.vp.zero_()
        room = lambda b: torch.empty(max(256, b), dtype=torch.uint8, device="cuda")  # noqa: E731
        self.ws = [room(ba.ba_paged_key_weights_workspace_bytes(self.heads, self.n, nq, self.max_len)),
                   room(ba.ba_page_select_workspace_bytes(self.heads, self.n, rows, self.max_len)),
                   room(ba.ba_paged_attention_selected_workspace_bytes(self.heads, self.n, nq, rows, self.max_len, n_select)),
                   room(ba.ba_paged_evict_workspace_bytes(self.heads, self.n, self.max_len, keep))]

    def run(self, decay=0.5, stream=None):
        ba, h, c = self.ba, self.heads, self.pool.cache  # noqa: F811
        ba.ba_paged_key_weights(h, c, self.q, self.lse, self.old, self.w, decay, self.lens, self.max_len, None, None, self.nq, self.ws[0], stream)
        ba.ba_page_bounds(h, c, self.bounds, None, self.lens, self.max_len, stream)
        ba.ba_page_select(h, c, self.bounds, self.q, self.lens, self.max_len, self.sel, self.scores, 1, 1, self.nq, self.ws[1], stream)
        ba.ba_paged_attention_selected(h, c, self.q, self.o, self.o_lse, self.lens, self.max_len, self.sel, self.nq, self.ws[2], stream)
        ba.ba_paged_evict(h, c, self.to.cache, self.w, self.lens, self.max_len, self.keep, 1, 2, self.kept, self.w_out, self.len_out, self.ws[3], stream)

    def results(self):
        return [x.clone() for x in (self.w, self.codes, self.exps, self.sel, self.scores, self.o, self.o_lse, self.kept, self.w_out, self.len_out, self.to.kp, self.to.vp)]

    def clear(self):
        for x in (self.w, self.codes, self.exps, self.sel, self.scores, self.o, self.o_lse, self.kept, self.w_out, self.len_out, self.to.kp, self.to.vp):
            x.zero_()


def test_the_python_half_of_the_face_makes_the_same_calls_of_long_caches(ba, monkeypatch):  # noqa: F811
    import torch
    step = Step(ba, 700, 8, 2, 64, 16, [300, 77, 1], 2, 8, 40)
    calls = []
    for native in (True, False):
        if not native:
            monkeypatch.setattr(ba, "_native", ba._NoNative())
            step.clear()
        step.run()
        calls.append(step.results())
        assert all(bool(x.any()) for x in calls[-1])
        step.run(1)  # (a whole number for the decay)
        assert bool((step.w[0, :, :290] >= calls[-1][0][0, :, :290]).all()) and not torch.equal(step.w, calls[-1][0])
        with pytest.raises(ValueError):
            ba.ba_paged_key_weights(step.heads, step.pool.cache, step.q, step.lse, step.old[:, :1], step.w, 0.5, step.lens, step.max_len)
        with pytest.raises(ValueError):
            ba.ba_page_select(step.heads, step.pool.cache, step.bounds, step.q, step.lens, step.max_len, step.sel, step.scores[:, :, :3], 1, 1, 2, step.ws[1])
    assert all(torch.equal(a, b) for a, b in zip(*calls))


def test_two_batches_at_once(ba):  # noqa: F811
    """Two batches of different shapes, each on a stream of its own, call by call in turn: what they leave one after the other."""
    import torch
    steps = [Step(ba, 710, 32, 8, 128, 16, [2000, 700, 33, 5], 1, 40, 300), Step(ba, 720, 8, 1, 64, 20, [900, 1500, 40], 9, 30, 64)]
    want = []
    for s in steps:
        s.run()
        want.append(s.results())
        s.clear()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in steps]
    for _ in range(5):
        for s, stream in zip(steps, streams):
            s.run(stream=stream)
    torch.cuda.synchronize()
    for s, w in zip(steps, want):
        assert all(torch.equal(a, b) for a, b in zip(s.results(), w))


@pytest.mark.parametrize("nq", [1, 8, 16])
def test_heads_far_apart(ba, nq):  # noqa: F811
    """Query heads half a gigabyte apart, key and value heads 4 GB: few and many rows a sequence."""
    import torch
    hq, hkv, d, rows, lens = 8, 2, 64, 16, [90, 40]
    step = Step(ba, 730, hq, hkv, d, rows, lens, nq, 4, 20)
    step.run()
    near = step.results()
    q_apart, k_apart = 1 << 28, (1 << 31) + 64
    far_q = torch.empty((hq - 1) * q_apart + len(lens) * nq * d, dtype=torch.bfloat16, device="cuda").as_strided(step.q.shape, (d, q_apart, 1))
    far_q.copy_(step.q)
    n_pages = step.pool.kp.shape[0]
    pools = []
    for x in (step.pool.kp, step.pool.vp):
        far = torch.empty((hkv - 1) * k_apart + n_pages * rows * d, dtype=torch.bfloat16, device="cuda").as_strided(x.shape, (rows * d, d, k_apart, 1))
        far.copy_(x)
        pools.append(far)
    step.clear()
    step.q, step.pool.cache = far_q, ba.PagedCache(*pools, step.pool.cache.page_table)
    step.run()
    for a, b in zip(step.results(), near):
        assert torch.equal(a, b)
