"""The longest sequences that the calls around paged caches take, 2^30 tokens: a page of 2^20 rows that the table names 1,024 times.  Every copy of a key gets
the same attention, so weights repeat bit for bit, and ties go to the first copy.

Tolerances, u = 2^-24: a weight as in test_long_cache_gpu.py.  A log-sum-exp adds positive terms, in parts of 1,024 keys at least and 4,096 at most and then part by
part: no chain of additions is longer than 4,096 + 2^20, so it is off by that many u and by its exponentials' errors; outputs by twice that of sum p |v|."""
import math

import numpy as np
import pytest

from test_long_cache_gpu import BF16_STEP, U, ba, codes64, f64, ints, rand  # noqa: F401

pytestmark = pytest.mark.gpu

ROWS, COPIES, D = 1 << 20, 1 << 10, 64
CHAIN = (4096 + (1 << 20)) * U


def room(nbytes):
    import torch
    return torch.empty(max(256, nbytes), dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("hq", [2, 32])  # few rows a key, and many
def test_the_longest_sequences(ba, hq):  # noqa: F811
    import torch
    n = ROWS * COPIES - 5
    gen = torch.Generator(device="cuda").manual_seed(hq)
    kp, vp = (torch.randn((1, ROWS, 1, D), generator=gen, device="cuda").bfloat16() for _ in range(2))
    heads, cache = ba.Heads(hq, 1, D), ba.PagedCache(kp, vp, torch.zeros((1, COPIES), dtype=torch.int32, device="cuda"))
    q, lens, max_len = rand(3, 1, hq, D), ints([n]), ROWS * COPIES
    k, v, r = kp[0, :, 0].double(), vp[0, :, 0].double(), q[0].double()
    s = (r @ k.T) * D ** -0.5
    size = (r.abs() @ k.abs().T * D ** -0.5).amax(-1)

    def expected(copies):
        """Over `copies` of the page, the last one without its last five rows."""
        whole = s.logsumexp(-1) + math.log(copies - 1)
        last = s[:, :-5].logsumexp(-1)
        lse = torch.logaddexp(whole, last)
        p = (s - lse[:, None]).exp()
        count = torch.full((ROWS,), float(copies), dtype=torch.float64, device="cuda")
        count[-5:] -= 1
        off = CHAIN + D * U * size + (2 * s.abs().amax(-1) + lse.abs() + 8) * U
        return (p * count) @ v, lse, (p * count) @ v.abs(), off

    def close(o, lse, copies):
        out, l64, weight, off = expected(copies)
        assert bool(((lse[0].double() - l64).abs() <= off).all()), float(((lse[0].double() - l64).abs() / off).max())
        tol = (BF16_STEP + 2.0 ** -11 + 2 * off[:, None]) * weight + BF16_STEP * (out.abs() + (BF16_STEP + 2.0 ** -11) * weight)
        assert bool(((o[0].double() - out).abs() <= tol).all())

    o, lse = torch.empty_like(q), torch.empty((1, hq), device="cuda")
    ba.ba_paged_attention(heads, cache, q, o, lse, lens, max_len, ws=room(ba.ba_paged_attention_workspace_bytes(heads, 1, 1, max_len)))
    close(o, lse, COPIES)

    w = torch.full((1, 1, max_len), -7.0, device="cuda")
    ba.ba_paged_key_weights(heads, cache, q, lse, None, w, 0.0, lens, max_len, ws=room(ba.ba_paged_key_weights_workspace_bytes(heads, 1, 1, max_len)))
    l = lse[0].double()[:, None]
    p = (s - l).exp()
    err = (p * (D * U * (r.abs() @ k.abs().T * D ** -0.5) + (s.abs() + l.abs() + 4 + hq) * U)).sum(0)
    first = w[0, 0, :ROWS]
    assert bool(((first.double() - p.sum(0)).abs() <= err + 1e-37).all())
    assert bool((w[0, 0, n:] == -7).all())
    pages = w.view(COPIES, ROWS)
    for i in range(0, COPIES - 1):
        assert torch.equal(pages[i], first), i
    assert torch.equal(pages[-1, :-5], first[:-5])

    keep = 100
    to_k, to_v = (torch.zeros((7, 16, 1, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kept, w_out, len_out = torch.empty((1, 1, keep), dtype=torch.int32, device="cuda"), torch.empty((1, 1, keep), device="cuda"), ints([9])
    ba.ba_paged_evict(heads, cache, ba.PagedCache(to_k, to_v, ints([range(7)])), w, lens, max_len, keep, 2, 3, kept, w_out, len_out)
    heaviest = int(first.argmax())
    assert 2 <= heaviest < ROWS - 8 and int((first == first[heaviest]).sum()) == 1 and len_out.tolist() == [keep]
    want = [0, 1] + [heaviest + i * ROWS for i in range(keep - 5)] + [n - 3, n - 2, n - 1]
    assert kept[0, 0].tolist() == want
    rows = torch.tensor(want, device="cuda") % ROWS
    assert torch.equal(w_out[0, 0], first[rows])
    assert torch.equal(to_k.view(-1, D)[:keep], kp[0, rows, 0]) and torch.equal(to_v.view(-1, D)[:keep], vp[0, rows, 0]) and not to_k.view(-1, D)[keep:].any()

    # (bounds of the rows that the last copy has would be those of fewer: a call up to a page's end)
    bounds = ba.PageBounds(torch.zeros((1, 1, 2, D), dtype=torch.int8, device="cuda"), torch.zeros((1, 1), dtype=torch.int8, device="cuda"))
    ba.ba_page_bounds(heads, cache, bounds, None, ints([max_len]), max_len)
    e, hi, lo = codes64(f64(kp[0, :, 0]))
    assert int(bounds.exponents) == e and np.array_equal(f64(bounds.codes)[0, 0], [hi, lo])
    sel = torch.empty((1, 1, 3), dtype=torch.int32, device="cuda")
    ba.ba_page_select(heads, cache, bounds, q, lens, max_len, sel, None, 1, 1, 1, room(ba.ba_page_select_workspace_bytes(heads, 1, ROWS, max_len)))
    assert sel[0, 0].tolist() == [0, 1, COPIES - 1]
    for selected in (sel, torch.arange(COPIES, device="cuda").int().view(1, 1, COPIES)):
        o, lse = torch.full_like(q, float("nan")), torch.full((1, hq), float("nan"), device="cuda")
        copies = selected.shape[2]
        ba.ba_paged_attention_selected(heads, cache, q, o, lse, lens, max_len, selected, 1,
                                       room(ba.ba_paged_attention_selected_workspace_bytes(heads, 1, 1, ROWS, max_len, copies)))
        close(o, lse, copies)
