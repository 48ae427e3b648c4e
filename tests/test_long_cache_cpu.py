"""Refusals of the entry points around long paged caches: bad arguments become status codes or exceptions before any device work,
without a GPU.  Only calls that have to be refused, or have nothing to do: none of the addresses here is one."""
import ctypes

import numpy as np
import pytest

from paper_2409_15355_amd import binding as ba
from test_paged_cpu import BAD_CACHES, HEADS, Q, QO, cache, fake, ip, lib, ref  # noqa: F401

FAR = 1 << 44


def weights(lib, heads=HEADS, c=None, q=Q, lse=0x500000, w_in=None, w_out=0x20000000, stride=64, decay=1.0, nq=1, lens=0x700000, max_len=64, cu=None,  # noqa: F811
            pre=None, ws=0x9000000, wsb=1 << 24):
    n = 0 if pre is None else len(pre)
    return lib.ba_paged_key_weights(ref(heads.c), ref(c or cache()), ref(q), lse, w_in, w_out, stride, decay, nq, lens, max_len, n, ip(cu), ip(pre), ws, wsb, None)


def test_key_weights_refusals(lib):  # noqa: F811
    for how, status in BAD_CACHES:
        assert weights(lib, c=cache(**how)) == status, how
    assert weights(lib, q=None) == -1 and weights(lib, lse=None) == -1 and weights(lib, w_out=None) == -1 and weights(lib, lens=None) == -1
    assert weights(lib, q=fake(dtype=1)) == -2 and weights(lib, heads=ba.Heads(7, 2, 128)) == -1 and weights(lib, heads=ba.Heads(8, 2, 96)) == -2
    assert weights(lib, nq=0) == -1 and weights(lib, max_len=-1) == -1 and weights(lib, max_len=65) == -1 and weights(lib, nq=1 << 27) == -2
    assert weights(lib, max_len=(1 << 30) + 1) == -2
    assert weights(lib, stride=63) == -1
    for bad in (float("nan"), float("inf"), -float("inf")):
        assert weights(lib, decay=bad) == -1
    for name in ("lse", "w_in", "w_out", "lens"):
        assert weights(lib, **{name: 0x600002}) == -3, name
    # where the weights lie: 3 sequences, 2 heads, 64 tokens
    assert weights(lib, w_in=0x20000004) == -1 and b"overlap" in lib.ba_last_error()
    assert weights(lib, w_in=0x20000000 + 6 * 64 * 4 - 4) == -1
    assert weights(lib, w_out=0x1000000) == -1 and weights(lib, w_out=0x500000 - 256) == -1      # q, lse
    assert weights(lib, lens=0x20000000 + 64) == -1 and b"seq_len" in lib.ba_last_error()
    assert weights(lib, w_out=0x10000000 + 9 * 16 * 2048) == -1 and weights(lib, w_out=0x11000000) == -1  # pages
    # groups
    assert weights(lib, cu=[0, 2], pre=[5]) == -1 and weights(lib, cu=[0, 3], pre=[65]) == -1 and weights(lib, cu=[0, 3, 2, 3], pre=[5, 5, 5]) == -1
    assert weights(lib, cu=None, pre=[5]) == -1
    # nothing to do
    assert weights(lib, c=cache(n_seqs=0), q=None, lse=None, w_out=None, lens=None) == 0
    assert weights(lib, max_len=0, stride=0, q=None, lse=None, w_out=None) == 0
    # pages whose rows lie further apart than 32 bits of bytes say
    wide = cache(k=fake(0x10000000, st=1 << 31))
    assert weights(lib, c=wide) == -2


def test_key_weights_workspace(lib):  # noqa: F811
    size = lambda n, nq, m, cu=None, pre=None, h=HEADS: lib.ba_paged_key_weights_workspace_bytes(ref(h.c), n, nq, m, 0 if pre is None else len(pre), ip(cu), ip(pre))  # noqa: E731
    assert size(3, 1, 64) == 0 and size(0, 1, 64) == 0 and size(3, 1, -1) == 0 and size(3, 0, 64) == 0
    assert size(1, 256, 400) > 0                 # many rows over few keys: in parts
    assert size(2, 256, 400, [0, 2], [100]) == 0 and size(2, 256, 400, [0, 2], [0]) == size(2, 256, 400)
    q = fake(FAR)
    need = size(3, 256, 64)
    assert need > 0 and weights(lib, q=q, nq=256, wsb=need - 1) == -4 and weights(lib, q=q, nq=256, ws=None, wsb=0) == -4
    assert weights(lib, q=q, nq=256, ws=0x9000080) == -4


def test_calls_larger_than_a_launch(lib):  # noqa: F811
    n = 1 << 18
    big = cache(n_seqs=n, max_pages=1 << 16, stride=1 << 16)
    assert weights(lib, c=big, max_len=1 << 20, stride=1 << 20, w_out=2 * FAR, q=fake(FAR), lse=3 * FAR) == -2
    assert evict(lib, c=big, t=cache(k=fake(FAR), v=fake(2 * FAR), n_seqs=n, max_pages=1 << 16, stride=1 << 16), w=3 * FAR, stride=1 << 20, max_len=1 << 20,
                 n_keep=1 << 19, kept=5 * FAR, lens=8 * FAR, w_out=None) == -2
    many = cache(n_seqs=1 << 22, max_pages=4)
    assert select(lib, c=many, q=fake(FAR), out=2 * FAR, lens=3 * FAR) == -2
    assert page_bounds(lib, c=many) == -2
    assert selected(lib, c=big, q=fake(FAR), o=fake(2 * FAR), max_len=1 << 20, sel=3 * FAR, n=1 << 20, wsb=1 << 62) == -2


def evict(lib, heads=HEADS, c=None, t=None, w=0x20000000, stride=64, lens=0x700000, max_len=64, n_keep=8, first=1, last=2, kept=0x22000000, w_out=0x23000000,  # noqa: F811
          stride_out=8, len_out=0x24000000, ws=None, wsb=0):
    to = t or cache(k=fake(0x12000000), v=fake(0x13000000), table=0x900000)
    return lib.ba_paged_evict(ref(heads.c), ref(c or cache()), ref(to), w, stride, lens, max_len, n_keep, first, last, kept, w_out, stride_out, len_out, ws, wsb, None)


def to(**how):
    return cache(**{**dict(k=fake(0x12000000), v=fake(0x13000000), table=0x900000), **how})


def test_evict_refusals(lib):  # noqa: F811
    for how, status in BAD_CACHES:
        assert evict(lib, c=cache(**how)) == status, how
        how = {x: (fake(y.ptr + 0x2000000, dtype=y.dtype) if x in "kv" else y) for x, y in how.items()}
        assert evict(lib, t=to(**how)) == status, how
    assert evict(lib, w=None) == -1 and evict(lib, lens=None) == -1 and evict(lib, kept=None) == -1
    assert evict(lib, n_keep=0) == -1 and evict(lib, first=-1) == -1 and evict(lib, last=-1) == -1 and evict(lib, first=5, last=4) == -1
    assert evict(lib, max_len=65) == -1 and evict(lib, max_len=-1) == -1 and evict(lib, stride=63) == -1 and evict(lib, stride_out=7) == -1
    assert evict(lib, t=to(n_seqs=2)) == -1                                  # another number of sequences
    assert evict(lib, t=to(max_pages=1), n_keep=20, stride_out=20) == -1     # no room for them
    for name in ("w", "lens", "kept", "w_out", "len_out"):
        assert evict(lib, **{name: 0x60000002}) == -3, name
    # pages: of the same pool described alike, with a table of their own, or apart
    same = dict(k=fake(0x10000000), v=fake(0x11000000))
    assert evict(lib, t=to(**same, table=0x800000)) == -1 and b"pages that the sequences read" in lib.ba_last_error()
    assert evict(lib, t=to(k=fake(0x10000000 + 2048), v=fake(0x11000000))) == -1
    assert evict(lib, t=to(**same, ksp=32 * 1024)) == -1
    assert evict(lib, t=to(k=fake(0x11000000), v=fake(0x10000000))) == -1    # keys over values
    assert evict(lib, t=to(k=fake(0x12000000), v=fake(0x12000000))) == -1    # keys and values of a page meet
    # arrays over each other, or over the pages
    assert evict(lib, kept=0x20000000) == -1 and evict(lib, w_out=0x20000000) == -1 and evict(lib, len_out=0x700004) == -1
    assert evict(lib, w_out=0x22000000 + 4) == -1 and evict(lib, len_out=0x22000000) == -1 and evict(lib, len_out=0x23000000) == -1
    assert evict(lib, kept=0x10000000) == -1 and evict(lib, w_out=0x12000000) == -1 and evict(lib, w=0x13000000) == -1 and evict(lib, lens=0x12000000) == -1
    # nothing to do
    assert evict(lib, c=cache(n_seqs=0), t=to(n_seqs=0), w=None, kept=None, lens=None) == 0


def page_bounds(lib, heads=HEADS, c=None, codes=0x30000000, exps=0x31000000, since=None, lens=0x700000, max_len=64, null=False):  # noqa: F811
    b = ba.BaPageBoundTable(codes, exps)
    return lib.ba_page_bounds(ref(heads.c), ref(c or cache()), None if null else ref(b), since, lens, max_len, None)


def test_page_bounds_refusals(lib):  # noqa: F811
    for how, status in BAD_CACHES:
        assert page_bounds(lib, c=cache(**how)) == status, how
    assert page_bounds(lib, null=True) == -1 and page_bounds(lib, codes=None) == -1 and page_bounds(lib, exps=None) == -1 and page_bounds(lib, lens=None) == -1
    assert page_bounds(lib, codes=0x30000008) == -3 and page_bounds(lib, lens=0x700002) == -3 and page_bounds(lib, since=0x700002) == -3
    assert page_bounds(lib, max_len=65) == -1 and page_bounds(lib, max_len=-1) == -1
    assert page_bounds(lib, codes=0x10000000) == -1 and page_bounds(lib, exps=0x11000005) == -1      # in the pages
    assert page_bounds(lib, exps=0x30000000 + 10 * 2 * 2 * 128 - 1) == -1                            # in the codes
    assert page_bounds(lib, max_len=0, lens=None) == 0 and page_bounds(lib, c=cache(n_seqs=0), lens=None) == 0


def select(lib, heads=HEADS, c=None, codes=0x30000000, exps=0x31000000, q=Q, nq=1, lens=0x700000, max_len=64, n=4, first=1, last=1, out=0x22000000,  # noqa: F811
           scores=None, ws=0x9000000, wsb=1 << 24):
    b = ba.BaPageBoundTable(codes, exps)
    return lib.ba_page_select(ref(heads.c), ref(c or cache()), ref(b), ref(q), nq, lens, max_len, n, first, last, out, scores, ws, wsb, None)


def test_page_select_refusals(lib):  # noqa: F811
    for how, status in BAD_CACHES:
        assert select(lib, c=cache(**how)) == status, how
    assert select(lib, codes=None) == -1 and select(lib, q=None) == -1 and select(lib, out=None) == -1 and select(lib, lens=None) == -1
    assert select(lib, q=fake(dtype=1)) == -2 and select(lib, heads=ba.Heads(7, 2, 128)) == -1
    assert select(lib, nq=0) == -1 and select(lib, max_len=65) == -1 and select(lib, max_len=-1) == -1
    assert select(lib, first=-1) == -1 and select(lib, last=-1) == -1 and select(lib, n=0) == -1
    assert select(lib, n=4, first=1, last=4) == -1                              # no room for both
    assert select(lib, n=3, first=1, nq=34) == -1                              # ... nor for the pages of 34 new tokens: three or four
    assert select(lib, n=2, first=(1 << 31) - 1, last=(1 << 31) - 1) == -1
    for name in ("lens", "out", "scores"):
        assert select(lib, **{name: 0x60000002}) == -3, name
    assert select(lib, out=0x1000000) == -1 and select(lib, out=0x30000000) == -1 and select(lib, scores=0x31000000) == -1 and select(lib, out=0x700000 - 4) == -1
    assert select(lib, scores=0x22000000 + 4) == -1
    need = lib.ba_page_select_workspace_bytes(ref(HEADS.c), 3, 16, 64)
    assert need > 0 and select(lib, wsb=need - 1) == -4 and select(lib, ws=None, wsb=0) == -4 and select(lib, ws=0x9000010) == -4
    assert select(lib, c=cache(n_seqs=0), q=None, out=None, lens=None) == 0
    size = lambda *a: lib.ba_page_select_workspace_bytes(ref(HEADS.c), *a)  # noqa: E731
    assert size(0, 16, 64) == 0 and size(3, 0, 64) == 0 and size(3, 16, -1) == 0 and size(3, 16, 0) == 0 and size(1 << 22, 16, 64) == 0


def selected(lib, heads=HEADS, c=None, q=Q, o=QO, lse=None, nq=1, lens=0x700000, max_len=64, sel=0x22000000, n=4, ws=0x9000000, wsb=1 << 24):  # noqa: F811
    return lib.ba_paged_attention_selected(ref(heads.c), ref(c or cache()), ref(q), ref(o), lse, nq, lens, max_len, sel, n, ws, wsb, None)


def test_selected_attention_refusals(lib):  # noqa: F811
    for how, status in BAD_CACHES:
        assert selected(lib, c=cache(**how)) == status, how
    assert selected(lib, q=None) == -1 and selected(lib, o=None) == -1 and selected(lib, lens=None) == -1 and selected(lib, sel=None) == -1
    assert selected(lib, nq=0) == -1 and selected(lib, n=0) == -1 and selected(lib, max_len=65) == -1 and selected(lib, max_len=-1) == -1
    assert selected(lib, q=fake(dtype=1)) == -2 and selected(lib, nq=1 << 27) == -2
    for name in ("lens", "sel", "lse"):
        assert selected(lib, **{name: 0x60000002}) == -3, name
    assert selected(lib, o=fake(0x1000100)) == -1 and b"overlap" in lib.ba_last_error()
    assert selected(lib, o=fake(0x10000400)) == -1 and b"overlap" in lib.ba_last_error()
    assert selected(lib, c=cache(n_seqs=0), q=None, o=None, sel=None) == 0
    c = cache(n_pages=2000, n_seqs=1, max_pages=2000, stride=2000, k=fake(FAR), v=fake(2 * FAR))
    need = lib.ba_paged_attention_selected_workspace_bytes(ref(HEADS.c), 1, 1, 16, 32000, 256)
    assert need > 0 and selected(lib, c=c, max_len=32000, n=256, wsb=need - 1) == -4 and selected(lib, c=c, max_len=32000, n=256, ws=None, wsb=0) == -4


def test_selected_attention_workspace(lib):  # noqa: F811
    size = lambda *a: lib.ba_paged_attention_selected_workspace_bytes(ref(HEADS.c), *a)  # noqa: E731
    assert size(3, 1, 16, 64, 1) == 0 and size(0, 1, 16, 64, 1) == 0 and size(3, 1, 16, 64, 0) == 0 and size(3, 1, 0, 64, 1) == 0 and size(3, 0, 16, 64, 1) == 0
    assert size(1, 1, 16, 100000, 256) == size(1, 1, 16, 4096, 1 << 20) > 0   # bounded by the pages listed, and by the sequences
    assert size(1, 1, 1 << 20, 1 << 30, (1 << 31) - 1) > 0                    # (no more than 2^30 keys, however many pages)


def test_python_face_refusals(lib):  # noqa: F811
    import torch
    x = torch.zeros(4, 2, 2, 128, dtype=torch.int8)
    with pytest.raises(ValueError):
        ba.PageBounds(x, x[:, :, 0, 0])  # not on the GPU
    for name, args in (("_per_key", (torch.zeros(3, 2, 64), "weights", HEADS, 3, 64)), ("_lists", (torch.zeros(3, 2, 4, dtype=torch.int32), "selected", HEADS, 3))):
        with pytest.raises(ValueError):
            getattr(ba, name)(*args)
    with pytest.raises(ValueError):
        ba.ba_paged_key_weights_workspace_bytes(HEADS, 3, 1, 64, [0, 3], None)


@pytest.mark.parametrize("call,n_args", [("key_weights", 14), ("evict", 14), ("page_bounds", 7), ("page_select", 13), ("paged_attention_selected", 11)])
def test_arguments_that_are_not_plain_are_left_to_the_python_functions(lib, call, n_args):  # noqa: F811
    import torch
    take = getattr(ba._face(), call)
    assert take() is None and take(*[None] * n_args) is None and take(HEADS, *[None] * (n_args - 1)) is None
    assert take(HEADS, *[torch.zeros(4, 8, 128)] * (n_args - 1)) is None  # (no tensor of the GPU's)
    assert take(HEADS, np.zeros(4, dtype=np.int32), *[[0, 1]] * (n_args - 2)) is None
