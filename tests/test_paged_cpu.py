"""Refusals of the entry points around head norms and the paged cache: bad arguments become status codes or exceptions before
any device work, without a GPU."""
import ctypes
import os

import numpy as np
import pytest

from paper_2409_15355_amd import binding as ba


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(ba.LIB_PATH):
        from paper_2409_15355_amd import build
        build.build()
    return ba.load()


def fake(ptr=0x1000000, st=1024, sh=128, dtype=0):
    return ba.BaTensor(ptr, st, sh, dtype)


def ref(x):
    return None if x is None else ctypes.byref(x)


def ip(a):
    return None if a is None else np.asarray(a, dtype=np.int32).tobytes()


HEADS = ba.Heads(8, 2, 128)
Q, K, V = fake(0x1000000), fake(0x2000000), fake(0x3000000)
QO, KO = fake(0x4000000), fake(0x5000000)


def head_norm(eps=1e-6, dtype=0, w=0x100):
    return ba.BaHeadNorm(w, w, dtype, eps)


def norm(lib, heads=HEADS, n=None, q=Q, k=K, qo=QO, ko=KO, tokens=4, pos=None, mode=1, norm_null=False):
    return lib.ba_norm_rotate(ref(heads.c), None if norm_null else ref(n or head_norm()), ref(q), ref(k), ref(qo), ref(ko), tokens, pos, mode, None)


def test_norm_rotate_refusals(lib):
    assert norm(lib, norm_null=True) == -1
    for eps in (0.0, -1.0, float("nan"), float("inf")):
        assert norm(lib, n=head_norm(eps)) == -1
    assert norm(lib, n=head_norm(dtype=3)) == -2
    assert norm(lib, n=head_norm(dtype=1, w=0x102)) == -3
    assert norm(lib, heads=ba.Heads(8, 2, 96)) == -2 and norm(lib, heads=ba.Heads(8, 3, 128)) == -1
    assert norm(lib, q=None, k=None, qo=None, ko=None) == -1 and norm(lib, qo=None) == -1 and norm(lib, ko=None) == -1
    assert norm(lib, tokens=-1) == -1 and norm(lib, mode=2) == -1 and norm(lib, pos=0x1002) == -3
    assert norm(lib, q=fake(0x1000008)) == -3 and norm(lib, qo=fake(0x4000000, dtype=1)) == -2
    assert norm(lib, q=fake(0x1000000, dtype=1), qo=fake(0x4000000, dtype=1)) == -2  # two types
    assert norm(lib, qo=fake(0x1000100)) == -1  # overlaps q without being in place
    assert norm(lib, qo=fake(0x2000000)) == -1 and b"k" in lib.ba_last_error()  # on top of k
    assert norm(lib, ko=fake(0x4000000)) == -1  # both outputs in one place
    assert norm(lib, tokens=0) == 0


def back(lib, heads=HEADS, n=None, q=Q, k=K, gq=fake(0x6000000), gk=fake(0x7000000), dq=QO, dk=KO, dwq=None, dwk=None, tokens=4, pos=None, mode=1,
         ws=0x9000000, wsb=1 << 20):
    return lib.ba_norm_rotate_backward(ref(heads.c), ref(n or head_norm()), ref(q), ref(k), ref(gq), ref(gk), ref(dq), ref(dk), dwq, dwk, tokens, pos,
                                       mode, ws, wsb, None)


def test_norm_rotate_backward_refusals(lib):
    assert back(lib, gq=None) == -1 and back(lib, dq=None) == -1 and back(lib, dk=None) == -1
    assert back(lib, n=head_norm(0.0)) == -1 and back(lib, mode=5) == -1 and back(lib, tokens=-2) == -1
    assert back(lib, ws=None, wsb=0) == -4 and back(lib, ws=0x9000010) == -4
    need = lib.ba_norm_rotate_backward_workspace_bytes(ref(HEADS.c), 4)
    assert need > 0 and back(lib, wsb=need - 1) == -4
    assert back(lib, q=None, gq=None, dq=None, dwq=0x100) == -1  # a gradient of gains that nothing went through
    assert back(lib, dwk=0x102) == -3 and back(lib, dq=fake(0x7000000)) == -1 and back(lib, dk=fake(0x1000000)) == -1
    assert back(lib, tokens=0, ws=None, wsb=0) == 0
    assert lib.ba_norm_rotate_backward_workspace_bytes(ref(HEADS.c), 0) == 0


def cache(k=None, v=None, ksp=16 * 1024, vsp=16 * 1024, n_pages=10, rows=16, table=0x800000, stride=4, n_seqs=3, max_pages=4):
    return ba.BaPagedCache(k or fake(0x10000000), v or fake(0x11000000), ksp, vsp, n_pages, rows, table, stride, n_seqs, max_pages)


def append(lib, heads=HEADS, n=None, c=None, q=Q, k=K, v=V, qo=QO, tokens=4, at=0x700000, seq=None, pos=None, mode=1):
    return lib.ba_paged_append(ref(heads.c), ref(n), ref(c or cache()), ref(q), ref(k), ref(v), ref(qo), tokens, at, seq, pos, mode, None)


BAD_CACHES = [(dict(n_pages=0), -1), (dict(rows=0), -1), (dict(n_seqs=-1), -1), (dict(max_pages=-1), -1), (dict(table=None), -1), (dict(table=0x800002), -3),
              (dict(stride=3), -1), (dict(ksp=4), -3), (dict(vsp=-16 * 1024), -1), (dict(k=fake(0x10000000, dtype=1)), -2),
              (dict(v=fake(0x11000004)), -3), (dict(rows=1 << 30, max_pages=4), -2)]


def test_paged_append_refusals(lib):
    for how, status in BAD_CACHES:
        assert append(lib, c=cache(**how)) == status, how
    assert lib.ba_paged_append(ref(HEADS.c), None, None, None, ref(K), ref(V), None, 4, 0x700000, None, None, 1, None) == -1
    assert append(lib, k=None) == -1 and append(lib, v=None) == -1 and append(lib, qo=None) == -1 and append(lib, at=None) == -1
    assert append(lib, k=fake(0x2000000, dtype=1)) == -2 and append(lib, q=fake(dtype=1), qo=fake(0x4000000, dtype=1)) == -2
    assert append(lib, n=head_norm(0.0)) == -1 and append(lib, mode=3) == -1 and append(lib, tokens=-1) == -1
    assert append(lib, at=0x700001) == -3 and append(lib, seq=0x700001) == -3 and append(lib, pos=0x700001) == -3
    assert append(lib, k=fake(0x10000400)) == -1 and append(lib, qo=fake(0x11000000)) == -1  # in the cache itself
    assert append(lib, qo=fake(0x2000000)) == -1
    assert append(lib, tokens=0) == 0
    assert append(lib, heads=ba.Heads(7, 2, 128), q=None, qo=None, tokens=0) == 0  # (without queries their heads do not matter)


def attend(lib, heads=HEADS, c=None, q=Q, o=QO, lse=None, nq=1, lens=0x700000, max_len=64, cu=None, pre=None, ws=0x9000000, wsb=1 << 24):
    n = 0 if pre is None else len(pre)
    return lib.ba_paged_attention(ref(heads.c), ref(c or cache()), ref(q), ref(o), lse, nq, lens, max_len, n, ip(cu), ip(pre), ws, wsb, None)


def test_paged_attention_refusals(lib):
    for how, status in BAD_CACHES:
        assert attend(lib, c=cache(**how)) == status, how
    assert attend(lib, q=None) == -1 and attend(lib, o=None) == -1 and attend(lib, lens=None) == -1
    assert attend(lib, nq=0) == -1 and attend(lib, max_len=-1) == -1 and attend(lib, max_len=65) == -1
    assert attend(lib, lens=0x700002) == -3 and attend(lib, lse=0x700002) == -3 and attend(lib, q=fake(dtype=1)) == -2
    assert attend(lib, cu=[0, 2], pre=[5]) == -1        # not all of the sequences
    assert attend(lib, cu=[1, 3], pre=[5]) == -1
    assert attend(lib, cu=[0, 3, 2, 3], pre=[5, 5, 5]) == -1
    assert attend(lib, cu=[0, 3], pre=[65]) == -1 and attend(lib, cu=[0, 3], pre=[-1]) == -1
    assert attend(lib, cu=None, pre=[5]) == -1
    assert attend(lib, nq=1 << 27) == -2
    need = lib.ba_paged_attention_workspace_bytes(ref(HEADS.c), 3, 1, 64, 1, ip([0, 3]), ip([32]))
    assert need > 0
    assert attend(lib, cu=[0, 3], pre=[32], wsb=need - 1) == -4 and attend(lib, cu=[0, 3], pre=[32], ws=None, wsb=0) == -4
    assert attend(lib, cu=[0, 3], pre=[32], ws=0x9000080) == -4
    assert attend(lib, c=cache(n_seqs=0), cu=[0], pre=[], max_len=64) == 0
    assert attend(lib, c=cache(n_seqs=0)) == 0


def test_paged_attention_workspace_follows_what_is_shared(lib):
    size = lambda n, nq, m, cu=None, pre=None: lib.ba_paged_attention_workspace_bytes(ref(HEADS.c), n, nq, m, 0 if pre is None else len(pre), ip(cu), ip(pre))  # noqa: E731
    assert size(3, 1, 64) == 0 and size(0, 1, 64) == 0          # one part a row: nothing to merge
    assert size(3, 1, 64, [0, 3], [32]) > 0
    assert size(3, 1, 64, [0, 1, 2, 3], [32, 32, 32]) == 0      # nobody to share with
    assert size(2, 1, 100000) > size(2, 1, 20000) > 0
    assert size(3, 0, 64) == 0 and size(3, 1, -1) == 0 and size(3, 1, 64, [0, 2], [32]) == 0
    # as many groups as one likes
    cu = np.arange(0, 1001, 2)
    assert size(1000, 1, 64, cu, [32] * 500) > 0


def test_python_face_refusals(lib):
    import torch
    x = torch.zeros(4, 8, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        ba.HeadNorm(torch.ones(128))  # not on the GPU
    with pytest.raises(ValueError):
        ba.PagedCache(x[None], x[None, :2], torch.zeros(1, 1, dtype=torch.int32))
    with pytest.raises(ValueError):
        ba.PagedCache(x, x, torch.zeros(1, 1, dtype=torch.int32))
    with pytest.raises(ValueError):
        ba.ba_norm_rotate(HEADS, ba.HeadNorm(), x, None, x, None)
    with pytest.raises(ValueError):
        ba.ba_norm_rotate(HEADS, ba.HeadNorm(), None, None, None, None)
    with pytest.raises(ValueError):
        ba.ba_paged_attention_workspace_bytes(HEADS, 3, 1, 64, [0, 3], None)
    with pytest.raises(ValueError):
        ba.ba_paged_attention_workspace_bytes(HEADS, 3, 1, 64, [0, 2, 3], [4])
