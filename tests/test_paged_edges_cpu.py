"""Refusals around the paged attention and the head norms that depend on where tensors lie and on how large a call is.  Only calls that have
to be refused: none of the addresses here is one."""
import numpy as np
import pytest

from test_paged_cpu import HEADS, Q, QO, append, attend, back, cache, fake, lib, norm  # noqa: F401

FAR = 1 << 44


def test_attention_refuses_outputs_over_what_it_reads(lib):  # noqa: F811
    assert attend(lib, o=fake(0x1000100)) == -1 and b"overlap" in lib.ba_last_error()       # over q, not in place
    assert attend(lib, o=fake(0x1000000, st=2048)) == -1 and b"overlap" in lib.ba_last_error()
    assert attend(lib, o=fake(0x10000400)) == -1 and b"overlap" in lib.ba_last_error()      # inside the pages
    assert attend(lib, o=fake(0x11000000 + 9 * 16 * 2048 + 15 * 2048)) == -1 and b"overlap" in lib.ba_last_error()  # their last row
    assert attend(lib, q=fake(0x11000000), o=fake(0x11000000)) == -1                        # in place, but of the pages


def test_heads_that_meet_are_refused_wherever_they_meet(lib):  # noqa: F811
    """Heads 384 apart (three tensors' one after the other): a query head over a key head, in the same row or another."""
    big = dict(st=8 * 384, sh=384)
    for d in (0, 240, -240):  # bytes
        assert norm(lib, q=fake(0x1000000, **big), qo=fake(0x1000000, **big), k=fake(0x1000000 + 768 + d, **big), ko=fake(FAR)) == -1, d
    row = 8 * 384 * 2
    k = fake(0x1000000 + 3 * row + 384 * 2 * 2 + 16, **big)  # row 3 of q's four, head 2 of eight
    assert norm(lib, q=fake(0x1000000, **big), qo=fake(0x1000000, **big), k=k, ko=fake(FAR)) == -1
    assert append(lib, q=fake(0x1000000, **big), qo=fake(0x1000000, **big), k=k) == -1
    assert back(lib, dq=fake(0x4000000, **big), dk=fake(0x4000000 + row * 2 + 384 * 4 - 128, **big)) == -1
    # steps that differ: key heads 512 apart, the second of them over a query head
    assert norm(lib, q=fake(0x1000000, **big), qo=fake(0x1000000, **big), k=fake(0x1000000 + 512, st=8 * 384, sh=512), ko=fake(FAR)) == -1


def test_append_refuses_pages_in_which_keys_and_values_meet(lib):  # noqa: F811
    one = fake(0x10000000)
    assert append(lib, c=cache(k=one, v=one)) == -1 and b"overlap" in lib.ba_last_error()
    assert append(lib, c=cache(k=one, v=fake(0x10000000 + 15 * 2048 + 256))) == -1 and b"overlap" in lib.ba_last_error()  # the last row's second head
    assert append(lib, c=cache(k=fake(0x10000000, 512, 256), v=fake(0x10000000 + 128, 512, 256))) == -1  # half a head on


def test_calls_larger_than_a_launch_are_refused_ahead_of_every_launch(lib):  # noqa: F811
    tokens = 1 << 27  # eight to a workgroup
    k, ko = fake(FAR, st=256), fake(2 * FAR, st=256)
    one = dict(q=None, qo=None, k=k, ko=ko, tokens=tokens)
    assert norm(lib, **one) == -2
    assert append(lib, q=None, qo=None, k=fake(FAR, st=256), v=fake(2 * FAR, st=256), tokens=tokens) == -2
    n = 1 << 18
    c = cache(n_seqs=n, max_pages=1 << 16, stride=1 << 16)
    far = dict(q=fake(FAR), o=fake(2 * FAR), wsb=1 << 62)
    assert attend(lib, c=c, max_len=1 << 20, **far) == -2
    # ninety-seven groups in one launch's table and the next, and behind them what no launch takes
    cu = np.concatenate([np.arange(0, 2 * 97 + 1, 2), [n]])
    assert attend(lib, c=c, max_len=1 << 20, cu=cu, pre=[1 << 20] * 97 + [0], **far) == -2


@pytest.mark.parametrize("n_seqs,q_per_seq,max_len", [(1 << 18, 1, 1 << 20)])
def test_workspace_queries_reject_calls_larger_than_a_launch(lib, n_seqs, q_per_seq, max_len):  # noqa: F811
    import ctypes
    assert lib.ba_paged_attention_workspace_bytes(ctypes.byref(HEADS.c), n_seqs, q_per_seq, max_len, 0, None, None) == 0
