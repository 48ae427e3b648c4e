"""The largest arguments of the entry points around long paged caches.  Only calls that have to be refused: none of the addresses here is one."""
from test_long_cache_cpu import FAR, evict, page_bounds, select, selected, to, weights
from test_paged_cpu import append, attend, cache, fake, lib  # noqa: F401


def test_lists_whose_places_do_not_fit_32_bits_are_refused(lib):  # noqa: F811
    """A list is filled up behind its last page a workgroup at a time: the place after the last one has to be a number, too."""
    far = dict(q=fake(FAR), codes=2 * FAR, exps=3 * FAR, out=4 * FAR, lens=5 * FAR)
    for n in ((1 << 31) - 1, (1 << 31) - 1024, (1 << 30) + 1):
        assert select(lib, n=n, **far) == -2 and b"n_select" in lib.ba_last_error(), n


def test_rows_that_lie_far_apart_are_refused(lib):  # noqa: F811
    """Offsets within sixteen rows of a page are counted in 32 bits: every call that reads a page refuses rows 2^24 elements apart and more, keys or values."""
    for st in (1 << 24, 143 << 20, 1 << 31, 1 << 40):
        for side in "kv":
            c = cache(**{side: fake(FAR, st=st)})
            for call in (weights, evict, page_bounds, select, selected, attend, append):
                assert call(lib, c=c) == -2 and b"stride" in lib.ba_last_error(), (st, side, call)
            assert evict(lib, t=to(**{side: fake(FAR, st=st)})) == -2
