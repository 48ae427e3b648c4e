"""The largest arguments of the entry points around long paged caches.  Only calls that have to be refused: none of the addresses here is one."""
from test_long_cache_cpu import FAR, select
from test_paged_cpu import fake, lib  # noqa: F401


def test_lists_whose_places_do_not_fit_32_bits_are_refused(lib):  # noqa: F811
    """A list is filled up behind its last page a workgroup at a time: the place after the last one has to be a number, too."""
    far = dict(q=fake(FAR), codes=2 * FAR, exps=3 * FAR, out=4 * FAR, lens=5 * FAR)
    for n in ((1 << 31) - 1, (1 << 31) - 1024, (1 << 30) + 1):
        assert select(lib, n=n, **far) == -2 and b"n_select" in lib.ba_last_error(), n
