"""Limits of the entry points for modified scores and spans: refused on the host, before anything is launched (CPU)."""
import paper_2407_00611_amd  # noqa: F401
from paper_2407_00611_amd import api

PTR = 0x10000                                        # never read


def test_documents_whose_numbers_the_search_cannot_add():
    """The search for a row's document takes the middle of two indexes: beyond 2^30 their sum left 32 bits and pointed before the bounds."""
    call = lambda n, Sq=4: api._lib.st_mask_spans(1, Sq, 0, 0, 0, 1, PTR, n, None, PTR, None)
    assert call(1 << 30) == 2 and call((1 << 31) - 1) == 2
    assert call(1 << 30, Sq=0) == 0                  # nothing to do
