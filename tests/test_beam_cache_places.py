"""Where the moves of beams and the rows of a path may lie, on the CPU: every call below returns
before any launch."""
import ctypes

import pytest

from paper_2608_24411_amd import native

FAKE = ctypes.c_void_p(0x10000)     # never dereferenced


@pytest.mark.parametrize("W,K", [(1, 4), (3, 6), (6, 2)])
def test_other_numbers_of_beams_within_a_cache(W, K):
    """A paged move within one cache gets past the check of places (and is refused for the size of
    its tables, which is looked at later); one without tables does not."""
    r = native.RsRows(2, 2 * max(W, K), 3, 5, 16, 8 * 3 * 5 * 16, 3 * 5 * 16, 5 * 16, 16)
    at = ctypes.addressof(r)
    n = 1 << 30
    assert native.lib.resispec_beam_reorder_paged(FAKE, at, FAKE, n, FAKE, at, FAKE, n, n, FAKE, FAKE, 2, W, K, None,
                                                  None) == native.RS_ERR_UNSUPPORTED
    other = native.RsRows(2, 2 * max(W, K), 3, 5, 16, 9 * 3 * 5 * 16, 3 * 5 * 16, 5 * 16, 16)
    assert native.lib.resispec_beam_reorder_paged(FAKE, at, FAKE, n, FAKE, ctypes.addressof(other), FAKE, n, n, FAKE, FAKE, 2,
                                                  W, K, None, None) == native.RS_ERR_INVALID_ARG
    assert native.lib.resispec_beam_reorder(FAKE, at, FAKE, at, FAKE, None, 2, W, K, None, None) == native.RS_ERR_INVALID_ARG
