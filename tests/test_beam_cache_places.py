"""Where the moves of beams and the rows of a path may lie, on the CPU: every call below returns
before any launch."""
import ctypes
import itertools
import random

import pytest
import torch

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


def places(t, *dims):
    """(layout, the bytes that its rows lie on) of a tensor, in its buffer."""
    r = native._layout(t.shape, t.stride(), t.element_size(), *dims, "t")[0]
    at = t.storage_offset() * t.element_size()
    starts = itertools.product(range(r.outer), range(r.pages), range(r.inner), range(r.positions))
    return bytes(r), at, {at + o * r.outer_stride + p * r.page_stride + i * r.inner_stride + s * r.position_stride + x
                          for o, p, i, s in starts for x in range(r.row_bytes)}


def interleaved(a, b, *dims):
    (x, at, mine), (y, to, other) = places(a, *dims), places(b, *dims)
    got = native._interleaved(x, y, to - at)
    assert got == native._interleaved(y, x, at - to)
    assert not (got and mine & other)       # never said of rows that share a byte
    return got


def test_rows_between_each_other():
    """Pairs of views of one buffer [layers, 2, beams, heads, positions, size] without a common
    byte, as a move back and forth has them, and pairs with one."""
    t = torch.zeros(3, 2, 6, 2, 4, 10, dtype=torch.bfloat16)
    dims = (1, 3)
    assert interleaved(t[:, 0], t[:, 1], *dims)
    assert interleaved(t[:, 0], t[:, 1, :4], *dims)                         # fewer beams
    flat = t.view(3, 12, 2, 4, 10)
    assert interleaved(flat[:, 0::2], flat[:, 1::2], *dims)                 # every other beam
    assert interleaved(flat[..., :6], flat[..., 6:], *dims)                 # ends of rows
    assert interleaved(flat[:, :, :, :2], flat[:, :, :, 2:], *dims)         # first and last positions
    assert interleaved(flat[:, :, :1], flat[:, :, 1:], *dims)               # heads
    assert interleaved(flat[:, :5], flat[:, 7:], *dims)
    for a, b in ((t[:, 0], t[:, 0]), (flat[:, :6], flat[:, 5:11]), (flat[..., :6], flat[..., 5:]), (flat[:, 0::2], flat[:, 0::2]),
                 (flat[:, 0::2], flat[:, 1:7]), (flat[:, :, :, :3], flat[:, :, :, 2:]), (flat[:2], flat[1:])):
        assert not interleaved(a, b, *dims)


def test_rows_between_each_other_at_random():
    """Whatever the views: rows that share a byte are never called apart."""
    rng = random.Random(5)
    t = torch.zeros(3, 8, 3, 4, 6, dtype=torch.uint8)
    found = shared = 0
    for _ in range(1500):
        def view():
            cut = []
            for n in t.shape[:-1]:
                step = rng.choice((1, 1, 2, 3))
                first = rng.randrange(n)
                cut.append(slice(first, rng.randrange(first, n) + 1, step))
            first = rng.randrange(6)
            return t[tuple(cut) + (slice(first, rng.randrange(first, 6) + 1),)]
        a, b = view(), view()
        got = interleaved(a, b, 1, 3)
        found += got
        shared += bool(places(a, 1, 3)[2] & places(b, 1, 3)[2])
    assert found and shared                 # both kinds came up
