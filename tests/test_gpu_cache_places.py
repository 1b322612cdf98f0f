"""Moves of beams whose rows come from and go to one and the same buffer, value for value."""
import numpy as np
import pytest
import torch

from test_gpu_cache import fill, paged_reference, parents, same

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("W,K", [(1, 4), (3, 6), (6, 2), (5, 10), (17, 33)])
@pytest.mark.parametrize("apart", [True, False], ids=["other-pages", "some-the-same"])
def test_other_numbers_of_beams_within_a_cache(gpu_lib, W, K, apart):
    """A first step's beam to K, W beams to 2 W, and fewer; into pages of their own, or with the
    first beams' pages kept: those rows are then sources too, at the same positions.  A prompt's
    page is every beam's."""
    B, P, M, outer, row = 3, 4, 6, 2, 9
    pages = B * (W + K) * M + 5
    g = np.random.default_rng([W, K])
    order = torch.as_tensor(g.permutation(pages), dtype=torch.int32, device="cuda")
    table, other = order[:B * W * M].view(B, W, M).clone(), order[B * W * M:B * (W + K) * M].view(B, K, M).clone()
    if not apart:
        n = min(W, K)
        other[:, :n] = table[:, :n]
        table[:, :, 0] = table[:, :1, 0]
        other[:, :, 0] = table[:, :1, 0]
    cache = fill((outer, pages, 1, P, row), torch.bfloat16)
    parent = parents(B, K, W, 4)
    lengths = torch.tensor([M * P, 11, 1], dtype=torch.int32, device="cuda")
    print("within a cache", W, K, apart, flush=True)
    table, other = table.view(B * W, M), other.view(B * K, M)
    state = cache.clone()
    want = paged_reference(cache.cpu(), table.cpu(), other.cpu(), parent.cpu(), lengths.cpu(), P, cache.cpu())
    out, st = gpu_lib.resispec_beam_reorder_paged(state, table, parent, lengths, page_dim=1, position_dim=3, out_table=other)
    torch.cuda.synchronize()
    assert out is state and same(out.cpu(), want) and (st == 0).all()


def test_tables_are_needed_for_that(gpu_lib):
    i32 = dict(dtype=torch.int32, device="cuda")
    cache, table = torch.zeros((9, 4, 5), device="cuda"), torch.zeros((6, 2), **i32)
    with pytest.raises(ValueError):
        gpu_lib.resispec_beam_reorder_paged(cache, table, torch.zeros((2, 4), **i32), torch.zeros(2, **i32))
    with pytest.raises(ValueError):
        gpu_lib.resispec_beam_reorder(cache[:6], torch.zeros((2, 4), **i32))
