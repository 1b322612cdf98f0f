"""Moves of beams whose rows come from and go to one and the same buffer, value for value."""
import numpy as np
import pytest
import torch

from test_gpu_cache import commit_reference, expected, fill, paged_reference, parents, same

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


@pytest.mark.parametrize("cut", [lambda t: (t[:, 0], t[:, 1]), lambda t: (t[:, 1], t[:, 0, :6]),
                                 lambda t: (t.flatten(1, 2)[:, 0::2], t.flatten(1, 2)[:, 1::2]),
                                 lambda t: (t[:, 0, ..., :7], t[:, 0, ..., 7:14]),
                                 lambda t: (t[:, 0, :, :, :3], t[:, 0, :, :, 3:])],
                         ids=["halves", "fewer-beams", "every-other", "ends-of-rows", "positions"])
def test_moves_back_and_forth(gpu_lib, cut):
    """Views of one buffer that lie between each other: the rows of the one are moved to the other,
    and nothing else is written."""
    B, W = 2, 4
    whole = fill((3, 2, B * W, 2, 6, 15), torch.bfloat16)
    a, b = cut(whole)
    K = b.shape[1] // B
    parent = parents(B, K, W, 8)
    lengths = torch.tensor([a.shape[3], 2], dtype=torch.int32, device="cuda")
    host = whole.cpu()
    x, y = cut(host)
    y.copy_(expected(x.clone(), y.clone(), parent.cpu(), W, lengths.cpu()))
    out, st = gpu_lib.resispec_beam_reorder(a, parent, beam_dim=1, position_dim=3, lengths=lengths, out=b)
    torch.cuda.synchronize()
    assert out is b and (st == 0).all() and same(whole.cpu(), host)


def test_paged_moves_back_and_forth(gpu_lib):
    B, W, P, M = 2, 3, 4, 3
    whole = fill((2, 2, 20, 1, P, 9), torch.bfloat16)
    order = torch.randperm(20, device="cuda").int()
    table = order[:B * W * M].view(B * W, M)
    parent, lengths = parents(B, W, W, 2), torch.tensor([12, 5], dtype=torch.int32, device="cuda")
    host = whole.cpu()
    host[:, 1] = paged_reference(host[:, 0], table.cpu(), table.cpu(), parent.cpu(), lengths.cpu(), P, host[:, 1])
    out, st = gpu_lib.resispec_beam_reorder_paged(whole[:, 0], table, parent, lengths, page_dim=1, position_dim=3, out=whole[:, 1])
    torch.cuda.synchronize()
    assert (st == 0).all() and same(whole.cpu(), host)


def test_rows_of_a_path_between_the_cache(gpu_lib):
    """The trees' rows in the same buffer as the cache, after each layer's pages."""
    B, N, P, pages = 3, 8, 4, 9
    whole = fill((2, pages * P + B * N, 13), torch.bfloat16)
    cache = whole[:, :pages * P].view(2, pages, P, 13)
    source = whole[:, pages * P:].view(2, B, N, 13)
    slots = torch.randperm(pages * P, device="cuda").int()[:B * N].view(B, N).contiguous()
    path = torch.tensor([[0, 2, 5], [0, -1, -1], [1, 6, 7]], dtype=torch.int32, device="cuda")
    host = whole.cpu()
    want = commit_reference(cache.cpu().unsqueeze(2), slots.cpu(), path.cpu(), P, source.cpu().unsqueeze(2))
    host[:, :pages * P] = want.view(2, pages * P, 13)
    out, st = gpu_lib.resispec_commit_path(cache, slots, path, source=source, page_dim=1, position_dim=2)
    torch.cuda.synchronize()
    assert out is cache and (st == 0).all() and same(whole.cpu(), host)
    with pytest.raises(ValueError):
        gpu_lib.resispec_commit_path(cache, slots, path, source=whole[:, 1:1 + B * N].view(2, B, N, 13), page_dim=1, position_dim=2)
