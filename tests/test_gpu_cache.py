"""States of chosen beams, pages and slots, accepted paths and their rows: every output against
plain Python, value for value (nothing is computed but places)."""
import numpy as np
import pytest
import torch

from beam_util import accepted_path, plan

pytestmark = pytest.mark.gpu


def fill(shape, dtype, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randint(0, 256, (*shape, torch.empty(0, dtype=dtype).element_size()), generator=g, device="cuda",
                      dtype=torch.uint8)
    return x.view(dtype).view(shape)


def same(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def parents(B, K, W, seed=0, none=0.1):
    g = np.random.default_rng([seed, B, K, W])
    p = g.integers(0, W, (B, K))
    p[g.random((B, K)) < none] = -1
    return torch.as_tensor(p, dtype=torch.int32, device="cuda")


def expected(old, new, parent, W, lengths=None):
    """old [outer, B * W, inner, S, row] and new [outer, B * K, inner, S, row], on the host."""
    B, K = parent.shape
    out = new.clone()
    for b in range(B):
        n = old.shape[3] if lengths is None else int(lengths[b])
        for k in range(K):
            p = int(parent[b, k])
            if p >= 0:
                out[:, b * K + k, :, :n] = old[:, b * W + p, :, :n]
    return out


SHAPES = [  # B, W, K, outer, inner, S, row
    (1, 1, 1, 1, 1, 1, 1), (2, 4, 4, 3, 2, 5, 16), (3, 5, 5, 2, 3, 7, 17), (2, 8, 8, 1, 1, 40, 130), (1, 16, 16, 2, 1, 9, 33),
    (2, 17, 17, 1, 2, 6, 24), (1, 64, 64, 1, 1, 3, 70), (4, 3, 6, 2, 2, 11, 8), (2, 6, 2, 1, 1, 100, 256), (1, 2, 33, 1, 1, 4, 5),
    (3, 4, 4, 1, 1, 1, 8192), (1, 4, 4, 2, 2, 700, 64),
]


@pytest.mark.parametrize("dtype", [torch.uint8, torch.bfloat16, torch.float32], ids=["u8", "bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_reorder(gpu_lib, shape, dtype):
    B, W, K, outer, inner, S, row = shape
    print("reorder", shape, dtype, flush=True)
    old = fill((outer, B * W, inner, S, row), dtype)
    new = fill((outer, B * K, inner, S, row), dtype, 2)
    parent = parents(B, K, W)
    lengths = torch.as_tensor(np.random.default_rng(row).integers(0, S + 1, B), dtype=torch.int32, device="cuda")
    lengths[0] = S
    for n in (None, lengths):
        to = new.clone()
        want = expected(old.cpu(), new.cpu(), parent.cpu(), W, None if n is None else n.cpu())
        out, st = gpu_lib.resispec_beam_reorder(old, parent, beam_dim=1, position_dim=3, lengths=n, out=to)
        torch.cuda.synchronize()
        assert out is to and same(out.cpu(), want) and (st == 0).all()
        if K == W:
            state = old.clone()
            want = expected(old.cpu(), old.cpu(), parent.cpu(), W, None if n is None else n.cpu())
            out, st = gpu_lib.resispec_beam_reorder(state, parent, beam_dim=1, position_dim=3, lengths=n)
            torch.cuda.synchronize()
            assert out is state and same(out.cpu(), want) and (st == 0).all()


def test_reorder_strides(gpu_lib):
    """Positions before heads, parts of larger tensors, rows that start anywhere, plain states."""
    B, W = 2, 4
    parent = parents(B, W, W, 5)
    big = fill((3, B * W, 6, 20, 9), torch.bfloat16)
    for view in (lambda t: t[:, :, 1:5, 3:17, :7], lambda t: t[1:2, :, 2:3, :, 1:], lambda t: t[..., 8:9],
                 lambda t: t[:, :, :, ::2, :]):
        state = big.clone()
        want = expected(view(state).cpu(), view(state).cpu(), parent.cpu(), W)
        whole = state.cpu()
        view(whole).copy_(want)
        gpu_lib.resispec_beam_reorder(view(state), parent, beam_dim=1, position_dim=3)
        torch.cuda.synchronize()
        assert same(state.cpu(), whole)             # nothing else is written
    # [layers, beams, positions, heads, size]
    state = fill((2, B * W, 11, 3, 5), torch.float32)
    lengths = torch.tensor([4, 11], dtype=torch.int32, device="cuda")
    want = state.cpu().clone()
    for b in range(B):
        for k in range(W):
            if int(parent[b, k]) >= 0:
                want[:, b * W + k, :int(lengths[b])] = state.cpu()[:, b * W + int(parent[b, k]), :int(lengths[b])]
    gpu_lib.resispec_beam_reorder(state, parent, beam_dim=1, position_dim=2, lengths=lengths)
    torch.cuda.synchronize()
    assert same(state.cpu(), want)
    # no positions, beams first
    state = fill((B * W, 33), torch.float32)
    want = expected(state.cpu()[None, :, None, None], state.cpu()[None, :, None, None], parent.cpu(), W)[0, :, 0, 0]
    gpu_lib.resispec_beam_reorder(state, parent)
    torch.cuda.synchronize()
    assert same(state.cpu(), want)


def test_reorder_faults(gpu_lib):
    B, W, S = 6, 4, 5
    old = fill((1, B * W, 1, S, 8), torch.float32)
    parent = parents(B, W, W, 3, none=0.0)
    parent[1, 2], parent[2, 0] = W, -2
    lengths = torch.tensor([5, 5, 5, 6, -1, 0], dtype=torch.int32, device="cuda")
    state = old.clone()
    out, st = gpu_lib.resispec_beam_reorder(state, parent, beam_dim=1, position_dim=3, lengths=lengths)
    torch.cuda.synchronize()
    assert st.tolist() == [0, 10, 10, 10, 10, 0]
    want = old.cpu().clone()
    want[:, :W] = expected(old.cpu()[:, :W], old.cpu()[:, :W], parent[:1].cpu(), W)
    assert same(state.cpu(), want)


def paged_reference(cache, table, to_table, parent, lengths, P, out):
    """cache and out [outer, pages, inner, P, row] on the host."""
    B, K = parent.shape
    W = table.shape[0] // B
    res = out.clone()
    for b in range(B):
        for k in range(K):
            p = int(parent[b, k])
            for t in range(int(lengths[b])) if p >= 0 else ():
                f, d = int(table[b * W + p, t // P]), int(to_table[b * K + k, t // P])
                if 0 <= f < cache.shape[1] and 0 <= d < out.shape[1]:
                    res[:, d, :, t % P] = cache[:, f, :, t % P]
    return res


@pytest.mark.parametrize("B,W,K,outer,inner,P,row,longest", [
    (1, 1, 1, 1, 1, 1, 3, 4), (2, 4, 4, 2, 1, 16, 32, 40), (3, 5, 5, 1, 2, 24, 17, 100), (1, 8, 8, 2, 2, 7, 130, 30),
    (2, 17, 17, 1, 1, 4, 9, 21), (2, 3, 6, 2, 1, 16, 64, 33), (1, 64, 64, 1, 1, 2, 5, 7), (1, 2, 2, 1, 1, 64, 1024, 130)])
def test_reorder_paged(gpu_lib, B, W, K, outer, inner, P, row, longest):
    M = -(-longest // P) + 1
    pages = B * (W + K) * M + 3
    g = np.random.default_rng([B, W, P, row])
    order = torch.as_tensor(g.permutation(pages), dtype=torch.int32, device="cuda")
    table, other = order[:B * W * M].view(B * W, M), order[B * W * M:B * (W + K) * M].view(B * K, M)
    cache = fill((outer, pages, inner, P, row), torch.bfloat16)
    parent = parents(B, K, W, 9)
    lengths = torch.as_tensor(g.integers(0, longest + 1, B), dtype=torch.int32, device="cuda")
    lengths[0] = longest
    print("paged", B, W, K, P, row, lengths.tolist(), flush=True)
    kw = dict(page_dim=1, position_dim=3)
    # into other pages of the cache, or of another
    if K == W:
        state = cache.clone()
        want = paged_reference(cache.cpu(), table.cpu(), other.cpu(), parent.cpu(), lengths.cpu(), P, cache.cpu())
        out, st = gpu_lib.resispec_beam_reorder_paged(state, table, parent, lengths, out_table=other, **kw)
        torch.cuda.synchronize()
        assert out is state and same(out.cpu(), want) and (st == 0).all()
        # in place, with the first pages of every sequence shared by its beams
        shared = table.clone()
        if longest >= P:
            shared.view(B, W, M)[:, :, 0] = shared.view(B, W, M)[:, :1, 0]
        state = cache.clone()
        want = paged_reference(cache.cpu(), shared.cpu(), shared.cpu(), parent.cpu(), lengths.cpu(), P, cache.cpu())
        out, st = gpu_lib.resispec_beam_reorder_paged(state, shared, parent, lengths, **kw)
        torch.cuda.synchronize()
        assert same(out.cpu(), want) and (st == 0).all()
    to = fill(cache.shape, torch.bfloat16, 7)
    want = paged_reference(cache.cpu(), table.cpu(), other.cpu(), parent.cpu(), lengths.cpu(), P, to.cpu())
    out, st = gpu_lib.resispec_beam_reorder_paged(cache, table, parent, lengths, out_table=other, out=to, **kw)
    torch.cuda.synchronize()
    assert out is to and same(out.cpu(), want) and (st == 0).all()


def test_reorder_paged_faults(gpu_lib):
    """Page numbers outside the cache, lengths past the table: the rows concerned stay."""
    B, W, P, M, pages = 5, 3, 4, 3, 50
    cache = fill((1, pages, 1, P, 6), torch.uint8)
    table = torch.randperm(pages, device="cuda").int()[:B * W * M].view(B * W, M).contiguous()
    parent = torch.tensor([[1, 2, 0]] * B, dtype=torch.int32, device="cuda")
    lengths = torch.tensor([12, 12, 13, 5, -1], dtype=torch.int32, device="cuda")
    table[4, 1], table[3, 2] = pages, -1
    table[10, 2] = 1 << 30          # past its sequence's length: not looked at
    state = cache.clone()
    out, st = gpu_lib.resispec_beam_reorder_paged(state, table, parent, lengths, page_dim=1, position_dim=3)
    torch.cuda.synchronize()
    assert st.tolist() == [0, 11, 10, 0, 10]
    lengths[2] = lengths[4] = 0
    want = paged_reference(cache.cpu(), table.cpu(), table.cpu(), parent.cpu(), lengths.cpu(), P, cache.cpu())
    assert same(state.cpu(), want)


# ----------------------------------------------------------------------- plan ----

def run_plan(lib, kept, added, held, table, free, count, P, T, alias=False, pad=0):
    i32 = dict(dtype=torch.int32, device="cuda")
    R, M = len(kept), len(table[0]) if table else 1
    t = torch.full((max(R, 1), M + pad), -9, **i32)
    if R:
        t[:, :M] = torch.tensor(table, **i32)
    t = t[:R, :M]
    f, c, h = torch.tensor(free, **i32), torch.tensor([count], **i32), torch.tensor(held, **i32)
    before = [list(x) for x in table]
    want = plan(kept, added, held, table, free, count, P, T)
    print("plan R", R, "P", P, "T", T, "statuses", sorted(set(want[6])), flush=True)
    kw = dict(out_held=h, out_free_count=c) if alias else {}
    slots, positions, requests, starts, got, left, st = lib.resispec_plan_cache(
        torch.tensor(kept, **i32), torch.tensor(added, **i32), h, t, f, c, page_size=P, max_slots=T, **kw)
    torch.cuda.synchronize()
    assert st.tolist() == want[6]
    assert starts.tolist() == want[3]
    assert got.tolist() == want[4] and left.tolist() == [want[5]]
    assert t.tolist() == table and f.tolist() == free
    assert slots.tolist() == want[0]
    on = [i for i in range(T) if want[1][i] >= 0]
    assert [positions.tolist()[i] for i in on] == [want[1][i] for i in on]
    assert [i for i in range(T) if positions.tolist()[i] >= 0] == on
    assert requests.tolist() == want[2]
    return before


def batch(R, P, longest, most, seed, spare=4, pages=None):
    g = np.random.default_rng([R, P, seed])
    M = -(-(longest + most) // P)
    held_tokens = g.integers(0, longest + 1, R)
    held = [-(-int(x) // P) for x in held_tokens]
    kept = [int(max(0, x - g.integers(0, 2 * P + 1))) if g.random() < 0.9 else 0 for x in held_tokens]
    added = [int(g.integers(0, most + 1)) if g.random() < 0.9 else 0 for _ in range(R)]
    pages = pages or sum(held) + sum(-(-a // P) + 1 for a in added) + spare
    order = [int(x) for x in g.permutation(pages)]
    table, at = [], 0
    for h in held:
        table.append(order[at:at + h] + [-1] * (M - h))
        at += h
    free = order[at:] + [-1] * at
    return kept, added, held, table, free, pages - at


@pytest.mark.parametrize("R,P,longest,most", [(1, 16, 100, 26), (7, 1, 9, 5), (64, 16, 200, 33), (300, 24, 100, 40),
                                               (1023, 8, 60, 4), (1024, 16, 40, 3), (1025, 16, 40, 3), (3000, 7, 30, 2),
                                               (5, 128, 3000, 2000)])
def test_plan(gpu_lib, R, P, longest, most):
    for seed, alias, pad in ((0, False, 0), (1, True, 5)):
        args = batch(R, P, longest, most, seed)
        run_plan(gpu_lib, *args, P, sum(args[1]) + 13, alias, pad)


def test_plan_room(gpu_lib):
    """Too few pages, too few slots, exactly enough of both."""
    for seed in range(6):
        args = list(batch(50, 8, 60, 20, seed))
        args[5] = seed * 7                 # so many of the free pages are there
        run_plan(gpu_lib, *args, 8, sum(args[1]))
        args = batch(50, 8, 60, 20, seed)
        run_plan(gpu_lib, *args, 8, sum(args[1]) * seed // 6)
    # the pages that one request gives back are what the next takes
    table, free = [[0, 1, 2, -1], [3, -1, -1, -1]], [-1, -1, -1, -1]
    run_plan(gpu_lib, [0, 4], [0, 8], [3, 1], table, free, 0, 4, 8)
    assert table[1] == [3, 2, 1, -1] and free[:1] == [0]
    run_plan(gpu_lib, [0, 4], [0, 13], [3, 1], [[0, 1, 2, -1], [3, -1, -1, -1]], [-1] * 4, 0, 4, 13)


def test_plan_many_tokens(gpu_lib):
    """Rows in a launch of their own, prompts of many pages, padding."""
    for R, P, longest, most in ((3, 16, 500, 4000), (200, 32, 300, 100), (2000, 16, 64, 20)):
        args = batch(R, P, longest, most, 4)
        run_plan(gpu_lib, *args, P, sum(args[1]) + 3000)


def test_plan_faults(gpu_lib):
    P, M = 4, 3
    table = [[0, 1, -1], [2, -1, -1], [3, -1, -1], [4, 5, -1], [6, 99, 7], [8, -1, -1], [-5, -1, -1]]
    kept, added, held = [3, -1, 4, 2, 8, 12, 2], [4, 1, -1, 3, 2, 1, 1], [2, 1, 1, 4, 3, 1, 1]
    run_plan(gpu_lib, kept, added, held, table, [9, 10, 11] + [-1] * 9, 3, P, 20)
    # a page number outside the cache among the free ones
    run_plan(gpu_lib, [4, 0], [2, 1], [1, 0], [[0, -1], [-1, -1]], [1, 77, 2, -1], 3, P, 4)
    # counts that no stack of this size has, and pages given back that do not fit on it
    for count in (-1, 5):
        run_plan(gpu_lib, [4, 0, 2, 0], [2, 0, 1, 0], [1, 1, 1, 0], [[0, -1], [1, -1], [2, -1], [-1, -1]],
                 [3, -1, -1, -1], count, P, 4)
    run_plan(gpu_lib, [0, 0, 4], [0, 0, 4], [2, 1, 1], [[0, 1], [2, -1], [3, -1]], [0, 1, 2, 3], 2, P, 4)
    # no requests: the padding and the counts
    run_plan(gpu_lib, [], [], [], [], [0, 1, 2], 2, P, 6)


# ----------------------------------------------------------------------- path ----

def trees(B, N, seed, vocab=6):
    """Random trees, tokens that repeat among siblings, and what a verification may return."""
    g = np.random.default_rng([B, N, seed])
    parent = np.full((B, N), -1, dtype=np.int32)
    for n in range(1, N):
        parent[:, n] = np.minimum(n - 1, (n * g.random(B) ** 2).astype(np.int32))
    token = g.integers(0, vocab, (B, N)).astype(np.int32)
    ways = []
    for b in range(B):
        n, way = int(g.integers(0, N)), []
        while n > 0:
            way.append(int(token[b, n]))
            n = int(parent[b, n])
        ways.append(way[::-1])
    D = max(1, max(len(w) for w in ways)) + 1
    tokens = np.full((B, D + 1), -1, dtype=np.int32)
    for b, w in enumerate(ways):
        tokens[b, :len(w)] = w
        tokens[b, len(w)] = 999
    return parent, token, tokens, np.array([len(w) for w in ways], dtype=np.int32)


@pytest.mark.parametrize("B,N", [(1, 1), (1, 2), (5, 3), (3, 26), (40, 33), (64, 64), (9, 65), (7, 300), (2, 1024), (3, 1025),
                                 (1, 8192)])
def test_accepted_path(gpu_lib, B, N):
    for seed, vocab in ((0, 3), (1, 1000)):
        parent, token, tokens, length = trees(B, N, seed, vocab)
        print("path", B, N, vocab, flush=True)
        dev = [torch.as_tensor(x, device="cuda") for x in (parent, token, tokens, length)]
        path, st = gpu_lib.resispec_accepted_path(*dev)
        torch.cuda.synchronize()
        assert (st == 0).all()
        for b in range(B):
            way = accepted_path(parent[b].tolist(), token[b].tolist(), tokens[b].tolist(), int(length[b]))
            assert path[b].tolist() == way + [-1] * (tokens.shape[1] - len(way))


def test_accepted_path_faults(gpu_lib):
    parent, token, tokens, length = trees(8, 10, 3, 1000)
    D = tokens.shape[1] - 1
    length[0], length[1], length[2] = -1, -2, D + 1
    parent[3, 5] = 5
    parent[4, 0] = 0
    parent[5, 9] = -1
    length[6], tokens[6, 0] = 1, -77
    length[7] = 0
    path, st = gpu_lib.resispec_accepted_path(*(torch.as_tensor(x, device="cuda") for x in (parent, token, tokens, length)))
    torch.cuda.synchronize()
    assert st.tolist() == [0, 6, 6, 4, 4, 4, 4, 0]
    assert path[7].tolist() == [0] + [-1] * D
    assert (path[:7] == -1).all()


# --------------------------------------------------------------------- commit ----

def commit_reference(cache, slots, path, P, source=None):
    res = cache.clone()
    for b in range(path.shape[0]):
        for i in range(path.shape[1]):
            n = int(path[b, i])
            if n < 0:
                break
            s, d = int(slots[b, n]), int(slots[b, i])
            res[:, d // P, :, d % P] = cache[:, s // P, :, s % P] if source is None else source[:, b, :, n]
    return res


@pytest.mark.parametrize("B,N,depth,outer,inner,P,row", [
    (1, 1, 1, 1, 1, 1, 1), (3, 26, 5, 2, 1, 16, 64), (2, 33, 33, 1, 2, 7, 17), (5, 60, 12, 3, 1, 1, 130), (1, 300, 200, 1, 1, 64, 40),
    (4, 9, 4, 1, 3, 24, 2000), (40, 5, 3, 2, 2, 16, 9)])
@pytest.mark.parametrize("dtype", [torch.uint8, torch.bfloat16], ids=["u8", "bf16"])
def test_commit(gpu_lib, B, N, depth, outer, inner, P, row, dtype):
    g = np.random.default_rng([B, N, depth])
    pages = -(-B * N // P) + 2
    slots = torch.as_tensor(g.permutation(pages * P)[:B * N].reshape(B, N), dtype=torch.int32, device="cuda")
    path = np.full((B, depth), -1, dtype=np.int32)
    for b in range(B):
        n = int(g.integers(0, depth + 1))
        path[b, :n] = np.sort(g.permutation(N)[:n])
    path[0] = np.sort(g.permutation(N)[:depth])
    path = torch.as_tensor(path, device="cuda")
    cache = fill((outer, pages, inner, P, row), dtype)
    source = fill((outer, B, inner, N, row), dtype, 5)
    print("commit", B, N, depth, P, row, flush=True)
    for src in (None, source):
        state = cache.clone()
        want = commit_reference(cache.cpu(), slots.cpu(), path.cpu(), P, None if src is None else src.cpu())
        out, st = gpu_lib.resispec_commit_path(state, slots, path, source=src, page_dim=1, position_dim=3)
        torch.cuda.synchronize()
        assert out is state and same(out.cpu(), want) and (st == 0).all()


def test_commit_faults(gpu_lib):
    B, N, P = 7, 6, 4
    cache = fill((1, 12, 1, P, 8), torch.float32)
    slots = torch.arange(B * N, dtype=torch.int32, device="cuda").view(B, N).contiguous()
    path = torch.tensor([[0, 2, 4], [0, 2, 2], [1, 0, -1], [0, 6, -1], [0, 3, -1], [0, 3, -1], [-2, 1, 2]],
                        dtype=torch.int32, device="cuda")
    slots[4, 3], slots[5, 1] = 48, -1
    state = cache.clone()
    out, st = gpu_lib.resispec_commit_path(state, slots, path, page_dim=1, position_dim=3)
    torch.cuda.synchronize()
    assert st.tolist() == [0, 4, 4, 4, 11, 11, 4]
    want = commit_reference(cache.cpu(), slots[:1].cpu(), path[:1].cpu(), P)
    assert same(state.cpu(), want)
    # a slot outside the cache that only the verification used: the source is elsewhere
    state = cache.clone()
    source = fill((1, B, 1, N, 8), torch.float32, 3)
    out, st = gpu_lib.resispec_commit_path(state, slots, path, source=source, page_dim=1, position_dim=3)
    torch.cuda.synchronize()
    assert st.tolist() == [0, 4, 4, 4, 0, 11, 4]


def test_no_sequences(gpu_lib):
    i32 = dict(dtype=torch.int32, device="cuda")
    state = torch.zeros((2, 0, 3, 5), device="cuda")
    out, st = gpu_lib.resispec_beam_reorder(state, torch.zeros((0, 4), **i32), beam_dim=1, position_dim=2)
    assert out is state and st.shape == (0,)
    cache = torch.ones((6, 4, 8), device="cuda")
    out, st = gpu_lib.resispec_beam_reorder_paged(cache, torch.zeros((0, 3), **i32), torch.zeros((0, 4), **i32),
                                                  torch.zeros(0, **i32))
    assert out is cache and st.shape == (0,)
    out, st = gpu_lib.resispec_commit_path(cache, torch.zeros((0, 5), **i32), torch.zeros((0, 2), **i32))
    assert out is cache and st.shape == (0,)
    path, st = gpu_lib.resispec_accepted_path(torch.zeros((0, 5), **i32), torch.zeros((0, 5), **i32), torch.zeros((0, 2), **i32),
                                              torch.zeros(0, **i32))
    assert path.shape == (0, 2) and st.shape == (0,)


def test_places_past_32_bits(gpu_lib):
    """Beams of 3 GiB, and pages that lie more than 4 GiB into a cache."""
    n = 3 << 30
    state = torch.empty((2, n), dtype=torch.uint8, device="cuda")
    state[0].random_(generator=torch.Generator(device="cuda").manual_seed(1))
    state[1].fill_(7)
    first = state[0].clone()
    out, st = gpu_lib.resispec_beam_reorder(state, torch.tensor([[1, 0]], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert int(st) == 0 and bool((state[0] == 7).all()) and torch.equal(state[1], first)
    del first, out
    # 96 pages of 16 positions of 4 MiB: 6 GiB
    cache = state.view(-1).view(96, 16, 1 << 22)
    cache.random_(generator=torch.Generator(device="cuda").manual_seed(2))
    before = {(p, t): cache[p, t].clone() for p, t in ((95, 3), (95, 9), (94, 15), (2, 0), (93, 1))}
    slots = torch.tensor([[2 * 16, 95 * 16 + 3, 94 * 16 + 15, 95 * 16 + 9, 93 * 16 + 1]], dtype=torch.int32, device="cuda")
    path = torch.tensor([[0, 2, 3, 4]], dtype=torch.int32, device="cuda")
    gpu_lib.resispec_commit_path(cache, slots, path)
    torch.cuda.synchronize()
    for to, of in (((2, 0), (2, 0)), ((95, 3), (94, 15)), ((94, 15), (95, 9)), ((95, 9), (93, 1)), ((93, 1), (93, 1))):
        assert torch.equal(cache[to], before[of])
    table = torch.tensor([[95], [1]], dtype=torch.int32, device="cuda")
    a, b = cache[95, :2].clone(), cache[1, :2].clone()
    gpu_lib.resispec_beam_reorder_paged(cache, table, torch.tensor([[1, 0]], dtype=torch.int32, device="cuda"),
                                        torch.tensor([2], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert torch.equal(cache[95, :2], b) and torch.equal(cache[1, :2], a)


def test_streams_and_places_of_outputs(gpu_lib):
    """A stream given by the caller, and outputs that are the caller's."""
    side = torch.cuda.Stream()
    state = fill((4, 6, 5), torch.float32)
    parent = torch.tensor([[1, 0], [0, 0]], dtype=torch.int32, device="cuda")
    old = state.view(4, 6, 5).clone()
    st = torch.full((2,), -7, dtype=torch.int32, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    out, got = gpu_lib.resispec_beam_reorder(state, parent, beam_dim=0, position_dim=1, out_status=st, stream=side)
    side.synchronize()
    assert got is st and (st == 0).all()
    assert same(out, old[[1, 0, 2, 2]])         # any bits, NaNs among them
    args = batch(20, 8, 60, 20, 3)
    i32 = dict(dtype=torch.int32, device="cuda")
    want = plan(*(list(x) if not isinstance(x[0], list) else [list(y) for y in x] for x in args[:4]), list(args[4]), args[5], 8, 300)
    t, f = torch.tensor(args[3], **i32), torch.tensor(args[4], **i32)
    rest = [torch.tensor(x, **i32) for x in (args[0], args[1], args[2])]
    outs = dict(out_slots=torch.empty(300, **i32), out_positions=torch.empty(300, **i32), out_requests=torch.empty(300, **i32))
    side.wait_stream(torch.cuda.current_stream())
    res = gpu_lib.resispec_plan_cache(*rest, t, f, torch.tensor([args[5]], **i32), page_size=8, stream=side, **outs)
    side.synchronize()
    assert res[0] is outs["out_slots"] and res[0].tolist() == want[0] and res[6].tolist() == want[6]


def test_binding_refusals(gpu_lib):
    i32 = dict(dtype=torch.int32, device="cuda")
    state, parent = torch.zeros((2, 6, 5), device="cuda"), torch.zeros((2, 3), **i32)
    for kw in (dict(lengths=torch.zeros(2, **i32), beam_dim=1),                       # lengths of what
               dict(beam_dim=0), dict(beam_dim=1, out=state[:, 1:]), dict(beam_dim=1, out=state.double()),
               dict(beam_dim=1, out=torch.zeros((2, 5, 5), device="cuda")), dict(beam_dim=1, position_dim=0),
               dict(beam_dim=1, out=torch.zeros((2, 6, 6), device="cuda")), dict(beam_dim=1, out_status=torch.zeros(3, **i32))):
        with pytest.raises((ValueError, TypeError, gpu_lib.ResiSpecError)):
            gpu_lib.resispec_beam_reorder(state, parent, **kw)
    with pytest.raises(ValueError):
        gpu_lib.resispec_beam_reorder(state, torch.zeros((2, 4), **i32), beam_dim=1)       # in place, more than there are
    big = torch.zeros((2, 12, 5), device="cuda")
    with pytest.raises(ValueError):
        gpu_lib.resispec_beam_reorder(big[:, :6], parent, beam_dim=1, out=big[:, 3:9])     # partly the same rows
    cache, table = torch.zeros((9, 4, 5), device="cuda"), torch.zeros((6, 2), **i32)
    lengths = torch.zeros(2, **i32)
    for kw in (dict(out_table=torch.zeros((6, 3), **i32)), dict(out_table=torch.zeros((5, 2), **i32)), dict(out=cache[1:])):
        with pytest.raises((ValueError, gpu_lib.ResiSpecError)):
            gpu_lib.resispec_beam_reorder_paged(cache, table, parent, lengths, **kw)
    slots, path = torch.zeros((2, 4), **i32), torch.zeros((2, 3), **i32)
    for kw in (dict(source=torch.zeros((2, 5, 5), device="cuda")), dict(source=torch.zeros((2, 4, 6), device="cuda")),
               dict(source=torch.zeros((2, 4, 5), device="cuda", dtype=torch.float64)), dict(source=cache[:2])):
        with pytest.raises((ValueError, TypeError, gpu_lib.ResiSpecError)):
            gpu_lib.resispec_commit_path(cache, slots, path, **kw)
    ones = [torch.zeros(3, **i32) for _ in range(3)]
    with pytest.raises(ValueError):
        gpu_lib.resispec_plan_cache(*ones, torch.zeros((3, 2), **i32), torch.zeros(4, **i32), torch.zeros(1, **i32), page_size=4)
    with pytest.raises(ValueError):
        gpu_lib.resispec_plan_cache(*ones, torch.zeros((2, 3), **i32).t(), torch.zeros(4, **i32), torch.zeros(1, **i32),
                                    page_size=4, max_slots=4)
    with pytest.raises(gpu_lib.ResiSpecError):
        gpu_lib.resispec_plan_cache(*ones, torch.zeros((3, 2), **i32), torch.zeros(4, **i32), torch.zeros(1, **i32), page_size=0,
                                    max_slots=4)
