"""Beam search's choice (resispec_beam_select) against plain 64-bit numpy.

Parents and tokens have to be equal: no two candidates of different beams come closer to each
other here than 1e-12, but for those of equal rows, which are equal on both sides.  Scores: half
a step of the result, and the sum's error.  That sum is of 32-bit masses: an exponent x is off by
3 * 2^-24 of itself (difference, factor and product rounded), a mass by 0.693 of that and 2^-23 of
itself; over a unit of 4096 elements with its maximum at 0 the mean of |x| by mass is at most 8.1,
so 1.00e-6 + 1.2e-7; the additions of eight masses are three of 2^-24 each, 1.8e-7, and the rest
is added in 64 bits: 1.3e-6 in all, and the logarithm of the sum by as much."""
import numpy as np
import pytest
import torch

from beam_util import close_scores, log_sum, select
from sampling_util import make_rows, to64

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.bfloat16]
IDS = ["f32", "bf16"]


def check(lib, logits, scores, k, T=1.0, ended=None, end_token=2, **kw):
    B, W = scores.shape
    print("select", tuple(logits.shape), logits.dtype, "k", k, flush=True)
    parent, token, score, st = lib.resispec_beam_select(logits, scores, k=k, temperature=T, ended=ended,
                                                        end_token=end_token, **kw)
    torch.cuda.synchronize()
    l = to64(logits).reshape(B, W, -1)
    s = scores.cpu().numpy().astype(np.float64)
    e = None if ended is None else ended.cpu().numpy()
    t = T.cpu().numpy() if isinstance(T, torch.Tensor) else np.float32(T)
    for b in range(B):
        tb = t if t.ndim == 0 else t.reshape(B, -1)[b]
        want = select(l[b], s[b], k, tb, None if e is None else e[b], end_token)
        if want is None:
            assert int(st[b]) != 0
            assert (parent[b] == -1).all() and (token[b] == -1).all() and torch.isnan(score[b]).all()
            continue
        assert int(st[b]) == 0
        assert parent[b].tolist() == want[0], b
        assert token[b].tolist() == want[1], b
        assert close_scores(score[b].cpu().numpy(), want[2]), b
    return parent, token, score, st


def scores_for(B, W, seed=0, spread=4.0):
    g = torch.Generator(device="cuda").manual_seed(seed + 100 * W + B)
    return -20.0 - spread * torch.rand((B, W), generator=g, device="cuda")


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("V", [1, 2, 3, 7, 8, 64, 511, 512, 513, 1000, 4097, 32001])
def test_vocabularies(gpu_lib, V, dtype):
    for W, k in ((1, 1), (4, 4), (5, 10)):
        k = min(k, W * V)
        check(gpu_lib, make_rows(3 * W, V, dtype, V).view(3, W, V), scores_for(3, W), k, T=0.8)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("kind", ["zipf", "flat", "peaked", "equal", "few", "masked", "lowest", "all-lowest", "large"])
def test_values(gpu_lib, kind, dtype):
    for V, W, k in ((2000, 4, 8), (5000, 3, 64), (40, 2, 7)):
        check(gpu_lib, make_rows(4 * W, V, dtype, 11, kind).view(4, W, V), scores_for(4, W), k)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("W,k", [(1, 64), (2, 1), (3, 5), (8, 8), (16, 32), (17, 64), (33, 33), (64, 64), (64, 1)])
def test_beams(gpu_lib, W, k, dtype):
    check(gpu_lib, make_rows(2 * W, 3001, dtype, W + k).view(2, W, 3001), scores_for(2, W), k, T=1.3)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
def test_large_rows(gpu_lib, dtype):
    check(gpu_lib, make_rows(10, 151936, dtype, 5).view(2, 5, -1), scores_for(2, 5), 10, T=0.7)
    check(gpu_lib, make_rows(2, 1 << 22, dtype, 6).view(1, 2, -1), scores_for(1, 2), 4)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
def test_strides_and_places(gpu_lib, dtype):
    """Rows apart, rows that start anywhere, [B * W, V] rows; what lies between is not read."""
    for V, pad, offset in ((1000, 24, 0), (1001, 1, 1), (4096, 8, 3), (5, 2, 1)):
        rows = make_rows(8, V, dtype, 21, pad=pad, offset=offset)
        check(gpu_lib, rows, scores_for(2, 4), min(6, 4 * V))


def test_same_rows_twice(gpu_lib):
    """Beams with equal rows and scores: equal scores, the lower beam first."""
    row = make_rows(1, 3000, torch.bfloat16, 9)
    logits = row.expand(4, 3000).contiguous().view(1, 4, 3000)
    check(gpu_lib, logits, torch.full((1, 4), -3.0, device="cuda"), 10)
    check(gpu_lib, logits, torch.tensor([[-3.0, -2.0, -3.0, -2.0]], device="cuda"), 64)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
def test_scores_that_nearly_meet(gpu_lib, dtype):
    """Candidates of two beams 2e-8 to 3e-7 apart, below what a 32-bit sum may be off by: the rows
    are summed again.  (The 32-bit sums of these rows have the same order; test_gpu_beam_close has
    rows whose sums do not.)"""
    V = 3000
    rows = make_rows(2, V, dtype, 31)
    l = to64(rows)
    tops = [np.sort(x)[::-1] for x in l]
    lse = [log_sum(x, 1.0) for x in l]
    for step in (1, -1):
        # the first beam's best and the second's: scores in 64 bits from fp32 ones, moved by
        # shifting a row by a constant, which changes no probability
        s = np.zeros(2)
        s[0] = -2.0
        a = (tops[0][0] - lse[0][0]) - lse[0][1] + s[0]
        s[1] = np.float32(a - ((tops[1][0] - lse[1][0]) - lse[1][1]))
        for _ in range(3):
            check(gpu_lib, rows.view(1, 2, V), torch.tensor(s[None], dtype=torch.float32, device="cuda"), 5)
            s[1] = np.nextafter(np.float32(s[1]), np.float32(step * 100.0))


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
def test_close_beams(gpu_lib, dtype):
    """Many beams whose rows are permutations of one another, their scores 1e-3 apart: candidates of
    all of them are among the chosen, in turn."""
    V, W = 4000, 6
    g = torch.Generator(device="cuda").manual_seed(3)
    row = make_rows(1, V, dtype, 13)[0]
    logits = torch.stack([torch.cat((row[:10], row[10:][torch.randperm(V - 10, generator=g, device="cuda")]))
                          for _ in range(W)]).view(1, W, V)
    scores = -2.0 - torch.arange(W, device="cuda").float().view(1, W) * 1e-3
    check(gpu_lib, logits, scores, 20)


def test_beams_that_are_not_there(gpu_lib):
    """A first step, gaps, none at all; rows that are not read may hold anything."""
    logits = make_rows(12, 700, torch.float32, 3).view(3, 4, 700).contiguous()
    scores = torch.full((3, 4), float("-inf"), device="cuda")
    scores[0, 0], scores[1, 1], scores[1, 3] = 0.0, -1.0, -1.5
    logits[2] = float("nan")
    logits[0, 1:] = float("inf")
    logits[1, 0] = float("nan")
    parent, token, score, st = check(gpu_lib, logits, scores, 8)
    assert (parent[2] == -1).all() and (score[2] == float("-inf")).all() and (st == 0).all()


def test_fewer_than_k(gpu_lib):
    logits = torch.tensor([[1.0, float("-inf"), 0.5], [0.0, float("-inf"), float("-inf")]], device="cuda").view(1, 2, 3)
    parent, token, score, st = check(gpu_lib, logits, torch.tensor([[-1.0, -2.0]], device="cuda"), 6)
    assert parent.tolist() == [[0, 0, 1, -1, -1, -1]] and int(st) == 0


@pytest.mark.parametrize("kind", [torch.uint8, torch.bool], ids=["u8", "bool"])
def test_ended_beams(gpu_lib, kind):
    B, W, V = 6, 5, 900
    logits = make_rows(B * W, V, torch.bfloat16, 4).view(B, W, V).contiguous()
    ended = (torch.arange(B * W, device="cuda").view(B, W) % 3 == 1).to(kind)
    ended[4], ended[5] = 1, 0
    logits[ended.bool()] = float("nan")         # not read
    scores = scores_for(B, W, spread=2.0)
    for k in (1, 5, 10):
        check(gpu_lib, logits, scores, k, ended=ended, end_token=V + 7)
    # the ended beams' scores are far above, equal to each other
    scores = torch.where(ended.bool(), torch.full_like(scores, -0.5), scores)
    check(gpu_lib, logits, scores, 7, ended=ended, end_token=0)


def test_temperatures(gpu_lib):
    B, W, V = 3, 4, 1200
    logits = make_rows(B * W, V, torch.bfloat16, 8).view(B, W, V)
    each = torch.tensor([0.5, 1.0, 1.7], device="cuda")
    check(gpu_lib, logits, scores_for(B, W), 8, T=each)
    check(gpu_lib, logits, scores_for(B, W), 8, T=each.repeat(4).view(B, W).contiguous())
    check(gpu_lib, logits, scores_for(B, W), 8, T=1e-3)
    check(gpu_lib, logits, scores_for(B, W), 8, T=1e4)


def test_faults(gpu_lib):
    B, W, V = 8, 3, 600
    logits = make_rows(B * W, V, torch.float32, 2).view(B, W, V).contiguous()
    scores = scores_for(B, W)
    T = torch.ones(B, device="cuda")
    logits[1, 2, 599] = float("nan")
    logits[2, 0, 0] = float("inf")
    logits[3, 1] = float("-inf")
    scores[4, 1] = float("nan")
    scores[5, 0] = float("inf")
    T[6] = 0.0
    parent, token, score, st = gpu_lib.resispec_beam_select(logits, scores, temperature=T)
    torch.cuda.synchronize()
    assert st.tolist() == [0, 3, 3, 3, 10, 10, 10, 0]
    for b in (0, 7):
        want = select(to64(logits[b]), scores[b].cpu().numpy(), W)
        assert parent[b].tolist() == want[0] and token[b].tolist() == want[1]
    for b in range(1, 7):
        assert (parent[b] == -1).all() and (token[b] == -1).all() and torch.isnan(score[b]).all()


def test_batch_does_not_matter(gpu_lib):
    """A sequence's outputs, bit for bit, alone and in a batch."""
    B, W, V = 70, 4, 20011
    logits = make_rows(B * W, V, torch.bfloat16, 77).view(B, W, V).contiguous()
    scores = scores_for(B, W)
    whole = gpu_lib.resispec_beam_select(logits, scores, k=8)
    for b in (0, 33, 69):
        one = gpu_lib.resispec_beam_select(logits[b:b + 1], scores[b:b + 1], k=8)
        torch.cuda.synchronize()
        for x, y in zip(whole, one):
            assert torch.equal(x[b:b + 1], y)


def test_no_sequences(gpu_lib):
    out = gpu_lib.resispec_beam_select(torch.zeros((0, 4, 10), device="cuda"), torch.zeros((0, 4), device="cuda"))
    assert [tuple(x.shape) for x in out] == [(0, 4), (0, 4), (0, 4), (0,)]


def test_graph_and_streams(gpu_lib):
    """Two captured graphs that share a workspace, replayed in turn between eager calls on
    another stream with a workspace of its own."""
    B, W, V, k = 4, 4, 9001, 8
    data = [(make_rows(B * W, V, torch.bfloat16, 40 + i).view(B, W, V).contiguous(), scores_for(B, W, i)) for i in range(4)]
    ws = torch.empty(gpu_lib.resispec_beam_workspace_bytes(B, W, V), dtype=torch.uint8, device="cuda")
    ref = [tuple(x.clone() for x in gpu_lib.resispec_beam_select(l, s, k=k)) for l, s in data]
    logits, scores = data[0][0].clone(), data[0][1].clone()
    graphs, outs = [], []
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            outs.append(gpu_lib.resispec_beam_select(logits, scores, k=k, workspace=ws))
        graphs.append(g)
    for i in (0, 1, 2, 3, 1):
        logits.copy_(data[i][0])
        scores.copy_(data[i][1])
        torch.cuda.synchronize()
        other = gpu_lib.resispec_beam_select(*data[(i + 1) % 4], k=k, stream=side)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for out in outs:
            assert all(torch.equal(x, y) for x, y in zip(out, ref[i]))
        assert all(torch.equal(x, y) for x, y in zip(other, ref[(i + 1) % 4]))


def test_scores_far_apart_and_far_from_zero(gpu_lib):
    """Scores so large that a logit's difference is below their last bit, and beams farther apart
    than 32 bits hold in steps of 1/16."""
    logits = make_rows(8, 900, torch.float32, 15).view(2, 4, 900)
    for scores in ([-1e6, -1e6, -1e6 - 1, -1e6 + 2], [-1e12, -1e12, -1e12, -2e12], [-1e30, -1e30, -3e38, 0.0],
                   [3e38, -3e38, 0.0, 1.0]):
        s = torch.tensor([scores, scores[::-1]], device="cuda")
        check(gpu_lib, logits, s, 9)
        check(gpu_lib, logits, s, 9, ended=torch.tensor([[0, 1, 1, 0]] * 2, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("T", [0.01, 0.5, 1.0, 3.0])
def test_lowest_values_are_chosen(gpu_lib, T, dtype):
    """So few others that elements masked with the type's lowest value are among the chosen, at
    scores past 32 bits where T < 1; and beams that have such a score."""
    low = torch.finfo(dtype).min
    logits = make_rows(4, 40, dtype, 3).view(2, 2, 40)
    masked = logits.clone()
    masked[:, :, 3:] = low
    for rows, scores, k in ((masked, [-1.0, -2.0], 20), (masked[:, :, 1:], [-1.0, -2.0], 64), (masked, [low, -1.0], 50),
                            (logits, [-1.0, low], 60), (logits, [low, low], 60)):
        check(gpu_lib, rows.contiguous(), torch.tensor([scores, scores], device="cuda"), k, T=T)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
def test_many_alike(gpu_lib, dtype):
    """More equal elements, and more chunks with the same maximum, than the lists hold, beside
    beams whose rows have an order."""
    V = 1 << 20
    rows = torch.zeros((3, V), dtype=dtype, device="cuda")
    rows[1, 700000:] = 1.0
    rows[2] = make_rows(1, V, dtype, 2)[0]
    check(gpu_lib, rows.view(1, 3, V), torch.tensor([[-3.0, -4.0, -14.0]], device="cuda"), 40)
    check(gpu_lib, rows.view(1, 3, V), torch.tensor([[-3.0, -3.0, -3.0]], device="cuda"), 64)


def test_fewer_chunks_than_chosen(gpu_lib):
    """One beam of a vocabulary with fewer chunks than continuations are asked for."""
    for V in (700, 5000, 33000):
        for dtype in DTYPES:
            check(gpu_lib, make_rows(2, V, dtype, V).view(2, 1, V), scores_for(2, 1), 64)


def test_binding_refusals(gpu_lib):
    l, s = torch.zeros((2, 3, 10), device="cuda"), torch.zeros((2, 3), device="cuda")
    i = lambda *n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
    for kw in (dict(k=0), dict(k=31), dict(k=1 << 33), dict(temperature=0.0), dict(temperature=float("nan")),
               dict(ended=i(2, 3)), dict(ended=[1]), dict(ended=torch.zeros((3, 2), dtype=torch.uint8, device="cuda")),
               dict(end_token=1 << 31), dict(out_parent=i(2, 4)), dict(out_score=i(2, 3)), dict(out_status=i(3)),
               dict(workspace=torch.empty(8, dtype=torch.uint8, device="cuda")), dict(workspace=i(4096)),
               dict(temperature=torch.ones(3, device="cuda"))):
        with pytest.raises((ValueError, TypeError, gpu_lib.ResiSpecError)):
            gpu_lib.resispec_beam_select(l, s, **kw)
    for a, b in ((l, s[:, :2].contiguous()), (l, s.view(6)), (l.half(), s), (l, s.double()), (l.transpose(1, 2), s),
                 (l[:, :1].expand(2, 3, 10), s), (l, s.t().contiguous().t()), (l.view(6, 10)[:5], s)):
        with pytest.raises((ValueError, TypeError)):
            gpu_lib.resispec_beam_select(a, b)
