"""Draws from filtered rows, filtered rows and log-probabilities of tokens on the GPU against
the plain 64-bit definition (sampling_util).

Tokens, kept sets and ranks are compared exactly: kernel and definition both sum in 64 bits,
so they part only where a draw or a cut lies within about 1e-13 of a border, which no row
here does by chance (rows of equal values have exact sums on both sides).

Tolerances.  A log-probability of a draw is a 64-bit value rounded once to 32 bits: half a
step, 2^-24 of it, and 1e-12 for the exponentials (3.7e-14 each) and the sums.  One of a
given token comes from a sum of 32-bit exponentials: the exponent's rounding is at most 2^-24
of up to 64 (what is smaller than 2^-64 does not count), 64 * 2^-24 * ln 2 = 2.7e-6 of a
term; the exponential's own 2^-23; a 32-bit sum of up to 32 terms 32 * 2^-24 = 1.9e-6.
Together 4.8e-6 of the sum, as much in its logarithm."""
import numpy as np
import pytest
import torch

from sampling_util import border, draw, kept, logprob, make_rows, to64

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
SETTINGS = [dict(), dict(temperature=0.7, top_k=50, top_p=0.95), dict(top_k=1), dict(top_k=7),
            dict(temperature=1.3, top_p=0.9), dict(temperature=0.05, top_p=0.999), dict(temperature=0.6, min_p=0.05),
            dict(top_k=300, top_p=0.5, min_p=0.001), dict(temperature=50.0, top_p=0.3), dict(top_p=1e-6),
            dict(min_p=1.0), dict(top_p=1.0 - 2.0 ** -24), dict(top_k=1000000)]


def uniforms(R, k, seed=0):
    g = np.random.default_rng([seed, R, k])
    u = (g.integers(0, 1 << 24, (R, k)) * 2.0 ** -24).astype(np.float32)
    if k > 1:
        u[:, 0], u[:, 1] = 0.0, 1.0 - 2.0 ** -24
    return torch.as_tensor(u, device="cuda")


def check_sample(native, rows, u, each=None, **kw):
    """One call on rows [R, V] against the definition; `each`: the settings of every row."""
    tok, lp, n, st = native.resispec_sample(rows, u, **kw)
    torch.cuda.synchronize()
    l, uu = to64(rows), u.cpu().numpy()
    for r in range(rows.shape[0]):
        s = each[r] if each else {k: v for k, v in kw.items() if not isinstance(v, torch.Tensor)}
        check_row(native, l[r], uu[r], s, tok[r].tolist(), lp[r].tolist(), int(n[r]), int(st[r]))


def check_row(native, l, u, s, tok, lp, n, st):
    s = {"T" if k == "temperature" else k: v for k, v in s.items()}
    mask = kept(l, **s)
    if mask is None:
        assert st == native.RS_SEQ_UNDERFLOW and n == -1
        assert all(t == -1 for t in tok) and all(np.isnan(lp))
        return
    assert st == native.RS_SEQ_OK
    assert n == mask.sum()
    for i, x in enumerate(u):
        j, p = draw(l, s.get("T", 1.0), mask, x)
        assert tok[i] == j, (tok[i], j, x, border(l, s.get("T", 1.0), mask, x))
        assert abs(lp[i] - p) <= abs(p) * 2.0 ** -24 + 1e-12, (lp[i], p)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("kind", ["zipf", "flat", "peaked", "equal", "few", "masked", "lowest", "all-lowest", "large"])
def test_sample_kinds_of_rows(gpu_lib, kind, dtype):
    """Every kind of row under every setting, a vocabulary of several slots."""
    rows = make_rows(3, 5003, dtype, 1, kind)
    for i, s in enumerate(SETTINGS):
        check_sample(gpu_lib, rows, uniforms(3, 5, i), **s)


KINDS = ["zipf", "flat", "peaked", "equal", "few", "masked", "lowest", "all-lowest", "large"]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("kind", KINDS)
def test_sample_kinds_of_long_rows(gpu_lib, kind, dtype):
    """The same over vocabularies long enough for every way a cut is found."""
    rows = make_rows(2, 70001, dtype, 2, kind)
    for i, s in enumerate(SETTINGS):
        check_sample(gpu_lib, rows, uniforms(2, 4, i), **s)


@pytest.mark.parametrize("kind", ["zipf", "few", "lowest"])
def test_sample_f32_rows_of_bf16_values(gpu_lib, kind):
    """fp32 rows that hold many equal values, as logits cast from bf16 do: more of them at the
    cut than are sorted."""
    rows = make_rows(2, 131077, F32, 5, kind).bfloat16().float()
    for i, s in enumerate(SETTINGS + [dict(top_p=0.99), dict(temperature=3.0, top_p=0.8), dict(top_k=30000)]):
        check_sample(gpu_lib, rows, uniforms(2, 3, i), **s)
    want, count = expected_filter(rows, [dict(top_p=0.99)] * 2)
    out, n, st = gpu_lib.resispec_filter_logits(rows, top_p=0.99)
    torch.cuda.synchronize()
    assert same_bits(out, want) and n.tolist() == count


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_values_next_to_zero_and_far_from_it(gpu_lib, dtype):
    """Values that share a place in the counts of a bf16 row: next to zero, and past a
    thousand; and a maximum that the row's sample misses by far."""
    g = np.random.default_rng(77)
    V = 33000
    tiny = torch.as_tensor(g.standard_normal((1, V)) * 1e-13, device="cuda")
    mixed = torch.as_tensor(np.where(g.random((1, V)) < 0.3, 0.0, g.standard_normal((1, V)) * 1e-12), device="cuda")
    signs = torch.as_tensor(np.where(g.random((1, V)) < 0.5, -0.0, 0.0), device="cuda")
    far = torch.as_tensor(g.standard_normal((1, V)) * 3000.0, device="cuda")
    low = torch.as_tensor(-2000.0 + 900.0 * g.standard_normal((1, V)), device="cuda")
    lone = torch.as_tensor(g.standard_normal((1, V)), device="cuda")
    lone[0, 12345] = 900.0
    for x in (tiny, mixed, signs, far, low, lone):
        rows = x.to(dtype)
        for i, s in enumerate((dict(), dict(top_k=40), dict(top_p=0.9), dict(top_p=0.5, min_p=0.2), dict(top_k=9000),
                               dict(temperature=1e-3, top_p=0.97), dict(temperature=300.0, top_p=0.6),
                               dict(temperature=20.0, min_p=0.3))):
            check_sample(gpu_lib, rows, uniforms(1, 3, i), **s)
        each, t = row_settings(13)
        many = rows.expand(13, V).contiguous()
        want, count = expected_filter(many, each)
        out, n, st = gpu_lib.resispec_filter_logits(many, **t)
        torch.cuda.synchronize()
        assert same_bits(out, want) and n.tolist() == count


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 3, 4, 7, 8, 9, 63, 64, 65, 511, 512, 1023, 1025, 2047, 2048, 2049, 16384, 32001])
def test_sample_sizes(gpu_lib, V, dtype):
    for pad, offset in ((0, 0), (5, 0), (16 - V % 8, 8), (1, 3)):
        rows = make_rows(2, V, dtype, V, pad=pad, offset=offset)
        for s in (dict(temperature=0.8), dict(top_k=max(1, V // 3)), dict(top_p=0.7), dict(min_p=0.1, top_p=0.99)):
            check_sample(gpu_lib, rows, uniforms(2, 3, V), **s)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_sample_many_draws(gpu_lib, dtype):
    rows = make_rows(2, 40003, dtype, 9)
    for s in (dict(), dict(top_p=0.97), dict(top_k=17)):
        check_sample(gpu_lib, rows, uniforms(2, 64), **s)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("top_k", [0, 5, 2000, 20000])
def test_long_rows(gpu_lib, dtype, top_k):
    """The longest vocabularies of real checkpoints, and far past them."""
    for V in (151936, 262145, 1 << 20):
        rows = make_rows(2, V, dtype, V)
        check_sample(gpu_lib, rows, uniforms(2, 4), temperature=0.9, top_k=top_k, top_p=0.95)
    rows = make_rows(1, 300001, dtype, 4, "few")     # ties by the ten thousand
    check_sample(gpu_lib, rows, uniforms(1, 4), top_k=top_k, top_p=0.6)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_largest_vocabulary(gpu_lib, dtype):
    V = 1 << 22
    rows = make_rows(1, V, dtype, 3)
    check_sample(gpu_lib, rows, uniforms(1, 2), top_p=0.9)
    check_sample(gpu_lib, rows, uniforms(1, 2), top_k=100)
    out, n, st = gpu_lib.resispec_filter_logits(rows, top_k=100)
    torch.cuda.synchronize()
    assert int(torch.isfinite(out).sum()) == 100 == int(n[0])


def row_settings(R, device="cuda"):
    each = [SETTINGS[r % len(SETTINGS)] for r in range(R)]
    full = [dict(dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0), **s) for s in each]
    t = dict(temperature=torch.tensor([s["temperature"] for s in full], dtype=F32, device=device),
             top_k=torch.tensor([s["top_k"] for s in full], dtype=torch.int32, device=device),
             top_p=torch.tensor([s["top_p"] for s in full], dtype=F32, device=device),
             min_p=torch.tensor([s["min_p"] for s in full], dtype=F32, device=device))
    return each, t


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("R", [13, 300])
def test_settings_of_each_row(gpu_lib, R, dtype):
    """Every row has settings of its own; all four arrays, and one of them beside numbers."""
    rows = make_rows(R, 3001, dtype, R)
    each, t = row_settings(R)
    check_sample(gpu_lib, rows, uniforms(R, 2), each, **t)
    for name in t:
        one = [dict(temperature=0.8, top_k=40, top_p=0.9, min_p=0.01) for _ in range(R)]
        kw = dict(one[0])
        for r in range(R):
            one[r][name] = t[name][r].item()
        kw[name] = t[name]
        check_sample(gpu_lib, rows, uniforms(R, 2), one, **kw)


def test_settings_of_each_sequence(gpu_lib):
    """[B, N, V] rows: an entry a sequence covers its N rows; an entry a row is taken too."""
    B, N, V = 5, 7, 2111
    rows = make_rows(B * N, V, BF16, 2).view(B, N, V)
    each, t = row_settings(B)
    u = uniforms(B * N, 3).view(B, N, 3)
    got = gpu_lib.resispec_sample(rows, u, **t)
    spread = {k: v.repeat_interleave(N).view(B, N) for k, v in t.items()}
    again = gpu_lib.resispec_sample(rows, u, **spread)
    torch.cuda.synchronize()
    for x, y in zip(got, again):
        assert torch.equal(x, y)
    assert got[0].shape == (B, N, 3) and got[2].shape == (B, N)
    l, uu = to64(rows), u.cpu().numpy()
    for b in range(B):
        for n in range(N):
            check_row(gpu_lib, l[b, n], uu[b, n], each[b], got[0][b, n].tolist(), got[1][b, n].tolist(),
                      int(got[2][b, n]), int(got[3][b, n]))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("V", [4099, 70001])
def test_rows_without_a_distribution(gpu_lib, V, dtype):
    """NaN of either sign, +inf and rows of -inf are reported, and do not touch their
    neighbours."""
    rows = make_rows(9, V, dtype, 6)
    rows[1, 4098] = float("nan")
    rows[3, V // 2] = -torch.tensor(float("nan"))
    rows[2, 0] = float("inf")
    rows[4] = float("-inf")
    rows[5] = float("nan")
    rows[7] = float("-inf")
    rows[7, 77] = -3.0                     # one finite element: always drawn
    for s in SETTINGS:
        check_sample(gpu_lib, rows, uniforms(9, 3), **s)
    tok, lp, n, st = gpu_lib.resispec_sample(rows, uniforms(9, 3), top_p=0.5)
    torch.cuda.synchronize()
    assert tok[7].tolist() == [77] * 3 and lp[7].tolist() == [0.0] * 3 and int(n[7]) == 1
    out, n, st = gpu_lib.resispec_filter_logits(rows, top_p=0.5)
    lpt, rank, st2 = gpu_lib.resispec_token_logprobs(rows, torch.zeros((9, 2), dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    for r in (1, 2, 3, 4, 5):
        assert (out[r] == float("-inf")).all() and int(n[r]) == -1
        assert int(st[r]) == int(st2[r]) == gpu_lib.RS_SEQ_UNDERFLOW
        assert torch.isnan(lpt[r]).all() and (rank[r] == -1).all()
    assert (st[[0, 6, 7, 8]] == 0).all() and (st2[[0, 6, 7, 8]] == 0).all()


def test_bad_uniforms_and_settings(gpu_lib):
    rows = make_rows(6, 1000, F32, 8)
    u = uniforms(6, 3)
    u[1, 2], u[2, 0], u[3, 1] = 1.0, -0.25, float("nan")
    tok, lp, n, st = gpu_lib.resispec_sample(rows, u)
    torch.cuda.synchronize()
    bad = gpu_lib.RS_SEQ_BAD_UNIFORM
    assert st.tolist() == [0, bad, bad, bad, 0, 0]
    assert (tok[1:4] == -1).all() and torch.isnan(lp[1:4]).all() and (n[1:4] == -1).all()
    assert (tok[[0, 4, 5]] >= 0).all()
    f = dict(device="cuda", dtype=F32)
    for kw in (dict(temperature=torch.tensor([1, 0, -1, float("inf"), float("nan"), 1.0], **f)),
               dict(top_k=torch.tensor([0, -1, -5, -2 ** 31, -3, 4], device="cuda", dtype=torch.int32)),
               dict(top_p=torch.tensor([1, 0, -1, 1.01, float("nan"), 0.5], **f)),
               dict(min_p=torch.tensor([0, -0.1, 1.01, -float("inf"), float("nan"), 0.5], **f))):
        bad = gpu_lib.RS_SEQ_BAD_PARAM
        tok, lp, n, st = gpu_lib.resispec_sample(rows, uniforms(6, 3), **kw)
        out, n2, st2 = gpu_lib.resispec_filter_logits(rows, **kw)
        torch.cuda.synchronize()
        assert st.tolist() == st2.tolist() == [0, bad, bad, bad, bad, 0]
        assert (tok[1:5] == -1).all() and (n[1:5] == -1).all() and (n2[1:5] == -1).all()
        assert (out[1:5] == float("-inf")).all() and (out[0] == rows[0]).any()
        if "temperature" in kw:
            lp, rank, st3 = gpu_lib.resispec_token_logprobs(rows, tok, **kw)
            torch.cuda.synchronize()
            assert st3.tolist() == st.tolist() and torch.isnan(lp[1:5]).all() and (rank[1:5] == -1).all()


def same_bits(a, b):
    t = torch.int16 if a.dtype == BF16 else torch.int32
    return torch.equal(a.contiguous().view(t), b.contiguous().view(t))


def expected_filter(rows, each):
    l, out, n = to64(rows), rows.clone(), []
    for r in range(rows.shape[0]):
        s = {"T" if k == "temperature" else k: v for k, v in each[r].items()}
        mask = kept(l[r], **s)
        out[r][torch.as_tensor(~mask, device=rows.device)] = float("-inf")
        n.append(int(mask.sum()))
    return out, n


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("V", [5003, 70001])
def test_filter_kinds_of_rows(gpu_lib, V, kind, dtype):
    rows = make_rows(13, V, dtype, 11, kind)
    each, t = row_settings(13)
    want, count = expected_filter(rows, each)
    out, n, st = gpu_lib.resispec_filter_logits(rows, **t)
    torch.cuda.synchronize()
    assert same_bits(out, want) and n.tolist() == count and (st == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 3, 5, 8, 9, 64, 513, 2048, 2051, 4096, 32001])
def test_filter_sizes_strides_and_places(gpu_lib, V, dtype):
    """Padded and shifted inputs and outputs, and in place: what lies between rows stays."""
    each, t = row_settings(13)
    for pad, offset, opad, ooffset in ((0, 0, 0, 0), (3, 1, 5, 2), (8, 8, 0, 1), (0, 0, 16 - V % 8, 8)):
        rows = make_rows(13, V, dtype, V, pad=pad, offset=offset)
        want, count = expected_filter(rows, each)
        store = torch.full((ooffset + 13 * (V + opad) + 9,), 7.0, dtype=dtype, device="cuda")
        out = store[ooffset:ooffset + 13 * (V + opad)].view(13, V + opad)[:, :V]
        got, n, st = gpu_lib.resispec_filter_logits(rows, out=out, **t)
        torch.cuda.synchronize()
        assert got is out and same_bits(out, want) and n.tolist() == count
        out.fill_(7.0)
        assert (store == 7.0).all()                       # nothing outside the rows was written
        whole = rows.as_strided((13 * (V + pad),), (1,)) if pad else None
        got, n, st = gpu_lib.resispec_filter_logits(rows, out=rows, **t)
        torch.cuda.synchronize()
        assert same_bits(rows, want) and n.tolist() == count
        if pad:
            assert torch.isnan(whole.view(13, V + pad)[:, V:]).all()


HELD = {F32: [4, 31, 2047, 2048, 2049, 32767, 32768, 32769, 65535, 65536, 65537],
        BF16: [8, 33, 4095, 4096, 4097, 65535, 65536, 65537, 131071, 131072, 131073]}


@pytest.mark.parametrize("V, dtype", [(V, d) for d in HELD for V in HELD[d]], ids=str)
def test_filter_under_min_p_alone(gpu_lib, V, dtype):
    """Rows that registers hold, and the first that they do not: padded, in place, a setting a
    row, faulted rows among them."""
    R = 7
    for i, (kind, pad, offset) in enumerate((("zipf", 0, 0), ("masked", 3, 1), ("lowest", 8, 0), ("few", 1, 5))):
        rows = make_rows(R, V, dtype, 31 + i, kind, pad=pad, offset=offset)
        for min_p in (0.0, 0.03, 1.0):
            each = [dict(min_p=min_p)] * R
            want, count = expected_filter(rows, each)
            out, n, st = gpu_lib.resispec_filter_logits(rows, min_p=min_p)
            torch.cuda.synchronize()
            assert same_bits(out, want) and n.tolist() == count and (st == 0).all()
        per_row = torch.linspace(0.001, 0.9, R, device="cuda")
        warm = torch.linspace(0.3, 2.0, R, device="cuda")
        want, count = expected_filter(rows, [dict(min_p=float(p), T=float(t)) for p, t in zip(per_row, warm)])
        base = rows._base.clone() if rows._base is not None else rows.clone()
        out, n, st = gpu_lib.resispec_filter_logits(rows, min_p=per_row, temperature=warm, out=rows)
        torch.cuda.synchronize()
        assert same_bits(out, want) and n.tolist() == count and (st == 0).all()
        flat = rows._base if rows._base is not None else rows
        if pad:      # what lies between the rows is as it was
            between = torch.ones(flat.numel(), dtype=torch.bool, device="cuda")
            between[offset:].view(R, V + pad)[:, :V] = False
            assert same_bits(flat.flatten()[between], base.flatten()[between])
    rows = make_rows(R, V, dtype, 40)
    rows[1, V - 1] = float("nan")
    rows[2, V // 2] = float("inf")
    rows[3] = float("-inf")
    rows[4, 0] = -torch.tensor(float("nan"))
    per_row = torch.full((R,), 0.1, device="cuda")
    per_row[5] = 1.5
    out, n, st = gpu_lib.resispec_filter_logits(rows, min_p=per_row)
    torch.cuda.synchronize()
    bad, param = gpu_lib.RS_SEQ_UNDERFLOW, gpu_lib.RS_SEQ_BAD_PARAM
    assert st.tolist() == [0, bad, bad, bad, bad, param, 0]
    assert (out[1:6] == float("-inf")).all() and (n[1:6] == -1).all()
    want, count = expected_filter(rows[[0, 6]], [dict(min_p=float(np.float32(0.1)))] * 2)
    assert same_bits(out[[0, 6]], want) and n[[0, 6]].tolist() == count


def test_filter_signed_zeros(gpu_lib):
    """-0 and +0 are equal in the order, and are written as they were."""
    for dtype in (F32, BF16):
        rows = torch.full((1, 600), -5.0, dtype=dtype, device="cuda")
        rows[0, 100:110] = 0.0
        rows[0, 105:300] = -0.0
        out, n, _ = gpu_lib.resispec_filter_logits(rows, top_k=8)
        torch.cuda.synchronize()
        want = torch.full_like(rows, float("-inf"))
        want[0, 100:108] = rows[0, 100:108]
        assert same_bits(out, want) and int(n[0]) == 8


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 7, 64, 1000, 2049, 32001, 151936])
def test_token_logprobs(gpu_lib, V, dtype):
    g = np.random.default_rng(V)
    for kind, pad, k, T in (("zipf", 0, 1, 1.0), ("few", 5, 6, 0.7), ("lowest", 3, 64, 1.3), ("large", 0, 3, 2.0),
                            ("masked", 1, 5, 0.3), ("peaked", 0, 20, 0.6)):
        rows = make_rows(4, V, dtype, V, kind, pad)
        tokens = g.integers(-1, V, (4, k)).astype(np.int32)
        tokens[0, 0], tokens[1, 0], tokens[2, 0] = V - 1, 0, -1
        lp, rank, st = gpu_lib.resispec_token_logprobs(rows, torch.as_tensor(tokens, device="cuda"), temperature=T)
        torch.cuda.synchronize()
        assert (st == 0).all()
        l = to64(rows)
        for r in range(4):
            for i in range(k):
                got = (float(lp[r, i]), int(rank[r, i]))
                if tokens[r, i] < 0:
                    assert got == (0.0, 0)
                    continue
                p, n = logprob(l[r], T, tokens[r, i])
                assert got[1] == n
                if p == -np.inf or p < -3.4e38:
                    assert got[0] == -np.inf
                else:
                    assert abs(got[0] - p) <= abs(p) * 2.0 ** -24 + 4.8e-6, (got[0], p, kind)


def test_token_logprobs_bad_tokens(gpu_lib):
    rows = make_rows(4, 100, F32, 1)
    tokens = torch.tensor([[0, 99], [5, 100], [-2, 3], [-1, -1]], dtype=torch.int32, device="cuda")
    lp, rank, st = gpu_lib.resispec_token_logprobs(rows, tokens)
    torch.cuda.synchronize()
    bad = gpu_lib.RS_SEQ_BAD_TOKEN
    assert st.tolist() == [0, bad, bad, 0]
    assert torch.isnan(lp[1:3]).all() and (rank[1:3] == -1).all() and (rank[3] == 0).all() and (lp[3] == 0).all()


def test_offsets_past_32_bits(gpu_lib):
    """Rows whose elements lie past 2^32 bytes and 2^31 elements of the first."""
    V, step = 1001, (1 << 26) + 8
    R = 40
    flat = torch.zeros((R - 1) * step + V + 8, dtype=BF16, device="cuda")
    rows = flat.as_strided((R, V), (step, 1))
    rows.copy_(make_rows(R, V, BF16, 21))
    each, t = row_settings(R)
    check_sample(gpu_lib, rows, uniforms(R, 2), each, **t)
    want, count = expected_filter(rows.contiguous(), each)
    tokens = torch.randint(0, V, (R, 2), dtype=torch.int32, device="cuda")
    a = gpu_lib.resispec_token_logprobs(rows, tokens)
    b = gpu_lib.resispec_token_logprobs(rows.contiguous(), tokens)
    gpu_lib.resispec_filter_logits(rows, out=rows, **t)
    torch.cuda.synchronize()
    assert same_bits(rows.contiguous(), want)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_same_results_on_every_call_stream_and_batch(gpu_lib):
    """A row's outputs do not depend on the call it is in: alone, among others, on another
    stream, with two calls under way at once."""
    R, V = 300, 40961
    rows = make_rows(R, V, BF16, 31)
    each, t = row_settings(R)
    u = uniforms(R, 4)
    tokens = torch.randint(-1, V, (R, 4), dtype=torch.int32, device="cuda")
    first = (*gpu_lib.resispec_sample(rows, u, **t), *gpu_lib.resispec_filter_logits(rows, **t),
             *gpu_lib.resispec_token_logprobs(rows, tokens, temperature=t["temperature"]))
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        a = (*gpu_lib.resispec_sample(rows, u, **t, stream=s1), *gpu_lib.resispec_filter_logits(rows, **t, stream=s2),
             *gpu_lib.resispec_token_logprobs(rows, tokens, temperature=t["temperature"], stream=s1))
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(a, first))
    for lo, hi in ((0, 1), (5, 6), (17, 40), (12, 13), (0, 150)):
        part = {k: v[lo:hi] for k, v in t.items()}
        a = (*gpu_lib.resispec_sample(rows[lo:hi], u[lo:hi], **part),
             *gpu_lib.resispec_filter_logits(rows[lo:hi], **part),
             *gpu_lib.resispec_token_logprobs(rows[lo:hi], tokens[lo:hi], temperature=part["temperature"]))
        torch.cuda.synchronize()
        assert all(torch.equal(x, y[lo:hi]) for x, y in zip(a, first))


@pytest.mark.parametrize("R", [2, 300])
def test_captured_and_replayed(gpu_lib, R):
    """All three operators in one graph, replayed with new inputs and the program's own work in
    between; each replay equals the eager calls."""
    V = 20011
    rows = make_rows(R, V, F32, 41)
    each, t = row_settings(R)
    u = uniforms(R, 2)

    def calls(x, v):
        y, n, st = gpu_lib.resispec_filter_logits(x, **t)
        s = gpu_lib.resispec_sample(x, v, **t)
        return (y, n, st, *s, *gpu_lib.resispec_token_logprobs(y, s[0], temperature=t["temperature"]))

    calls(rows, u)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = calls(rows, u)
    for seed in (42, 43, 44, 45):
        rows.copy_(make_rows(R, V, F32, seed))
        u.copy_(uniforms(R, 2, seed))
        graph.replay()
        torch.cuda.synchronize()
        want = calls(rows, u)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(held, want))
        torch.randn(1 << 20, device="cuda").sum().item()


@pytest.mark.parametrize("dtype, V", [(F32, 20011), (F32, 60001), (BF16, 128257)], ids=str)
def test_min_p_alone_captured_and_on_other_streams(gpu_lib, dtype, V):
    """Rows that registers hold, filtered in place in a replayed graph and by two streams at
    once; and the cut of a batch is that of its rows alone."""
    rows = make_rows(300, V, dtype, 51)
    work = rows.clone()
    want, count = expected_filter(rows[:3], [dict(min_p=0.05, T=0.8)] * 3)
    whole, n0, _ = gpu_lib.resispec_filter_logits(rows, min_p=0.05, temperature=0.8)
    torch.cuda.synchronize()
    assert same_bits(whole[:3], want) and n0[:3].tolist() == count
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, n, st = gpu_lib.resispec_filter_logits(work, min_p=0.05, temperature=0.8, out=work)
    for _ in range(3):
        work.copy_(rows)
        graph.replay()
        torch.cuda.synchronize()
        assert same_bits(work, whole) and torch.equal(n, n0) and (st == 0).all()
        torch.randn(1 << 20, device="cuda").sum().item()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    parts = [gpu_lib.resispec_filter_logits(rows[i:i + 100], min_p=0.05, temperature=0.8, stream=streams[i // 100])
             for i in (0, 100)]
    torch.cuda.synchronize()
    for i, (out, m, _) in enumerate(parts):
        assert same_bits(out, whole[100 * i:100 * i + 100]) and torch.equal(m, n0[100 * i:100 * i + 100])


def test_empty_batches(gpu_lib):
    x = torch.empty((0, 100), device="cuda")
    tok, lp, n, st = gpu_lib.resispec_sample(x, torch.empty((0, 2), device="cuda"))
    assert tok.shape == (0, 2) and st.shape == (0,)
    out, n, st = gpu_lib.resispec_filter_logits(x)
    assert out.shape == (0, 100)
    lp, rank, st = gpu_lib.resispec_token_logprobs(x, torch.empty((0, 3), dtype=torch.int32, device="cuda"))
    assert lp.shape == (0, 3)


def test_extreme_temperatures(gpu_lib):
    """The smallest and largest temperatures, masked elements among the row's."""
    for kind in ("zipf", "masked", "lowest"):
        rows = make_rows(2, 9001, F32, 3, kind)
        for T in (1e-45, 1e-38, 1e-6, 1e4, 1e30, 3.0e38):
            for s in (dict(), dict(top_k=20), dict(top_p=0.7), dict(min_p=0.5)):
                check_sample(gpu_lib, rows, uniforms(2, 2), temperature=T, **s)
            tokens = torch.tensor([[5, 17], [9000, 0]], dtype=torch.int32, device="cuda")
            lp, rank, st = gpu_lib.resispec_token_logprobs(rows, tokens, temperature=T)
            torch.cuda.synchronize()
            assert (st == 0).all()
            for r in range(2):
                for i in range(2):
                    p, n = logprob(to64(rows)[r], T, int(tokens[r, i]))
                    assert int(rank[r, i]) == n
                    got = float(lp[r, i])
                    assert got == -np.inf if p < -3.4e38 else abs(got - p) <= abs(p) * 2.0 ** -24 + 4.8e-6


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("V", [700, 9001, 33000])
def test_a_maximum_far_above_the_row(gpu_lib, V, dtype):
    """One logit whose mass, against any other's, is past the range of 64 bits; at the places
    where a sample of the row may miss it."""
    x = np.random.default_rng([3, V]).standard_normal((6, V))
    for r, j in enumerate((0, V // 16 + 100, V // 3, V // 2 - 1, 15 * V // 16, V - 1)):
        x[r, j] = 900.0
    rows = torch.as_tensor(x, device="cuda").to(dtype)
    for i, s in enumerate((dict(), dict(top_k=1), dict(top_k=40), dict(top_k=V // 2), dict(top_k=V), dict(top_p=0.9),
                           dict(min_p=1e-6), dict(top_k=V // 2, min_p=0.5), dict(top_k=60, top_p=0.5))):
        for T in (1.0, 0.5, 1e-3):
            check_sample(gpu_lib, rows, uniforms(6, 2, i), temperature=T, **s)


def test_many_short_rows(gpu_lib):
    """A row of a few elements each, more rows than a grid has compute units by far; and the
    first row count that is refused."""
    R, V = 70000, 5
    rows = make_rows(R, V, F32, 9)
    tok, lp, n, st = gpu_lib.resispec_sample(rows, uniforms(R, 1), top_k=1)
    out, n2, _ = gpu_lib.resispec_filter_logits(rows, top_k=2)
    torch.cuda.synchronize()
    assert torch.equal(tok[:, 0].long(), rows.argmax(1)) and (lp == 0).all() and (n == 1).all() and (n2 == 2).all()
    assert (torch.isfinite(out).sum(1) == 2).all()
    x = torch.zeros((1 << 23, 1), dtype=BF16, device="cuda")
    with pytest.raises(gpu_lib.ResiSpecError):
        gpu_lib.resispec_filter_logits(x)


def test_binding_refusals(gpu_lib):
    x = make_rows(4, 64, F32, 1)
    u = uniforms(4, 1)
    tok = torch.zeros((4, 1), dtype=torch.int32, device="cuda")
    bad = [lambda: gpu_lib.resispec_sample(x.double(), u), lambda: gpu_lib.resispec_sample(x.half(), u),
           lambda: gpu_lib.resispec_sample(x[0], u[0]), lambda: gpu_lib.resispec_sample(x, u[:3]),
           lambda: gpu_lib.resispec_sample(x, u[:, 0]), lambda: gpu_lib.resispec_sample(x.t(), u),
           lambda: gpu_lib.resispec_sample(x, u.double()), lambda: gpu_lib.resispec_sample(x, u.cpu()),
           lambda: gpu_lib.resispec_sample(x, u.expand(4, 65)),
           lambda: gpu_lib.resispec_sample(x, u[:, :0]), lambda: gpu_lib.resispec_sample(x[:1].expand(4, 64), u),
           lambda: gpu_lib.resispec_sample(x, u, temperature=0.0), lambda: gpu_lib.resispec_sample(x, u, top_p=1.5),
           lambda: gpu_lib.resispec_sample(x, u, top_k=-1), lambda: gpu_lib.resispec_sample(x, u, min_p=-1.0),
           lambda: gpu_lib.resispec_sample(x, u, top_k=torch.ones(4, device="cuda")),
           lambda: gpu_lib.resispec_sample(x, u, top_p=torch.ones(3, device="cuda")),
           lambda: gpu_lib.resispec_sample(x, u, top_p=torch.ones(4)),
           lambda: gpu_lib.resispec_sample(x, u, out_token=tok[:3]),
           lambda: gpu_lib.resispec_sample(x, u, out_token=tok.float()),
           lambda: gpu_lib.resispec_filter_logits(x, out=x[:3]),
           lambda: gpu_lib.resispec_filter_logits(x, out=x.bfloat16()),
           lambda: gpu_lib.resispec_filter_logits(x[:3], out=x[1:]),
           lambda: gpu_lib.resispec_filter_logits(x, out=x.cpu()),
           lambda: gpu_lib.resispec_token_logprobs(x, tok.long()),
           lambda: gpu_lib.resispec_token_logprobs(x, tok[:2]),
           lambda: gpu_lib.resispec_token_logprobs(x, tok, temperature=-1.0),
           lambda: gpu_lib.resispec_token_logprobs(x.view(2, 2, 64), tok)]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, TypeError, gpu_lib.ResiSpecError)):
            call()
            print("refusal", i, "was not made")
