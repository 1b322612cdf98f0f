"""Log-probabilities of tokens where the row's sample misses its maximum by far.

Bounds.  The exponents (l - r) c, in bits, are taken against r, the highest of the row's sample
and of the given tokens, and are below 128 (a sum past that is redone against the maximum).
Three roundings of 2^-24 each (the difference, its product with the high part of c, the sum
with the low part's) make 3 * 128 * 2^-24 * ln 2 = 1.59e-5 of a term; the exponential's own
2^-23 and three 32-bit additions 3e-7: 1.62e-5 of the sum at most, as much in its logarithm.

Where a given token is the maximum, exponents are -e <= 0 and the sum is at least 1, to which
V terms of 2^-e add at most V 2^-e.  With V < 2^18 the error 3 e 2^-24 ln 2 * V 2^-e / (1 + V
2^-e) is below 1.24e-7 * 18 for every e (e = 18: half of it; above 18 the weight halves with
each step): 2.2e-6, and 3e-7.  Half a step of the result is added to each.

A log-probability is never above 0: its token's logit is at most r (or the maximum), whose own
term is exactly 1."""
import numpy as np
import pytest
import torch

from sampling_util import logprob, to64

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def check(native, rows, tokens, T):
    lp, rank, st = native.resispec_token_logprobs(rows, torch.as_tensor(tokens, device="cuda"), temperature=T)
    torch.cuda.synchronize()
    assert (st == 0).all()
    l = to64(rows)
    for r in range(rows.shape[0]):
        top = l[r].max()
        given = any(x >= 0 and l[r, x] == top for x in tokens[r])
        bound = 2.2e-6 + 3e-7 if given else 1.62e-5
        for i, x in enumerate(tokens[r]):
            got = float(lp[r, i])
            if x < 0:
                assert got == 0.0 and int(rank[r, i]) == 0
                continue
            p, n = logprob(l[r], T, x)
            assert int(rank[r, i]) == n
            if p == -np.inf:
                assert got == -np.inf
                continue
            assert got <= 0.0, (got, p)
            assert abs(got - p) <= abs(p) * 2.0 ** -24 + bound, (got, p, given)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("V", [9001, 40003, 151936])
@pytest.mark.parametrize("T, heights", [(1.0, (5.3, 21.7, 50.3, 67.1, 80.9, 85.2, 300.0)),
                                        (0.25, (1.7, 5.9, 12.3, 15.1, 18.7, 21.1, 60.0))])
def test_a_maximum_above_the_sample(gpu_lib, T, heights, V, dtype):
    g = np.random.default_rng([91, V])
    places = (V // 16 + 700, V // 3, V // 2 - 1, 15 * V // 16, V - 1)
    x = np.concatenate([g.standard_normal((len(places), V)) for _ in heights])
    at = [j for _ in heights for j in places]
    for r, j in enumerate(at):
        x[r, j] = x[r].max() + heights[r // len(places)]
    rows = torch.as_tensor(x, device="cuda").to(dtype)
    R = len(at)
    rest = g.integers(0, V, (R, 3)).astype(np.int32)
    top = np.asarray(at, dtype=np.int32)[:, None]
    for tokens in (top, rest, np.concatenate((rest[:, :1], top, np.full((R, 1), -1, np.int32)), 1),
                   np.full((R, 1), -1, np.int32)):
        check(gpu_lib, rows, tokens, T)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_many_elements_above_the_sample(gpu_lib, dtype):
    """A thousand of them, some among the tokens; masked elements and masked samples beside."""
    V = 70001
    g = np.random.default_rng(92)
    x = g.standard_normal((6, V))
    for r, lo in enumerate((10.0, 40.0, 55.0, 70.0, 80.0, 83.0)):
        x[r, 30000:31000] = lo + 2.0 * g.random(1000)
    x[3, g.random(V) < 0.3] = -np.inf
    x[4, :30000] = -np.inf
    x[5, :30000] = -np.inf
    x[5, 31000:] = -np.inf
    rows = torch.as_tensor(x, device="cuda").to(dtype)
    for tokens in ([30000, 30500, 30999], [40000, 60001, -1], [5, 69999, 30001]):
        t = np.tile(np.asarray(tokens, dtype=np.int32), (6, 1))
        t[5] = [30000, 30001, 30002]
        if -np.inf in x[3][t[3][t[3] >= 0]] or -np.inf in x[4][t[4][t[4] >= 0]]:
            t[3] = t[4] = [30003, 30004, -1]
        check(gpu_lib, rows, t, 1.0)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("T", [1.0, 0.25])
def test_no_drawn_log_probability_is_above_zero(gpu_lib, T, dtype):
    """Nearly certain tokens: 64-bit sums against a reference other than the maximum."""
    R, V = 64, 40003
    g = np.random.default_rng(93)
    x = g.standard_normal((R, V))
    x[np.arange(R), g.integers(0, V, R)] = np.linspace(30.0, 90.0, R)
    rows = torch.as_tensor(x, device="cuda").to(dtype)
    u = torch.full((R, 2), 0.5, device="cuda")
    for s in (dict(), dict(top_k=40), dict(top_p=0.9), dict(min_p=0.1), dict(top_k=20000)):
        tok, lp, n, st = gpu_lib.resispec_sample(rows, u, temperature=T, **s)
        torch.cuda.synchronize()
        assert (st == 0).all() and (lp <= 0.0).all() and (lp > -1e-6).all()
        assert torch.equal(tok[:, 0].long(), rows.argmax(1))
