"""Beams whose order a 32-bit sum gets wrong: the choice has to sum their rows again in 64 bits.

Pairs of rows.  The first has elements d below its maximum, so many that they carry most of its
sum; all have the same exponent x = -d log2(e) / T, so that the rounding of the factor and of the
product moves its 32-bit sum by up to |x| ln 2 * 2 * 2^-24 of its value, always the same way.  The
second row has elements equal to its maximum and nothing else: its sum is a whole number in 32
bits too.  The second beam's score puts its candidates a third of that error from the first
beam's, on the side where 32 bits have them the other way round; the scores are near zero, where
fp32 has the numbers for it."""
import math

import numpy as np
import pytest
import torch

from beam_util import select
from sampling_util import to64

DTYPES = [torch.float32, torch.bfloat16]
IDS = ["f32", "bf16"]
UNIT = 4096                              # elements that are summed against one maximum


def mass(T, d):
    """(exponent in 32 bits, how much too large the mass is by it, of its value)."""
    x = np.float32(-d) * np.float32(1.4426950408889634 / float(np.float32(T)))
    return float(x), float(x) * math.log(2.0) + d / float(np.float32(T))


def pair(sign, V, tops):
    """(T, rows [2, V], scores [2], 64-bit scores of the two beams' best, error of the first one's
    32-bit score by its exponents, what that may be off): `tops` elements at the maximum in each
    unit of the first row."""
    best = None
    for T in np.linspace(0.6, 1.6, 2001).astype(np.float32):
        for d in (4.0, 5.0, 6.0, 7.0, 8.0):
            x, off = mass(T, d)
            # a mantissa near 2: a step of the mass is little of its value
            if -10.0 < x < -7.5 and 2.0 ** (x - math.floor(x)) > 1.7 and (best is None or sign * off > sign * best[2]):
                best = (float(T), d, off)
    T, d, off = best
    a = np.full(V, -d)
    for u in range(0, V, UNIT):
        a[u + 5:u + 5 + tops] = 0.0
    n = int((a == 0.0).sum())
    bulk = (V - n) * math.exp(-d / float(np.float32(T)))
    b = np.full(V, -np.inf)
    m = round(n + bulk)
    b[np.linspace(0, V - 1, m).astype(int)] = 0.0
    first = -math.log(n + bulk)
    error = -math.log1p(off * bulk / (n + bulk))        # of the first beam's score
    second = np.float32(first + math.log(m) + error / 3.0)
    # the exponential's own step, of a mantissa above 1.7; three roundings where eight elements with a
    # maximum among them are added (without one they are equal, and their sums exact)
    rest = (2.0 ** -23 / 1.7 * bulk + 3 * 2.0 ** -24 * n * (1.0 + 7 * 2.0 ** -7)) / (n + bulk)
    return T, np.stack((a, b)), np.array([0.0, second], dtype=np.float32), (first, float(second) - math.log(m)), error, rest


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("V,tops", [(UNIT, 1), (3 * UNIT + 5, 1), (1 << 20, 4)])
def test_32_bits_have_them_the_wrong_way_round(V, tops, sign):
    """The inputs do what they are for, whatever the roundings that are not counted in the error."""
    T, rows, scores, (first, second), error, rest = pair(sign, V, tops)
    assert (first > second) == (error < 0.0)
    nearest = abs(error) - rest                         # the least that it is off in 32 bits
    assert 1e-8 < abs(first - second) < 0.75 * nearest and abs(error) + rest < 3.0e-6
    wrong = first + math.copysign(nearest, error)
    assert (wrong > second) != (first > second)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("V,tops", [(UNIT, 1), (3 * UNIT + 5, 1), (1 << 20, 4)])
def test_order_is_that_of_64_bits(gpu_lib, V, tops, sign, dtype):
    """The last size has more equal elements than are listed."""
    T, rows, scores, _, _, _ = pair(sign, V, tops)
    for W, at in ((2, (0, 1)), (2, (1, 0)), (40, (3, 37)), (40, (39, 0)))[:4 if V < 1 << 16 else 2]:
        logits = torch.full((1, W, V), -1.0, dtype=dtype)
        logits[0, list(at)] = torch.as_tensor(rows).to(dtype)
        s = np.full((1, W), -50.0, dtype=np.float32)
        s[0, list(at)] = scores
        logits = logits.cuda()
        for k in (1, 4):
            print("close", V, W, at, k, logits.dtype, flush=True)
            parent, token, score, st = gpu_lib.resispec_beam_select(logits, torch.as_tensor(s, device="cuda"), k=k, temperature=T)
            torch.cuda.synchronize()
            want = select(to64(logits[0]), s[0].astype(np.float64), k, T)
            assert st.tolist() == [0] and parent[0].tolist() == want[0] and token[0].tolist() == want[1]
            # both beams were summed again, so their scores are rounded once; a 32-bit sum's is
            # off by more than that
            got = score[0].double().cpu().numpy()
            assert (np.abs(got - want[2]) <= np.abs(want[2]) * 2.0 ** -24 + 1e-12).all()
