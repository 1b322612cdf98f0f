"""Kept elements whose mass is far below the last bit of the row's maximum: a draw of u = 0 is
the first kept element with any mass, whichever way the cut was found.  Against the plain
definition (sampling_util), whose running sums begin with those masses and hold them; draws
are compared where u times the total lies far from every border (0, or less than a tenth or
more than ten times any running sum before the row's maximum).

The range of the masses.  64-bit numbers have 2^-1022 as their smallest normal one; numpy's
exponential goes on below it, with fewer and fewer bits, to 2^-1075, the kernels' is zero from
2^-1023 on (the exponent field of 2^x is x + 1023, and there is none below 0).  rs_filter says
so: such masses count as none.  An element has one where (l - m) / T < -1023 ln 2 = -709.09;
among the rows below that is 12.33 and less at T = 0.008, and no element within 1e-6 of it."""
import numpy as np
import pytest
import torch

from sampling_util import draw, kept, to64

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def rows_with_a_peak(V, dtype, seed):
    """Three rows: noise around 8, a few elements around 14 early on, the maximum of 18 late."""
    g = np.random.default_rng([seed, V])
    x = 8.0 + g.standard_normal((3, V))
    x[0, 5] = 14.0
    x[1, V // 5], x[1, V // 4] = 13.5, 14.5
    x[2, [7, 700, V // 2]] = 12.75, 14.0, 14.5
    x[:, 2 * V // 3] = 18.0
    return torch.as_tensor(x, device="cuda").to(dtype)


def check_draws(native, rows, u, s):
    """One call against the definition, masses below 2^-1023 of the maximum counting as none."""
    tok, lp, n, st = native.resispec_sample(rows, u, **s)
    torch.cuda.synchronize()
    l, uu, T = to64(rows), u.cpu().numpy(), s["temperature"]
    for r in range(rows.shape[0]):
        mask = kept(l[r], **{"T" if k == "temperature" else k: v for k, v in s.items()})
        assert int(st[r]) == native.RS_SEQ_OK and int(n[r]) == mask.sum()
        x = (l[r] - l[r].max()) / float(np.float32(T)) / np.log(2.0)
        assert (np.abs(x + 1023.0) > 1e-6).all()
        for i in range(u.shape[1]):
            j, p = draw(l[r], T, mask & (x > -1023.0), uu[r, i])
            assert int(tok[r, i]) == j, (r, int(tok[r, i]), j, uu[r, i])
            # half a step of the result, and the 64-bit sums
            assert abs(float(lp[r, i]) - p) <= abs(p) * 2.0 ** -24 + 1e-12


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("V", [1200, 5003, 20000, 32768, 70001])
@pytest.mark.parametrize("T", [0.1, 0.05, 0.02, 0.008])
def test_draws_among_tiny_masses(gpu_lib, T, V, dtype):
    rows = rows_with_a_peak(V, dtype, 71)
    l = to64(rows)
    for s in (dict(top_k=2), dict(top_k=50), dict(top_k=300), dict(top_k=1100), dict(min_p=1e-18), dict(min_p=1e-38),
              dict(top_k=50, min_p=1e-44), dict()):
        s = dict(s, temperature=T)
        us = [0.0, 1e-45, 1e-38, 1e-30, 1e-20, 1e-18, 2.0 ** -24, 0.5, 1.0 - 2.0 ** -24]
        u = np.zeros((3, len(us)), dtype=np.float32)
        for r in range(3):
            mask = kept(l[r], **{"T" if k == "temperature" else k: v for k, v in s.items()})
            w = np.exp((l[r] - 18.0) / float(np.float32(T))).astype(np.longdouble) * mask
            before = w[:2 * V // 3].cumsum()
            before = before[before > 0.0]
            for i, x in enumerate(np.float32(us)):
                # a border within a factor of ten: the sums' rounding may decide
                near = ((before > x / 10.0) & (before < x * 10.0)).any()
                u[r, i] = 0.0 if near else x
        check_draws(gpu_lib, rows, torch.as_tensor(u, device="cuda"), s)


def test_the_first_kept_token_whatever_the_search(gpu_lib):
    """The worked case: masses 4e-18 and 1, the smaller one first.  Rows short and long, and
    top-k small and large, take different searches; u = 0 is token 5 in all."""
    for V in (5000, 16384, 32768, 70001):
        g = np.random.default_rng([72, V])
        x = g.standard_normal((1, V))
        x[0, 5], x[0, V - 3000] = 6.0, 10.0
        for dtype in (F32, BF16):
            rows = torch.as_tensor(x, device="cuda").to(dtype)
            u = torch.zeros((1, 2), device="cuda")
            u[0, 1] = 2.0 ** -24
            tok, lp, n, st = gpu_lib.resispec_sample(rows, u, temperature=0.1, top_k=2)
            torch.cuda.synchronize()
            assert tok.tolist() == [[5, V - 3000]] and int(n[0]) == 2 and int(st[0]) == 0
            mask = kept(to64(rows)[0], T=0.1, top_k=2)
            assert draw(to64(rows)[0], 0.1, mask, 0.0)[0] == 5
