"""Cuts of rows masked with the type's lowest value, under top-k and min-p together: the
counts of a bf16 row's values say what min-p keeps where top-k reaches into the masked
elements, below every bin of the counts.  Everything is compared exactly with the plain 64-bit
definition (sampling_util), log-probabilities as in test_gpu_sampling."""
import numpy as np
import pytest
import torch

from sampling_util import make_rows
from test_gpu_sampling import check_sample, expected_filter, same_bits, uniforms

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def lowest_rows(R, V, unmasked, dtype, seed):
    """R rows of V logits, all but `unmasked` of each at the type's lowest value."""
    g = np.random.default_rng([seed, R, V, unmasked])
    x = 3.0 * g.standard_normal((R, V))
    for r in range(R):
        x[r, g.permutation(V)[unmasked:]] = torch.finfo(dtype).min
    return torch.as_tensor(x, device="cuda").to(dtype)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("V, unmasked, top_ks", [(1000, 100, (50, 101, 500, 999, 1000, 5000)),
                                                (5003, 2502, (7, 2503, 3000, 5002, 5003)),
                                                (70001, 35000, (7, 4000, 35001, 60000, 70001)),
                                                (151936, 1500, (1000, 1501, 2000, 100000))])
def test_top_k_past_the_unmasked_elements_with_min_p(gpu_lib, V, unmasked, top_ks, dtype):
    rows = lowest_rows(3, V, unmasked, dtype, 61)
    for i, top_k in enumerate(top_ks):
        for kw in (dict(min_p=0.05), dict(min_p=0.05, temperature=0.6), dict(min_p=1e-45), dict(min_p=1.0), dict(),
                   dict(min_p=0.002, top_p=0.98)):
            s = dict(top_k=top_k, **kw)
            check_sample(gpu_lib, rows, uniforms(3, 4, i), **s)
            want, count = expected_filter(rows, [s] * 3)
            out, n, st = gpu_lib.resispec_filter_logits(rows, **s)
            torch.cuda.synchronize()
            assert same_bits(out, want) and n.tolist() == count and (st == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("V", [5003, 70001])
@pytest.mark.parametrize("kind", ["zipf", "flat", "peaked", "equal", "few", "masked", "lowest", "all-lowest", "large"])
def test_top_k_and_min_p_on_every_kind_of_row(gpu_lib, kind, V, dtype):
    rows = make_rows(2, V, dtype, 62, kind)
    for i, s in enumerate((dict(top_k=7, min_p=0.05), dict(top_k=4000, min_p=0.05), dict(top_k=60000, min_p=0.05),
                           dict(top_k=V, min_p=0.3, temperature=0.5), dict(top_k=4000, min_p=1e-45))):
        check_sample(gpu_lib, rows, uniforms(2, 3, i), **s)
        want, count = expected_filter(rows, [s] * 2)
        out, n, st = gpu_lib.resispec_filter_logits(rows, **s)
        torch.cuda.synchronize()
        assert same_bits(out, want) and n.tolist() == count and (st == 0).all()


def test_top_k_and_min_p_of_each_row(gpu_lib):
    """The same from arrays of settings, a faulted row among them, on many rows at once."""
    R, V = 300, 5003
    rows = lowest_rows(R, V, 2502, BF16, 63)
    rows[7, 5] = float("nan")
    each = [dict(top_k=(7, 2503, 3000, 5002, 5003, 0)[r % 6], min_p=(0.05, 0.0, 0.3)[r % 3]) for r in range(R)]
    t = dict(top_k=torch.tensor([s["top_k"] for s in each], dtype=torch.int32, device="cuda"),
             min_p=torch.tensor([s["min_p"] for s in each], device="cuda"))
    check_sample(gpu_lib, rows, uniforms(R, 3), each, **t)
    out, n, st = gpu_lib.resispec_filter_logits(rows, **t)
    torch.cuda.synchronize()
    good = [r for r in range(R) if r != 7]
    want, count = expected_filter(rows[good], [each[r] for r in good])
    assert same_bits(out[good], want) and n[good].tolist() == count
    assert int(n[7]) == -1 and (out[7] == float("-inf")).all()
