"""Beam search's choice at temperatures near the ends of their range, where a difference of two
logits, or a logit over the temperature, passes 32 bits.  The tolerance is test_gpu_beam's: an
exponent is the rounded difference, times the rounded factor, rounded, at every temperature."""
import numpy as np
import pytest
import torch

from test_gpu_beam import check, scores_for

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.bfloat16]
IDS = ["f32", "bf16"]


def rows(values, B, W, V, dtype, seed):
    """[B, W, V] rows of the given values, in any order, bits as they are."""
    g = np.random.default_rng([seed, V])
    x = torch.as_tensor(np.asarray(values, dtype=np.float32)[g.integers(0, len(values), (B, W, V))])
    return x.to(dtype).to("cuda")


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("T", [1e31, 1e37, 1e38, 3.4e38])
def test_highest(gpu_lib, T, dtype):
    """Logits from the type's lowest value to its highest."""
    top = torch.finfo(dtype).max
    values = np.linspace(-1.0, 1.0, 41) * top
    for V, k in ((7, 6), (600, 8), (9001, 16)):
        check(gpu_lib, rows(values, 2, 3, V, dtype, 1), scores_for(2, 3, spread=1.0), k, T=T)
    # most of a row at the lowest value, few others
    x = rows(values, 2, 3, 5000, dtype, 2)
    x[:, :, 5:] = -top
    check(gpu_lib, x, scores_for(2, 3, spread=1.0), 12, T=T)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("steps", [1, 3, 1000, 1 << 20])
def test_lowest(gpu_lib, steps, dtype):
    """A temperature of so many of the smallest steps of the type, logits some of those apart, near
    zero and beside a logit that is far from it."""
    unit = 2.0 ** -149 if dtype == torch.float32 else 2.0 ** -133
    T = steps * unit
    values = -np.arange(41.0) * max(1, steps // 8) * unit
    for V, k in ((7, 6), (600, 8), (9001, 16)):
        check(gpu_lib, rows(values, 2, 3, V, dtype, 3), scores_for(2, 3, spread=1.0), k, T=T)
    x = rows(values, 2, 3, 5000, dtype, 4)
    x[0, 0, 17] = 1.0
    x[0, 1, 18] = 3e38
    x[1, :, 4097:] = -1.0
    x[1, 2, 9] = float("-inf")
    # scores this low are past 32 bits: only what is among the first is asked for
    check(gpu_lib, x, torch.full((2, 3), -2.0, device="cuda"), 2, T=T)
