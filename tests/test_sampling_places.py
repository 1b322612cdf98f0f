"""Where resispec_filter_logits may write: rows apart from the logits, the logits themselves,
or rows that lie between theirs."""
import numpy as np
import pytest
import torch

from paper_2608_24411_amd import native


def shared(a, a_step, b, b_step, R, V):
    """By element: whether the rows at a and b have one in common."""
    at = lambda s, step: {s + r * step + j for r in range(R) for j in range(V)}  # noqa: E731
    return bool(at(a, a_step) & at(b, b_step))


@pytest.mark.parametrize("size", [2, 4])
def test_rows_that_share_memory(size):
    g = np.random.default_rng(7)
    refused = 0
    for _ in range(4000):
        R, V = int(g.integers(0, 6)), int(g.integers(1, 9))
        a_step, b_step = (V + int(x) for x in g.integers(0, 12, 2))
        if g.random() < 0.6:
            b_step = a_step
        a, b = (int(x) for x in g.integers(0, 60, 2))
        says = native._overlap(a * size, a_step, b * size, b_step, R, V, size)
        if shared(a, a_step, b, b_step, R, V):
            assert says
        elif a_step == b_step and says:
            # refused though apart: only rows past the other's last would meet
            refused += 1
            assert shared(a, a_step, b, b_step, 2 * R + 60, V)
    assert native._overlap(0, 8, 4, 8, 3, 4, 4) and not native._overlap(0, 8, 16, 8, 3, 4, 4)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("V", [64, 1001, 40003])
def test_output_rows_between_the_logits(gpu_lib, V, dtype):
    """Both halves of one tensor's rows, either way round, and a tree's rows."""
    from test_gpu_sampling import expected_filter, make_rows, same_bits
    R = 6
    for first in (0, 1):
        both = torch.full((R, 2, V), 3.0, dtype=dtype, device="cuda")
        rows, out = both[:, first], both[:, 1 - first]
        rows.copy_(make_rows(R, V, dtype, 5))
        before = rows.clone()
        want, count = expected_filter(before, [dict(top_p=0.9, temperature=0.8)] * R)
        got, n, st = gpu_lib.resispec_filter_logits(rows, top_p=0.9, temperature=0.8, out=out)
        torch.cuda.synchronize()
        assert got is out and same_bits(out, want) and n.tolist() == count and (st == 0).all()
        assert same_bits(rows, before)
        with pytest.raises(ValueError):
            gpu_lib.resispec_filter_logits(rows[:, 1:], out=rows[:, :-1])
