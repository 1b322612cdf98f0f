"""Cuts on a border between two bins of the search over key ranges: rows of two clusters, the
higher of which holds the share of the mass that top_p asks for, to within 1e-17.  Where the
search begins comes from 32-bit sums whose order is not fixed; what it finds must not."""
import numpy as np
import pytest
import torch

from sampling_util import kept, to64
from test_gpu_sampling import check_sample, uniforms

pytestmark = pytest.mark.gpu


def clusters(g, V, high, top_k, spread):
    """A row with `high` elements around 0 and the others around -3; top_p (fp32), the high
    ones' share of the mass of the first top_k."""
    x = (-3.0 + 0.1 * g.standard_normal(V)).astype(np.float32).astype(np.float64)
    at = g.permutation(V)[:high]
    x[at] = (spread * g.standard_normal(high)).astype(np.float32)
    knobs = at[:2]
    x[knobs] = 0.0
    top = x.max()

    def sums():
        w = np.exp((np.sort(x)[::-1][:top_k] - top).astype(np.longdouble)).cumsum()
        return w[high - 1], w[-1]
    part, whole = sums()
    top_p = np.longdouble(np.float32(part / whole))
    for j in knobs:
        need = (top_p * whole - part) / (1.0 - top_p)
        x[j] = float(np.float32(top + np.log(np.exp(np.longdouble(x[j] - top)) + need)))
        part, whole = sums()
    assert abs(part - top_p * whole) < 1e-17 * whole and x.max() == top
    return x, float(top_p)


@pytest.mark.parametrize("V, high, top_k", [(40003, 2500, 12000), (5003, 900, 4000), (151936, 20000, 100000)], ids=str)
@pytest.mark.parametrize("spread", [0.01, 0.3])
def test_cuts_between_two_bins(gpu_lib, V, high, top_k, spread):
    g = np.random.default_rng([101, V])
    made = [clusters(g, V, high, top_k, spread) for _ in range(50)]
    R = 300
    rows = torch.as_tensor(np.stack([x for x, _ in made]), device="cuda").float().repeat(R // 50, 1)
    top_p = torch.tensor([p for _, p in made], device="cuda").repeat(R // 50)
    kw = dict(top_k=top_k)
    first = gpu_lib.resispec_filter_logits(rows, top_p=top_p, **kw)
    torch.cuda.synchronize()
    # the border is between the clusters, or one element past it
    assert ((first[1] == high) | (first[1] == high + 1)).all() and (first[2] == 0).all()
    for _ in range(4):
        for lo, hi in ((0, 300), (0, 150), (50, 100), (200, 300)):
            part = gpu_lib.resispec_filter_logits(rows[lo:hi], top_p=top_p[lo:hi], **kw)
            torch.cuda.synchronize()
            assert torch.equal(part[1], first[1][lo:hi]), int((part[1] != first[1][lo:hi]).sum())
            assert torch.equal(part[0], first[0][lo:hi])
    # copies of a row in one batch
    assert (first[1].view(-1, 50) == first[1][:50]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("noise", [1e-4, 2e-3, 0.3])
def test_bins_whose_sums_pass_64_bits(gpu_lib, noise, dtype):
    """Nearly all of a row lies 6.8 above the eight runs that are its sample: masses of 2^9.8
    against the sample's maximum, 2^49.8 units each, 140,000 of them in a few bins."""
    V = 151936
    g = np.random.default_rng([111, int(noise * 1e5)])
    x = 6.8 + noise * np.abs(g.standard_normal((2, V)))
    x = np.minimum(x, 6.9)
    unit = 512 if dtype == torch.float32 else 1024          # elements of a chunk, 256 slots at most
    slots = -(-V // unit)
    per = -(-slots // 256)
    slots = -(-slots // per)
    for w in range(8):
        at = w * slots // 8 * per * unit
        x[:, at:at + 1024] = -0.01 * g.random((2, len(x[0, at:at + 1024])))
    rows = torch.as_tensor(x, device="cuda").to(dtype)
    for i, s in enumerate((dict(top_p=0.9), dict(top_p=0.3), dict(top_p=1.0 - 2.0 ** -24), dict(top_p=1e-6),
                           dict(top_k=30000), dict(top_p=0.5, min_p=0.999), dict())):
        check_sample(gpu_lib, rows, uniforms(2, 3, i), **s)
        mask = np.stack([kept(l, **s) for l in to64(rows)])
        out, n, st = gpu_lib.resispec_filter_logits(rows, **s)
        torch.cuda.synchronize()
        assert (torch.isfinite(out).cpu().numpy() == mask).all() and n.tolist() == mask.sum(1).tolist()
