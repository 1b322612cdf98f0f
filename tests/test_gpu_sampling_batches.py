"""A row's outputs are the same in every batch, where rounding decides them too: the cuts of
these rows lie within 1e-17 of the row's mass from the border between two elements, so that
another order of the same sums puts some of them on its other side.  Batches of up to 256 rows
and larger ones take workgroups of different sizes."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

F32 = torch.float32


def border_row(g, V, sigma, T, top_k, share):
    """A row of V fp32 logits and the top_p (an fp32 number near `share`) whose cut, under
    temperature T and top_k, falls on a border: two elements near zero, where fp32 numbers
    are dense, are set so that a prefix of the order has that share of the mass."""
    x = (sigma * g.standard_normal(V)).astype(np.float32).astype(np.float64)
    n = V if top_k == 0 else top_k
    T = float(np.float32(T))

    def sums():
        order = np.lexsort((np.arange(V), -x))[:n]
        w = np.exp((x[order] - x[order[0]]).astype(np.longdouble) / np.longdouble(T))
        return order, w.cumsum()
    order, c = sums()
    at = int((c < share * c[-1]).sum())
    shift = x[order[at // 2]]
    x = (x - shift).astype(np.float32).astype(np.float64)
    order, c = sums()
    knobs = order[at // 2 + 1], order[at // 2 + 2]
    x[knobs[0]], x[knobs[1]] = 0.0, 0.0
    order, c = sums()
    top_p = np.longdouble(np.float32(c[at] / c[-1]))
    top = x[order[0]]
    for j in knobs:
        # mass to be added to the element, to the prefix and to the whole
        need = (top_p * c[-1] - c[at]) / (1.0 - top_p)
        w = np.exp(np.longdouble(x[j] - top) / np.longdouble(T))
        x[j] = float(np.float32(top + T * np.log(w + need)))
        order, c = sums()
    assert abs(c[at] - top_p * c[-1]) < 1e-17 * c[-1]
    return x, float(top_p)


# V, standard deviation of the logits, temperature, top_k, share: the search over linear bins
# with few and with many elements in the cut's bin, a long list under top-k, the search over
# ranges of keys, and rows too short for a sample
KINDS = [(20011, 1.0, 1.0, 0, 0.9), (151936, 0.3, 1.0, 0, 0.8), (151936, 1.0, 1.0, 540, 0.6), (40003, 1.0, 0.8, 3000, 0.7),
         (5003, 1.0, 1.0, 0, 0.9), (5003, 1.0, 1.0, 2000, 0.9)]


@pytest.mark.parametrize("V, sigma, T, top_k, share", KINDS, ids=str)
def test_cuts_on_a_border_in_every_batch(gpu_lib, V, sigma, T, top_k, share):
    g = np.random.default_rng([81, V, top_k])
    made = [border_row(g, V, sigma, T, top_k, share) for _ in range(60)]
    R = 300
    rows = torch.as_tensor(np.stack([x for x, _ in made]), device="cuda").to(F32).repeat(R // 60, 1)
    top_p = torch.tensor([p for _, p in made], device="cuda", dtype=F32).repeat(R // 60)
    u = torch.as_tensor((np.random.default_rng(82).integers(0, 1 << 24, (60, 3)) * 2.0 ** -24).astype(np.float32),
                        device="cuda").repeat(R // 60, 1)
    whole = (*gpu_lib.resispec_sample(rows, u, temperature=T, top_k=top_k, top_p=top_p),
             *gpu_lib.resispec_filter_logits(rows, temperature=T, top_k=top_k, top_p=top_p))
    torch.cuda.synchronize()
    for lo, hi in ((0, 150), (60, 61), (59, 240), (120, 300)):
        part = (*gpu_lib.resispec_sample(rows[lo:hi], u[lo:hi], temperature=T, top_k=top_k, top_p=top_p[lo:hi]),
                *gpu_lib.resispec_filter_logits(rows[lo:hi], temperature=T, top_k=top_k, top_p=top_p[lo:hi]))
        torch.cuda.synchronize()
        for i, (x, y) in enumerate(zip(part, whole)):
            assert torch.equal(x, y[lo:hi]), (i, lo, hi, int((x != y[lo:hi]).flatten(1).any(1).sum())
                                              if x.dim() > 1 else int((x != y[lo:hi]).sum()))
    # the filtered rows keep what the draws are made from, on either side of the border
    assert torch.equal(whole[2], whole[5]) and (whole[3] == 0).all() and (whole[6] == 0).all()
    assert torch.equal(torch.isfinite(whole[4]).sum(1).int(), whole[5])
