"""The sampling operators as a decoding loop uses them together: filtered draft rows give the
candidates, filtered target rows verify them, the returned tokens get their log-probabilities;
and positions without trees draw their candidates, verify them and fall back to a draw."""
import numpy as np
import pytest
import torch

from paper_2608_24411_amd import synth
from parity_util import compare_walk, oracle_walk
from sampling_util import kept, logprob, to64

pytestmark = pytest.mark.gpu


def settings(B, T):
    g = torch.Generator().manual_seed(B)
    pick = torch.randint(4, (B,), generator=g)
    top_k = torch.tensor([0, 40, 0, 8], dtype=torch.int32)[pick].cuda()
    top_p = torch.tensor([0.9, 0.95, 1.0, 1.0])[pick].cuda()
    min_p = torch.tensor([0.0, 0.0, 0.05, 0.01])[pick].cuda()
    return dict(temperature=T, top_k=top_k, top_p=top_p, min_p=min_p)


@pytest.mark.parametrize("mode", ["resispec", "specinfer"])
@pytest.mark.parametrize("cfg,over", [(1, dict(B=8)), (2, dict(B=4, V=40961)), (4, dict(B=6, V=32128))],
                         ids=["chain-f32", "wide-bf16", "serving-bf16"])
def test_speculative_step_under_filters(gpu_lib, cfg, over, mode):
    w = synth.make_workload(cfg, device="cuda", **over)
    B, N, T, md = w["B"], w["N"], w["temperature"], w["max_depth"]
    s = settings(B, T)
    draft, dn, ds = gpu_lib.resispec_filter_logits(w["draft"], **s)
    target, tn, ts = gpu_lib.resispec_filter_logits(w["target"], **s)
    tok, ua, ur, st = gpu_lib.resispec_draft_candidates(draft, w["parent"], temperature=T,
                                                        without_replacement=w["without_replacement"], seed=17)
    kw = dict(temperature=T, max_depth=md, mode=mode, without_replacement=w["without_replacement"])
    out, length, vst = gpu_lib.resispec_verify_tree(target, draft, tok, w["parent"], ua, ur, **kw)
    others = (gpu_lib.resispec_verify_tree_deferred(target, draft, tok, w["parent"], ua, ur, **kw),
              gpu_lib.resispec_verify_tree_path_group(target, draft, tok, w["parent"], ua, ur, **kw))
    torch.cuda.synchronize()
    assert (ds == 0).all() and (ts == 0).all() and (st == 0).all()
    for a in others:
        assert torch.equal(a[0], out) and torch.equal(a[1], length) and torch.equal(a[2], vst)
    # candidates come from the kept part of their parent's draft row (-1: without replacement
    # a row can keep fewer elements than the node has children)
    par = synth.to_host(w["parent"])
    host = tok.cpu().numpy()
    keep = [[kept(to64(x[b, n]), T, int(s["top_k"][b]), float(s["top_p"][b]), float(s["min_p"][b]))
             for n in range(N)] for x in (w["draft"],) for b in range(B)]
    for b in range(B):
        for n in range(1, N):
            if host[b, n] >= 0:
                assert keep[b][par[b, n]][host[b, n]]
    # the verification of the filtered rows is the oracle's
    h = dict(target=synth.to_host(target), draft=synth.to_host(draft), node_token=host.copy(), parent=par,
             u_accept=ua.cpu().numpy(), u_resample=ur.cpu().numpy())
    whole = np.array([(host[b, 1:] >= 0).all() for b in range(B)])
    assert whole.any()
    h["node_token"][:, 0] = 0
    pick = torch.as_tensor(np.flatnonzero(whole), device="cuda")
    hw = {k: v[whole] for k, v in h.items()}
    gpu = {"tokens": out[pick], "accepted_len": length[pick], "status": vst[pick]}
    compare_walk(gpu, oracle_walk(hw, w, mode), hw, w, mode)
    # every emitted token is kept by the target row that it follows, and its log-probability
    # there is that of the filtered distribution
    tokens, lens, status = out.cpu().numpy(), length.cpu().numpy(), vst.cpu().numpy()
    rows, at = np.zeros((B, md + 1), dtype=np.int64), np.full((B, md + 1), -1, dtype=np.int32)
    for b in np.flatnonzero(status == 0):
        node = 0
        for i in range(lens[b] + 1):
            rows[b, i], at[b, i] = node, tokens[b, i]
            kids = [n for n in range(1, N) if par[b, n] == node and host[b, n] == tokens[b, i]]
            node = kids[0] if kids else node
    path = target[torch.arange(B, device="cuda").unsqueeze(1), torch.as_tensor(rows, device="cuda")].contiguous()
    lp, rank, lst = gpu_lib.resispec_token_logprobs(path, torch.as_tensor(at, device="cuda").unsqueeze(2),
                                                    temperature=T)
    torch.cuda.synchronize()
    assert (lst == 0).all()
    for b in range(B):
        for i in range(md + 1):
            if at[b, i] < 0:
                assert float(lp[b, i]) == 0.0 and int(rank[b, i]) == 0
                continue
            l = to64(w["target"][b, rows[b, i]])
            mask = kept(l, T, int(s["top_k"][b]), float(s["top_p"][b]), float(s["min_p"][b]))
            assert mask[at[b, i]]
            p, n = logprob(np.where(mask, l, -np.inf), T, at[b, i])
            # half a step of the result, and the 32-bit exponentials' 4.8e-6 (test_gpu_sampling)
            assert int(rank[b, i]) == n and abs(float(lp[b, i]) - p) <= abs(p) * 2.0 ** -24 + 4.8e-6


def test_candidates_of_a_flat_verification(gpu_lib):
    """Candidates drawn for positions without trees: what resispec_verify accepts of them is
    kept by both rows, and what it draws instead is kept by the target row."""
    B, k, T = 40, 6, 0.8
    w = synth.make_workload(0, device="cuda", B=B, V=32000)
    s = settings(B, T)
    g = torch.Generator(device="cuda").manual_seed(3)
    u = torch.rand((B, 2 * k + 2), generator=g, device="cuda")
    cand, clp, n, st = gpu_lib.resispec_sample(w["draft"], u[:, :k].contiguous(), **s)
    draft, _, _ = gpu_lib.resispec_filter_logits(w["draft"], **s)
    target, _, _ = gpu_lib.resispec_filter_logits(w["target"], **s)
    tok, length, vst = gpu_lib.resispec_verify(target, draft, cand, u[:, k:2 * k].contiguous(), u[:, -1].contiguous(),
                                               temperature=T)
    lp, rank, lst = gpu_lib.resispec_token_logprobs(draft, cand, temperature=T)
    # a draw from the rows already filtered is the same draw
    again = gpu_lib.resispec_sample(draft, u[:, :k].contiguous(), temperature=T)
    torch.cuda.synchronize()
    assert (st == 0).all() and (vst == 0).all() and (lst == 0).all()
    assert torch.equal(again[0], cand) and torch.equal(again[2], n)
    # both are the candidate's log-probability among what is kept (4.8e-6: test_gpu_sampling)
    assert ((lp - clp).abs() <= clp.abs() * 2.0 ** -23 + 4.8e-6).all()
    assert (rank <= n.unsqueeze(1)).all()
    assert torch.isfinite(target.float().gather(1, tok.long().unsqueeze(1))).all()
    hit = length == 1
    assert hit.any() and (cand == tok.unsqueeze(1)).any(1)[hit].all()
    # positions without a draft: one draw each, from the target's own settings
    one, olp, on, ost = gpu_lib.resispec_sample(w["target"], u[:, -2:-1].contiguous(), **s)
    torch.cuda.synchronize()
    assert (ost == 0).all() and torch.isfinite(target.float().gather(1, one.long())).all()
