"""Argument checks of beam search's choice, the moves of states and the paged cache: every call
below returns before any launch."""
import ctypes
import itertools

import numpy as np
import pytest
import torch

from beam_util import accepted_path, plan, select
from paper_2608_24411_amd import native

lib = native.lib
FAKE = ctypes.c_void_p(0x10000)     # never dereferenced
INVALID, WORKSPACE, UNSUPPORTED = native.RS_ERR_INVALID_ARG, native.RS_ERR_WORKSPACE, native.RS_ERR_UNSUPPORTED


def flt(**kw):
    f = native.RsFilter(native.RS_BF16, 1, 1.0, 0, 1.0, 0.0)
    for k, v in kw.items():
        setattr(f, k, v)
    return f


def beam(logits=FAKE, stride=100, scores=FAKE, B=2, W=4, V=100, k=4, f=None, parent=FAKE, token=FAKE, score=FAKE, ws=FAKE,
         size=1 << 20):
    return lib.resispec_beam_select(logits, stride, scores, None, 2, B, W, V, k, ctypes.byref(f or flt()), parent, token,
                                    score, None, ws, size, None)


def test_beam_select_refusals():
    for bad in (dict(logits_dtype=2), dict(rows_per_entry=0), dict(temperature=0.0), dict(temperature=float("nan")),
                dict(temperature=float("inf")), dict(top_k=1), dict(top_p=0.5), dict(min_p=0.1), dict(top_ks=0x10000),
                dict(top_ps=0x10000), dict(min_ps=0x10000)):
        assert beam(f=flt(**bad)) == INVALID, bad
    assert lib.resispec_beam_select(FAKE, 100, FAKE, None, 2, 2, 4, 100, 4, None, FAKE, FAKE, FAKE, None, FAKE, 1 << 20,
                                    None) == INVALID
    for kw in (dict(B=-1), dict(W=0), dict(V=0), dict(k=0), dict(stride=99), dict(W=2, V=3, stride=3, k=7), dict(logits=None),
               dict(scores=None), dict(parent=None), dict(token=None), dict(score=None)):
        assert beam(**kw) == INVALID, kw
    for kw in (dict(W=65), dict(k=65), dict(V=(1 << 22) + 1, stride=1 << 23), dict(B=1 << 21, W=4), dict(B=1 << 22, W=1)):
        assert beam(**kw) == UNSUPPORTED, kw
    need = native.resispec_beam_workspace_bytes(2, 4, 100)
    assert need > 0
    for kw in (dict(ws=None), dict(size=need - 1), dict(ws=ctypes.c_void_p(0x10008))):
        assert beam(**kw) == WORKSPACE, kw
    assert beam(B=0, logits=None, ws=None) == native.RS_OK


def test_workspace_bytes():
    f = native.resispec_beam_workspace_bytes
    assert [f(0, 4, 100), f(2, 0, 100), f(2, 4, 0), f(2, 65, 100), f(2, 4, (1 << 22) + 1), f(1 << 21, 4, 100)] == [0] * 6
    assert f(3, 5, 151936) == 15 * f(1, 1, 151936) > 0
    # past 32 bits: the most rows of the largest vocabulary
    assert f((1 << 17) - 1, 64, 1 << 22) == ((1 << 17) - 1) * 64 * f(1, 1, 1 << 22) > 1 << 32


def rows(**kw):
    d = dict(outer=2, pages=8, inner=3, positions=5, row_bytes=16, outer_stride=8 * 3 * 5 * 16, page_stride=3 * 5 * 16,
             inner_stride=5 * 16, position_stride=16)
    return native.RsRows(**{**d, **kw})


def reorder(src=FAKE, s=None, dst=ctypes.c_void_p(0x90000), d=None, parent=FAKE, lengths=None, B=2, W=4, K=4):
    return lib.resispec_beam_reorder(src, ctypes.byref(s or rows()), dst, ctypes.byref(d or rows()), parent, lengths, B, W, K, None, None)


def paged(src=FAKE, s=None, table=FAKE, step=6, dst=FAKE, d=None, to=FAKE, to_step=6, n=6, parent=FAKE, lengths=FAKE, B=2,
          W=4, K=4):
    return lib.resispec_beam_reorder_paged(src, ctypes.byref(s or rows()), table, step, dst, ctypes.byref(d or rows()), to, to_step, n, parent,
                                           lengths, B, W, K, None, None)


@pytest.mark.parametrize("call", [reorder, paged])
def test_reorder_refusals(call):
    for name, bad in itertools.product(("outer", "pages", "inner", "positions", "row_bytes"), (0, -1)):
        assert call(s=rows(**{name: bad})) == INVALID and call(d=rows(**{name: bad})) == INVALID
    for name in ("outer_stride", "page_stride", "inner_stride", "position_stride"):
        assert call(s=rows(**{name: -16})) == INVALID
    for name in ("outer", "inner", "positions", "row_bytes"):
        assert call(d=rows(**{name: 4})) == INVALID, name
    for kw in (dict(B=-1), dict(W=0), dict(K=0), dict(src=None), dict(dst=None), dict(parent=None)):
        assert call(**kw) == INVALID, kw
    assert call(W=65) == UNSUPPORTED and call(K=65) == UNSUPPORTED
    big = dict(outer=1 << 16, inner=1 << 16)
    assert call(s=rows(**big), d=rows(**big)) == UNSUPPORTED
    assert call(s=rows(positions=1 << 40), d=rows(positions=1 << 40)) == UNSUPPORTED
    assert call(s=rows(row_bytes=1 << 62), d=rows(row_bytes=1 << 62)) == UNSUPPORTED
    wide = rows(pages=1 << 26)
    assert call(s=wide, d=wide, B=1 << 24) == UNSUPPORTED
    assert call(B=0, src=None) == native.RS_OK


def test_reorder_places():
    assert reorder(s=rows(pages=7)) == INVALID and reorder(d=rows(pages=9)) == INVALID
    # in place: the same layout, as many beams
    assert reorder(dst=FAKE, d=rows(outer_stride=4096)) == INVALID
    assert reorder(dst=FAKE, K=2, d=rows(pages=4)) == INVALID
    for kw in (dict(table=None), dict(to=None), dict(lengths=None), dict(n=0), dict(step=5), dict(to_step=5)):
        assert paged(**kw) == INVALID, kw
    assert paged(d=rows(page_stride=4096)) == INVALID
    assert paged(n=1 << 30, step=1 << 30, to_step=1 << 30) == UNSUPPORTED


def plan_call(kept=FAKE, added=FAKE, held=FAKE, R=3, P=16, table=FAKE, step=8, n=8, free=FAKE, count=FAKE, pages=100,
              got=FAKE, left=FAKE, starts=FAKE, T=10, slots=FAKE):
    return lib.resispec_plan_cache(kept, added, held, R, P, table, step, n, free, count, pages, got, left, starts, T, slots,
                                   None, None, None, None)


def test_plan_refusals():
    for kw in (dict(R=-1), dict(T=-1), dict(P=0), dict(pages=0), dict(n=0), dict(step=7), dict(kept=None), dict(added=None),
               dict(held=None), dict(table=None), dict(free=None), dict(count=None), dict(got=None), dict(left=None),
               dict(starts=None), dict(slots=None)):
        assert plan_call(**kw) == INVALID, kw
    assert plan_call(pages=1 << 27) == UNSUPPORTED
    assert plan_call(n=1 << 28, step=1 << 28) == UNSUPPORTED


def path_call(parent=FAKE, token=FAKE, tokens=FAKE, length=FAKE, B=2, N=5, D=3, out=FAKE):
    return lib.resispec_accepted_path(parent, token, tokens, length, B, N, D, out, None, None)


def commit_call(cache=FAKE, c=None, slots=FAKE, path=FAKE, source=None, s=None, B=8, N=5, depth=3):
    return lib.resispec_commit_path(cache, ctypes.byref(c or rows()), slots, path, source, None if s is None else ctypes.byref(s), B,
                                    N, depth, None, None)


def test_path_and_commit_refusals():
    for kw in (dict(B=-1), dict(N=0), dict(D=-1), dict(D=(1 << 31) - 1), dict(parent=None), dict(token=None),
               dict(tokens=None), dict(length=None), dict(out=None)):
        assert path_call(**kw) == INVALID, kw
    assert path_call(N=native.RS_MAX_PATH_NODES + 1) == UNSUPPORTED and path_call(B=1 << 22) == UNSUPPORTED
    assert path_call(B=0, parent=None) == native.RS_OK
    for kw in (dict(B=-1), dict(N=0), dict(depth=0), dict(cache=None), dict(slots=None), dict(path=None),
               dict(c=rows(row_bytes=0)), dict(source=FAKE), dict(source=FAKE, s=rows(pages=7)),
               dict(source=FAKE, s=rows(positions=6)), dict(source=FAKE, s=rows(row_bytes=8)),
               dict(source=FAKE, s=rows(outer=1)), dict(source=FAKE, s=rows(inner=1))):
        assert commit_call(**kw) == INVALID, kw
    for kw in (dict(N=native.RS_MAX_PATH_NODES + 1), dict(depth=native.RS_MAX_PATH_NODES + 1),
               dict(c=rows(pages=1 << 30)), dict(c=rows(outer=1 << 20, inner=1 << 20)), dict(c=rows(row_bytes=1 << 31)),
               dict(B=1 << 24, c=rows(pages=8))):
        assert commit_call(**kw) == UNSUPPORTED, kw
    assert commit_call(B=0, cache=None) == native.RS_OK


def test_binding_refuses_host_tensors():
    x, i = torch.zeros(2, 4, 8), torch.zeros(2, 4, dtype=torch.int32)
    n = torch.zeros(2, dtype=torch.int32)
    for call in (lambda: native.resispec_beam_select(x, x[:, :, 0]), lambda: native.resispec_beam_reorder(x, i),
                 lambda: native.resispec_beam_reorder_paged(x, i, i, n),
                 lambda: native.resispec_plan_cache(n, n, n, i, n, n[:1], page_size=4, max_slots=3),
                 lambda: native.resispec_accepted_path(i, i, i, n), lambda: native.resispec_commit_path(x, i, i)):
        with pytest.raises(ValueError):
            call()


def layout(t, *dims):
    r, span, _ = native._layout(t.shape, t.stride(), t.element_size(), *dims, "t")
    return tuple(getattr(r, n) for n, _ in native.RsRows._fields_), span


def test_layouts():
    t = torch.zeros(3, 2, 8, 4, 5, 6, dtype=torch.bfloat16)
    whole = t.numel() * 2
    assert layout(t, 2, 4) == ((6, 8, 4, 5, 12, 8 * 4 * 60, 240, 60, 12), whole)
    assert layout(t, 2, 3) == ((6, 8, 1, 4, 60, 8 * 240, 240, 0, 60), whole)
    assert layout(t, 2, None) == ((6, 8, 1, 1, 240, 8 * 240, 240, 0, 0), whole)
    assert layout(t, -4, -1) == ((6, 8, 20, 6, 2, 8 * 240, 240, 12, 2), whole)
    # heads behind positions, and part of a tensor
    assert layout(t.transpose(3, 4)[..., :5], 2, 4) == ((6, 8, 5, 4, 10, 8 * 240, 240, 12, 60), whole - 2)
    for bad, dims in ((t[..., ::2], (2, 4)), (t[:, :1].expand(3, 2, 8, 4, 5, 6), (2, 4)), (t[:, :, :, :, :1].expand_as(t), (2, 4)),
                      (t[:, :, :, 1:, :3].transpose(0, 1), (2, 4)), (t, (4, 2)), (t, (2, 2)), (t, (6, 7)), (t[:0], (2, 4)),
                      (t[..., :0], (2, 4)), (t.transpose(4, 5), (2, 4))):
        with pytest.raises(ValueError):
            layout(bad, *dims)


def test_struct_matches_the_header():
    import os
    import re
    root = os.path.dirname(os.path.dirname(os.path.abspath(native.__file__)))
    text = open(os.path.join(root, "include", "resispec.h")).read()
    fields = re.search(r"typedef struct \{([^}]*)\} rs_rows;", text).group(1)
    fields = re.sub(r"/\*.*?\*/", "", fields, flags=re.S)
    names = [n.strip() for line in re.findall(r"int64_t ([^;]*);", fields) for n in line.split(",")]
    assert names == [n for n, _ in native.RsRows._fields_] and ctypes.sizeof(native.RsRows) == 72
    assert int(re.search(r"#define RS_MAX_PATH_NODES (\d+)", text).group(1)) == native.RS_MAX_PATH_NODES


def test_plain_forms_by_hand():
    l = np.log(np.array([[1.0, 2.0, 1.0], [3.0, 3.0, 2.0]]))
    l[1, 1] = l[1, 0]
    parent, token, score = select(l, np.log([0.5, 0.25]), 4)
    assert (parent, token) == ([0, 0, 0, 1], [1, 0, 2, 0])
    assert np.allclose(score, np.log([0.25, 0.125, 0.125, 0.09375]))
    parent, token, score = select(l, np.log([0.5, 0.25]), 3, ended=[1, 0], end_token=7)
    assert (parent, token) == ([0, 1, 1], [7, 0, 1])
    assert select(l, np.array([0.0, -np.inf]), 4)[0] == [0, 0, 0, -1]
    # two requests: one keeps 3 of its 6 positions and gets 2, one is new
    table, free = [[4, 5, 6], [-1, -1, -1]], [1, 2, 3, 0, -1, -1, -1]
    got = plan([3, 0], [2, 5], [3, 0], table, free, 4, 2, 8)
    assert table == [[4, 5, 6], [0, 3, 2]] and free[:2] == [1, 2]
    assert got[0] == [11, 12, 0, 1, 6, 7, 4, -1] and got[3:] == ([0, 2, 7], [3, 3], 1, [0, 0])
    assert accepted_path([-1, 0, 0, 1, 2], [9, 5, 5, 6, 7], [5, 7, 1], 2) == [0, 2, 4]
    assert accepted_path([-1, 0, 0, 1, 2], [9, 5, 5, 6, 7], [5, 8], 1) == [0, 1]
    assert accepted_path([-1, 0], [9, 5], [6, 1], 1) is None
