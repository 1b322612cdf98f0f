"""The sampling entry points' argument checks: every call below returns before any launch."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2608_24411_amd import native
from sampling_util import draw, kept, logprob

FAKE = ctypes.c_void_p(0x10000)     # never dereferenced


def flt(**kw):
    f = native.RsFilter(native.RS_BF16, 1, 1.0, 0, 1.0, 0.0)
    for k, v in kw.items():
        setattr(f, k, v)
    return f


def sample(logits=FAKE, stride=100, u=FAKE, R=4, V=100, k=2, f=None, token=FAKE):
    return native.lib.resispec_sample(logits, stride, u, R, V, k, ctypes.byref(f or flt()), token, None, None,
                                      None, None)


def filt(logits=FAKE, stride=100, R=4, V=100, f=None, out=FAKE, out_stride=100):
    return native.lib.resispec_filter_logits(logits, stride, R, V, ctypes.byref(f or flt()), out, out_stride, None,
                                             None, None)


def logp(logits=FAKE, stride=100, tokens=FAKE, R=4, V=100, k=2, f=None, out=FAKE):
    return native.lib.resispec_token_logprobs(logits, stride, tokens, R, V, k, ctypes.byref(f or flt()), out, None,
                                              None, None)


BAD_FILTERS = [dict(logits_dtype=2), dict(logits_dtype=-1), dict(rows_per_entry=0), dict(rows_per_entry=-1),
               dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=float("inf")),
               dict(temperature=float("nan")), dict(top_k=-1), dict(top_p=0.0), dict(top_p=-0.5), dict(top_p=1.5),
               dict(top_p=float("nan")), dict(min_p=-0.1), dict(min_p=1.5), dict(min_p=float("nan"))]


@pytest.mark.parametrize("bad", BAD_FILTERS, ids=str)
def test_bad_settings(bad):
    for call in (sample, filt, logp):
        assert call(f=flt(**bad)) == native.RS_ERR_INVALID_ARG


@pytest.mark.parametrize("call", (sample, filt, logp))
def test_bad_sizes(call):
    assert call(R=-1) == native.RS_ERR_INVALID_ARG
    assert call(V=0) == native.RS_ERR_INVALID_ARG
    assert call(stride=99) == native.RS_ERR_INVALID_ARG
    assert call(logits=None) == native.RS_ERR_INVALID_ARG
    big = (1 << 22) + 1
    kw = dict(stride=big, V=big)
    if call is filt:
        kw["out_stride"] = big
    assert call(**kw) == native.RS_ERR_UNSUPPORTED
    # no rows: nothing to do, whatever the pointers
    assert call(R=0, logits=None) == native.RS_OK


def test_bad_pointers_and_counts():
    assert sample(u=None) == native.RS_ERR_INVALID_ARG
    assert sample(token=None) == native.RS_ERR_INVALID_ARG
    assert sample(k=0) == native.RS_ERR_INVALID_ARG
    assert sample(k=native.RS_MAX_CANDIDATES + 1) == native.RS_ERR_UNSUPPORTED
    assert filt(out=None) == native.RS_ERR_INVALID_ARG
    assert filt(out_stride=99) == native.RS_ERR_INVALID_ARG
    assert logp(tokens=None) == native.RS_ERR_INVALID_ARG
    assert logp(out=None) == native.RS_ERR_INVALID_ARG
    assert logp(k=0) == native.RS_ERR_INVALID_ARG
    assert logp(k=native.RS_MAX_CANDIDATES + 1) == native.RS_ERR_UNSUPPORTED
    for kw in (dict(top_k=5), dict(top_p=0.9), dict(min_p=0.1), dict(top_ks=0x10000), dict(top_ps=0x10000),
               dict(min_ps=0x10000)):      # a log-probability is that of the whole row
        assert logp(f=flt(**kw)) == native.RS_ERR_INVALID_ARG
    for call in (native.lib.resispec_sample, native.lib.resispec_filter_logits):
        args = [FAKE, 100, FAKE, 4, 100, 2, None, FAKE, None, None, None, None]
        if call is native.lib.resispec_filter_logits:
            args = [FAKE, 100, 4, 100, None, FAKE, 100, None, None, None]
        assert call(*args) == native.RS_ERR_INVALID_ARG


def test_an_array_stands_in_for_its_number():
    """A device array wins over the number beside it, so the number is not checked; the
    call is stopped here by a NULL output instead."""
    f = flt(temperature=0.0, top_k=-1, top_p=0.0, min_p=-1.0, temperatures=0x10000, top_ks=0x10000,
            top_ps=0x10000, min_ps=0x10000)
    assert sample(f=f, R=0) == native.RS_OK
    assert filt(f=f, R=0) == native.RS_OK
    assert sample(f=f, token=None) == native.RS_ERR_INVALID_ARG


def test_binding_refuses_host_tensors_and_types():
    x = torch.zeros(2, 8)
    u = torch.zeros(2, 1)
    for call in (lambda t: native.resispec_sample(t, u), native.resispec_filter_logits,
                 lambda t: native.resispec_token_logprobs(t, u.int())):
        with pytest.raises(ValueError):
            call(x)
        with pytest.raises(ValueError):
            call(None)


def test_status_codes_match_the_header():
    import os
    import re
    root = os.path.dirname(os.path.dirname(os.path.abspath(native.__file__)))
    text = open(os.path.join(root, "include", "resispec.h")).read()
    codes = dict(re.findall(r"(RS_SEQ_\w+) = (\d+)", text))
    for name, value in codes.items():
        assert getattr(native, name) == int(value)
    fields = re.search(r"typedef struct \{([^}]*)\} rs_filter;", text).group(1)
    fields = re.sub(r"/\*.*?\*/", "", fields, flags=re.S)
    assert re.findall(r"(\w+);", fields) == [n for n, _ in native.RsFilter._fields_]
    assert ctypes.sizeof(native.RsFilter) == 56


def test_plain_definition_on_a_row_worked_by_hand():
    """Masses 4, 2, 2, 1, 1 (powers of two in ln 2 steps), vocabulary order mixed."""
    l = np.log(np.array([1.0, 2.0, 4.0, 2.0, 1.0]))
    l[3] = l[1]
    assert kept(l).all()
    assert kept(l, top_k=1).tolist() == [0, 0, 1, 0, 0]
    assert kept(l, top_k=2).tolist() == [0, 1, 1, 0, 0]       # of equal logits the first
    assert kept(l, top_k=3).tolist() == [0, 1, 1, 1, 0]
    assert kept(l, top_p=0.35).tolist() == [0, 0, 1, 0, 0]
    assert kept(l, top_p=0.55).tolist() == [0, 1, 1, 0, 0]
    assert kept(l, top_p=0.65).tolist() == [0, 1, 1, 1, 0]
    assert kept(l, top_k=3, top_p=0.7).tolist() == [0, 1, 1, 0, 0]   # of the three's mass 8
    assert kept(l, min_p=0.4).tolist() == [0, 1, 1, 1, 0]
    assert kept(l, min_p=1.0).tolist() == [0, 0, 1, 0, 0]
    assert kept(np.array([-np.inf, -np.inf])) is None
    every = np.ones(5, dtype=bool)
    assert [draw(l, 1.0, every, u)[0] for u in (0.0, 0.0999, 0.15, 0.35, 0.75, 0.95)] == [0, 0, 1, 2, 3, 4]
    assert abs(draw(l, 1.0, every, 0.35)[1] - np.log(0.4)) < 1e-12
    assert logprob(l, 1.0, 3)[1] == 3 and abs(logprob(l, 1.0, 3)[0] - np.log(0.2)) < 1e-12


def test_binding_refuses_a_count_past_32_bits():
    """ctypes keeps the low 32 bits: 2^32 would turn top-k off, 2^32 + 5 keep five."""
    x = torch.zeros(2, 8)
    for top_k in (1 << 31, 1 << 32, (1 << 32) + 5, -(1 << 31) - 1):
        with pytest.raises(ValueError):
            native._settings(x, x.shape[:1], 2, 1.0, top_k, 1.0, 0.0)
    assert native._settings(x, x.shape[:1], 2, 1.0, (1 << 31) - 1, 1.0, 0.0).top_k == (1 << 31) - 1
