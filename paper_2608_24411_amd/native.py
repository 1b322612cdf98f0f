"""Python binding of libresispec.so: argument marshalling only.

Every entry point of include/resispec.h has a function of the same name here.  Torch
is used for device memory and the current HIP stream; every step of the verification
runs in the library's kernels.  There is no fallback: if the library cannot be loaded
the import fails.
"""
import ctypes
import functools
import os

HERE = os.path.dirname(os.path.abspath(__file__))
# an instrumented build (the sanitizer run of the CPU tests) is picked with this variable
LIB_PATH = os.environ.get("RESISPEC_LIBRARY") or os.path.join(HERE, "libresispec.so")

RS_OK, RS_ERR_INVALID_ARG, RS_ERR_WORKSPACE, RS_ERR_UNSUPPORTED, RS_ERR_HIP = range(5)
(RS_SEQ_OK, RS_SEQ_BAD_TOKEN, RS_SEQ_ZERO_DRAFT, RS_SEQ_UNDERFLOW, RS_SEQ_BAD_TREE,
 RS_SEQ_BAD_UNIFORM, RS_SEQ_DEPTH_EXCEEDED, RS_SEQ_TOO_MANY_CHILDREN, RS_SEQ_GROUP_TIMEOUT,
 RS_SEQ_DEFERRED, RS_SEQ_BAD_PARAM, RS_SEQ_BAD_PAGE, RS_SEQ_NO_ROOM) = range(13)
RS_MODE_RESISPEC, RS_MODE_SPECINFER = 0, 1
RS_F32, RS_BF16 = 0, 1
RS_MAX_CANDIDATES = 64
RS_MAX_PATH_NODES = 8192

MODES = {"resispec": RS_MODE_RESISPEC, "specinfer": RS_MODE_SPECINFER}

# Every symbol include/resispec.h declares.
EXPORTS = ("resispec_verify", "resispec_verify_tree", "resispec_verify_tree_noalloc",
           "resispec_verify_tree_deferred", "resispec_decide_nodes", "resispec_walk_draw",
           "resispec_deferred_workspace_bytes",
           "resispec_verify_tree_path",
           "resispec_verify_tree_path_group", "resispec_path_workspace_bytes",
           "resispec_path_group_size", "resispec_debug_set_group_waits", "resispec_debug_pool_held",
           "resispec_debug_fail_pool_launches",
           "resispec_verify_tree_group", "resispec_tree_group_workspace_bytes",
           "resispec_tree_group_size",
           "resispec_draft_candidates",
           "resispec_verify_nodes", "resispec_walk", "resispec_node_outcomes",
           "resispec_workspace_bytes", "resispec_validate_tree_host",
           "resispec_verify_tree_debug", "resispec_sample", "resispec_filter_logits",
           "resispec_token_logprobs", "resispec_beam_select", "resispec_beam_workspace_bytes",
           "resispec_beam_reorder", "resispec_beam_reorder_paged", "resispec_plan_cache",
           "resispec_accepted_path", "resispec_commit_path", "resispec_status_string", "resispec_abi_version")


class RsParams(ctypes.Structure):
    _fields_ = [("mode", ctypes.c_int32), ("logits_dtype", ctypes.c_int32),
                ("temperature", ctypes.c_float), ("without_replacement", ctypes.c_int32),
                ("bonus", ctypes.c_int32)]


class RsFilter(ctypes.Structure):
    _fields_ = [("logits_dtype", ctypes.c_int32), ("rows_per_entry", ctypes.c_int32),
                ("temperature", ctypes.c_float), ("top_k", ctypes.c_int32),
                ("top_p", ctypes.c_float), ("min_p", ctypes.c_float),
                ("temperatures", ctypes.c_void_p), ("top_ks", ctypes.c_void_p),
                ("top_ps", ctypes.c_void_p), ("min_ps", ctypes.c_void_p)]


class RsRows(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int64) for name in
                ("outer", "pages", "inner", "positions", "row_bytes", "outer_stride", "page_stride",
                 "inner_stride", "position_stride")]


class ResiSpecError(RuntimeError):
    pass


def _load():
    if not os.path.exists(LIB_PATH):
        from . import build as _build
        _build.build()
    lib = ctypes.CDLL(LIB_PATH)
    P, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    prm = ctypes.POINTER(RsParams)
    lib.resispec_verify.argtypes = [P, P, P, P, P, i32, i32, i32, prm, P, P, P, P]
    lib.resispec_verify.restype = i32
    lib.resispec_verify_tree.argtypes = [P, P, P, P, P, P, i32, i32, i32, i32, prm, P, P, P,
                                         P, sz, P]
    lib.resispec_verify_tree.restype = i32
    lib.resispec_verify_tree_noalloc.argtypes = [P, P, P, P, P, P, i32, i32, i32, i32, prm, P, P,
                                                 P, P]
    lib.resispec_verify_tree_noalloc.restype = i32
    lib.resispec_verify_tree_path.argtypes = [P, P, P, P, P, P, i32, i32, i32, i32, prm, P, P, P,
                                              P]
    lib.resispec_verify_tree_path.restype = i32
    lib.resispec_verify_tree_path_group.argtypes = [P, P, P, P, P, P, i32, i32, i32, i32, prm, P,
                                                    P, P, i32, P, sz, P]
    lib.resispec_verify_tree_path_group.restype = i32
    lib.resispec_path_workspace_bytes.argtypes = [i32, i32]
    lib.resispec_path_workspace_bytes.restype = sz
    lib.resispec_path_group_size.argtypes = [i32, i32, prm]
    lib.resispec_path_group_size.restype = i32
    lib.resispec_debug_set_group_waits.argtypes = [ctypes.c_uint64, ctypes.c_uint64]
    lib.resispec_debug_set_group_waits.restype = i32
    lib.resispec_debug_pool_held.argtypes = []
    lib.resispec_debug_pool_held.restype = i32
    lib.resispec_debug_fail_pool_launches.argtypes = [i32]
    lib.resispec_debug_fail_pool_launches.restype = i32
    lib.resispec_verify_tree_group.argtypes = [P, P, P, P, P, P, i32, i32, i32, i32, prm, P, P, P,
                                               i32, P, sz, P]
    lib.resispec_verify_tree_group.restype = i32
    lib.resispec_tree_group_workspace_bytes.argtypes = [i32, i32]
    lib.resispec_tree_group_workspace_bytes.restype = sz
    lib.resispec_tree_group_size.argtypes = [i32, i32, i32, prm]
    lib.resispec_tree_group_size.restype = i32
    lib.resispec_draft_candidates.argtypes = [P, P, i32, i32, i32, prm, ctypes.c_uint64,
                                              ctypes.c_uint64, P, P, P, P, P]
    lib.resispec_draft_candidates.restype = i32
    lib.resispec_verify_tree_debug.argtypes = [P, P, P, P, P, P, i32, i32, i32, i32, prm, P, P,
                                               P, P, sz, P, P, P, P, P]
    lib.resispec_verify_tree_debug.restype = i32
    lib.resispec_verify_tree_deferred.argtypes = [P, P, P, P, P, P, i32, i32, i32, i32, prm, P, P,
                                                  P, P, sz, P]
    lib.resispec_verify_tree_deferred.restype = i32
    lib.resispec_decide_nodes.argtypes = [P, P, P, P, P, P, i32, i32, i32, prm, P, sz, P]
    lib.resispec_decide_nodes.restype = i32
    lib.resispec_walk_draw.argtypes = [P, P, P, P, P, P, i32, i32, i32, i32, prm, P, sz, P, P, P, P]
    lib.resispec_walk_draw.restype = i32
    lib.resispec_deferred_workspace_bytes.argtypes = [i32, i32]
    lib.resispec_deferred_workspace_bytes.restype = sz
    lib.resispec_verify_nodes.argtypes = [P, P, P, P, P, P, i32, i32, i32, prm, P, sz, P]
    lib.resispec_verify_nodes.restype = i32
    lib.resispec_walk.argtypes = [P, i32, i32, i32, P, sz, P, P, P, P]
    lib.resispec_walk.restype = i32
    lib.resispec_node_outcomes.argtypes = [P, sz, i32, i32, P, P, P, P]
    lib.resispec_node_outcomes.restype = i32
    lib.resispec_workspace_bytes.argtypes = [i32, i32]
    lib.resispec_workspace_bytes.restype = sz
    lib.resispec_validate_tree_host.argtypes = [P, P, i32, i32, i32, ctypes.POINTER(i64)]
    lib.resispec_validate_tree_host.restype = i32
    flt = ctypes.POINTER(RsFilter)
    lib.resispec_sample.argtypes = [P, i64, P, i32, i32, i32, flt, P, P, P, P, P]
    lib.resispec_sample.restype = i32
    lib.resispec_filter_logits.argtypes = [P, i64, i32, i32, flt, P, i64, P, P, P]
    lib.resispec_filter_logits.restype = i32
    lib.resispec_token_logprobs.argtypes = [P, i64, P, i32, i32, i32, flt, P, P, P, P]
    lib.resispec_token_logprobs.restype = i32
    lib.resispec_beam_select.argtypes = [P, i64, P, P, i32, i32, i32, i32, i32, P, P, P, P, P, P, sz, P]
    lib.resispec_beam_select.restype = i32
    lib.resispec_beam_workspace_bytes.argtypes = [i32, i32, i32]
    lib.resispec_beam_workspace_bytes.restype = sz
    rows = P            # an rs_rows by its address: a struct kept with its layout is not wrapped again
    lib.resispec_beam_reorder.argtypes = [P, rows, P, rows, P, P, i32, i32, i32, P, P]
    lib.resispec_beam_reorder.restype = i32
    lib.resispec_beam_reorder_paged.argtypes = [P, rows, P, i64, P, rows, P, i64, i32, P, P, i32, i32, i32, P, P]
    lib.resispec_beam_reorder_paged.restype = i32
    lib.resispec_plan_cache.argtypes = [P, P, P, i32, i32, P, i64, i32, P, P, i32, P, P, P, i32, P, P, P, P, P]
    lib.resispec_plan_cache.restype = i32
    lib.resispec_accepted_path.argtypes = [P, P, P, P, i32, i32, i32, P, P, P]
    lib.resispec_accepted_path.restype = i32
    lib.resispec_commit_path.argtypes = [P, rows, P, P, P, rows, i32, i32, i32, P, P]
    lib.resispec_commit_path.restype = i32
    lib.resispec_status_string.argtypes = [i32]
    lib.resispec_status_string.restype = ctypes.c_char_p
    lib.resispec_abi_version.argtypes = []
    lib.resispec_abi_version.restype = i32
    return lib


lib = _load()


# ------------------------------------------------------------ plain entries --

def resispec_status_string(status: int) -> str:
    return lib.resispec_status_string(int(status)).decode()


def resispec_abi_version() -> int:
    return lib.resispec_abi_version()


def resispec_workspace_bytes(B: int, N: int) -> int:
    return lib.resispec_workspace_bytes(int(B), int(N))


def resispec_validate_tree_host(parent, node_token, V: int):
    """parent, node_token: host int32 arrays [B, N] (numpy).  Returns (status, first_bad)."""
    import numpy as np
    par = np.ascontiguousarray(parent, dtype=np.int32)
    tok = np.ascontiguousarray(node_token, dtype=np.int32)
    B, N = par.shape
    bad = ctypes.c_int64(-1)
    st = lib.resispec_validate_tree_host(par.ctypes.data, tok.ctypes.data, B, N, int(V),
                                         ctypes.byref(bad))
    return st, bad.value


# ------------------------------------------------------- torch marshalling --

def _params(logits, temperature, mode, without_replacement, bonus):
    import torch
    if logits.dtype == torch.float32:
        dt = RS_F32
    elif logits.dtype == torch.bfloat16:
        dt = RS_BF16
    else:
        raise TypeError("logits must be float32 or bfloat16")
    return RsParams(MODES[mode] if isinstance(mode, str) else int(mode), dt, float(temperature),
                    int(bool(without_replacement)), int(bool(bonus)))


def _dev(t, dtype, name):
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError("%s must be a device tensor" % name)
    if t.dtype != dtype:
        raise TypeError("%s must be %s" % (name, dtype))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return t.data_ptr()


def _shape(t, shape, name):
    if t.shape != shape and tuple(t.shape) != tuple(shape):
        raise ValueError("%s has shape %s, expected %s" % (name, tuple(t.shape), tuple(shape)))


def _same_device(*ts):
    devs = {t.device for t in ts if t is not None}
    if len(devs) > 1:
        raise ValueError("all tensors must be on one device, got %s" % devs)


def _check_tree_shapes(target_logits, draft_logits, node_token, parent, u_accept, u_resample):
    if target_logits.dim() != 3:
        raise ValueError("target_logits must be [B, N, V]")
    B, N, V = target_logits.shape
    _shape(draft_logits, (B, N, V), "draft_logits")
    for t, name in ((node_token, "node_token"), (parent, "parent"), (u_accept, "u_accept"),
                    (u_resample, "u_resample")):
        _shape(t, (B, N), name)
    _same_device(target_logits, draft_logits, node_token, parent, u_accept, u_resample)
    return B, N, V


@functools.lru_cache(maxsize=None)
def _runtime():
    """(current device, a device's current stream handle), as functions without the objects
    that torch.cuda makes around them (2.8 us of a 15.7 us call for the Stream alone)."""
    import torch
    device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is None:
        def raw(d):
            return torch.cuda.current_stream(d).cuda_stream
    return device, raw


def _stream(stream):
    if stream is not None:
        return ctypes.c_void_p(stream.cuda_stream)
    device, raw = _runtime()
    return ctypes.c_void_p(raw(device()))


def _check(st):
    if st != RS_OK:
        raise ResiSpecError(resispec_status_string(st))


def resispec_verify(target_logits, draft_logits, cand_ids, u_accept, u_resample, *,
                    temperature, mode="resispec", out_token=None, out_accepted_len=None,
                    out_status=None, stream=None):
    """Flat verify of B rows with k candidates each; returns (token, accepted_len, status)."""
    import torch
    if target_logits.dim() != 2 or cand_ids.dim() != 2:
        raise ValueError("target_logits must be [B, V] and cand_ids [B, k]")
    B, V = target_logits.shape
    k = cand_ids.shape[1]
    _shape(draft_logits, (B, V), "draft_logits")
    _shape(cand_ids, (B, k), "cand_ids")
    _shape(u_accept, (B, k), "u_accept")
    _shape(u_resample, (B,), "u_resample")
    _same_device(target_logits, draft_logits, cand_ids, u_accept, u_resample)
    dev = target_logits.device
    if out_token is None:
        out_token = torch.empty(B, dtype=torch.int32, device=dev)
    if out_accepted_len is None:
        out_accepted_len = torch.empty(B, dtype=torch.int32, device=dev)
    if out_status is None:
        out_status = torch.empty(B, dtype=torch.int32, device=dev)
    for t, name in ((out_token, "out_token"), (out_accepted_len, "out_accepted_len"),
                    (out_status, "out_status")):
        _shape(t, (B,), name)
    prm = _params(target_logits, temperature, mode, False, True)
    st = lib.resispec_verify(
        _dev(target_logits, target_logits.dtype, "target_logits"),
        _dev(draft_logits, target_logits.dtype, "draft_logits"),
        _dev(cand_ids, torch.int32, "cand_ids"), _dev(u_accept, torch.float32, "u_accept"),
        _dev(u_resample, torch.float32, "u_resample"), B, V, k, ctypes.byref(prm),
        _dev(out_token, torch.int32, "out_token"),
        _dev(out_accepted_len, torch.int32, "out_accepted_len"),
        _dev(out_status, torch.int32, "out_status"), _stream(stream))
    _check(st)
    return out_token, out_accepted_len, out_status


def _tree_common(target_logits, draft_logits, node_token, parent, u_accept, u_resample,
                 max_depth):
    if max_depth is None or int(max_depth) < 0:
        raise ValueError("max_depth (>= 0) is required")
    return _check_tree_shapes(target_logits, draft_logits, node_token, parent, u_accept,
                              u_resample)


def resispec_verify_tree(target_logits, draft_logits, node_token, parent, u_accept, u_resample,
                         *, temperature, max_depth, mode="resispec", without_replacement=False,
                         bonus=True, out_tokens=None, out_accepted_len=None, out_status=None,
                         workspace=None, stream=None):
    """Tree verify; returns (tokens [B, max_depth+1], accepted_len [B], status [B])."""
    import torch
    B, N, V = _tree_common(target_logits, draft_logits, node_token, parent, u_accept, u_resample,
                           max_depth)
    dev = target_logits.device
    if out_tokens is None:
        out_tokens = torch.empty((B, max_depth + 1), dtype=torch.int32, device=dev)
    if out_accepted_len is None:
        out_accepted_len = torch.empty(B, dtype=torch.int32, device=dev)
    if out_status is None:
        out_status = torch.empty(B, dtype=torch.int32, device=dev)
    _shape(out_tokens, (B, max_depth + 1), "out_tokens")
    _shape(out_accepted_len, (B,), "out_accepted_len")
    _shape(out_status, (B,), "out_status")
    wsb = resispec_workspace_bytes(B, N)
    if workspace is None:
        workspace = torch.empty(max(wsb, 1), dtype=torch.uint8, device=dev)
    prm = _params(target_logits, temperature, mode, without_replacement, bonus)
    st = lib.resispec_verify_tree(
        _dev(target_logits, target_logits.dtype, "target_logits"),
        _dev(draft_logits, target_logits.dtype, "draft_logits"),
        _dev(node_token, torch.int32, "node_token"), _dev(parent, torch.int32, "parent"),
        _dev(u_accept, torch.float32, "u_accept"), _dev(u_resample, torch.float32, "u_resample"),
        B, N, V, int(max_depth), ctypes.byref(prm),
        _dev(out_tokens, torch.int32, "out_tokens"),
        _dev(out_accepted_len, torch.int32, "out_accepted_len"),
        _dev(out_status, torch.int32, "out_status"),
        _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(stream))
    _check(st)
    return out_tokens, out_accepted_len, out_status


RS_NOALLOC_MAX_ROWS = 65536


def resispec_verify_tree_noalloc(target_logits, draft_logits, node_token, parent, u_accept,
                                 u_resample, *, temperature, max_depth, mode="resispec",
                                 without_replacement=False, bonus=True, out_tokens, out_accepted_len,
                                 out_status=None, stream=None):
    """resispec_verify_tree with the library's static per-GPU scratch instead of a
    workspace (B * N <= RS_NOALLOC_MAX_ROWS); the caller passes the outputs.  Calls that
    overlap on one GPU race."""
    import torch
    B, N, V = _tree_common(target_logits, draft_logits, node_token, parent, u_accept, u_resample,
                           max_depth)
    _shape(out_tokens, (B, max_depth + 1), "out_tokens")
    _shape(out_accepted_len, (B,), "out_accepted_len")
    if out_status is not None:
        _shape(out_status, (B,), "out_status")
    prm = _params(target_logits, temperature, mode, without_replacement, bonus)
    st = lib.resispec_verify_tree_noalloc(
        _dev(target_logits, target_logits.dtype, "target_logits"),
        _dev(draft_logits, target_logits.dtype, "draft_logits"),
        _dev(node_token, torch.int32, "node_token"), _dev(parent, torch.int32, "parent"),
        _dev(u_accept, torch.float32, "u_accept"), _dev(u_resample, torch.float32, "u_resample"),
        B, N, V, int(max_depth), ctypes.byref(prm),
        _dev(out_tokens, torch.int32, "out_tokens"),
        _dev(out_accepted_len, torch.int32, "out_accepted_len"),
        _dev(out_status, torch.int32, "out_status") if out_status is not None else None,
        _stream(stream))
    _check(st)
    return out_tokens, out_accepted_len, out_status


def resispec_verify_tree_path(target_logits, draft_logits, node_token, parent, u_accept,
                              u_resample, *, temperature, max_depth, mode="resispec",
                              without_replacement=False, bonus=True, out_tokens=None,
                              out_accepted_len=None, out_status=None, stream=None):
    """Path-only schedule of resispec_verify_tree (same results); returns
    (tokens [B, max_depth+1], accepted_len [B], status [B])."""
    import torch
    B, N, V = _tree_common(target_logits, draft_logits, node_token, parent, u_accept, u_resample,
                           max_depth)
    dev = target_logits.device
    if out_tokens is None:
        out_tokens = torch.empty((B, max_depth + 1), dtype=torch.int32, device=dev)
    if out_accepted_len is None:
        out_accepted_len = torch.empty(B, dtype=torch.int32, device=dev)
    if out_status is None:
        out_status = torch.empty(B, dtype=torch.int32, device=dev)
    _shape(out_tokens, (B, max_depth + 1), "out_tokens")
    _shape(out_accepted_len, (B,), "out_accepted_len")
    _shape(out_status, (B,), "out_status")
    prm = _params(target_logits, temperature, mode, without_replacement, bonus)
    st = lib.resispec_verify_tree_path(
        _dev(target_logits, target_logits.dtype, "target_logits"),
        _dev(draft_logits, target_logits.dtype, "draft_logits"),
        _dev(node_token, torch.int32, "node_token"), _dev(parent, torch.int32, "parent"),
        _dev(u_accept, torch.float32, "u_accept"), _dev(u_resample, torch.float32, "u_resample"),
        B, N, V, int(max_depth), ctypes.byref(prm),
        _dev(out_tokens, torch.int32, "out_tokens"),
        _dev(out_accepted_len, torch.int32, "out_accepted_len"),
        _dev(out_status, torch.int32, "out_status"), _stream(stream))
    _check(st)
    return out_tokens, out_accepted_len, out_status


def resispec_path_workspace_bytes(B: int, V: int) -> int:
    return lib.resispec_path_workspace_bytes(int(B), int(V))


def resispec_path_group_size(B: int, V: int, *, dtype, mode="resispec") -> int:
    """Members per sequence the grouped path schedule picks by itself (dtype: "bf16" or
    "f32"); -1 for invalid arguments."""
    prm = RsParams(MODES[mode], RS_BF16 if dtype == "bf16" else RS_F32, 1.0, 0, 1)
    return lib.resispec_path_group_size(int(B), int(V), ctypes.byref(prm))


def resispec_tree_group_workspace_bytes(B: int, N: int) -> int:
    return lib.resispec_tree_group_workspace_bytes(int(B), int(N))


def resispec_tree_group_size(B: int, N: int, V: int, *, dtype, mode="resispec") -> int:
    """Members per row the grouped all-nodes schedule picks by itself (dtype: "bf16" or
    "f32"); -1 for invalid arguments."""
    prm = RsParams(MODES[mode], RS_BF16 if dtype == "bf16" else RS_F32, 1.0, 0, 1)
    return lib.resispec_tree_group_size(int(B), int(N), int(V), ctypes.byref(prm))


def resispec_verify_tree_group(target_logits, draft_logits, node_token, parent, u_accept,
                               u_resample, *, temperature, max_depth, mode="resispec",
                               without_replacement=False, bonus=True, group_size=0,
                               workspace=None, out_tokens=None, out_accepted_len=None,
                               out_status=None, stream=None):
    """All-nodes verification with row groups (group_size workgroups per node row, 0 =
    automatic); same results as resispec_verify_tree.  Returns (tokens [B, max_depth+1],
    accepted_len [B], status [B])."""
    import torch
    B, N, V = _tree_common(target_logits, draft_logits, node_token, parent, u_accept, u_resample,
                           max_depth)
    dev = target_logits.device
    if out_tokens is None:
        out_tokens = torch.empty((B, max_depth + 1), dtype=torch.int32, device=dev)
    if out_accepted_len is None:
        out_accepted_len = torch.empty(B, dtype=torch.int32, device=dev)
    if out_status is None:
        out_status = torch.empty(B, dtype=torch.int32, device=dev)
    if workspace is None:
        workspace = torch.empty(max(1, resispec_tree_group_workspace_bytes(B, N)),
                                dtype=torch.uint8, device=dev)
    _shape(out_tokens, (B, max_depth + 1), "out_tokens")
    _shape(out_accepted_len, (B,), "out_accepted_len")
    _shape(out_status, (B,), "out_status")
    prm = _params(target_logits, temperature, mode, without_replacement, bonus)
    st = lib.resispec_verify_tree_group(
        _dev(target_logits, target_logits.dtype, "target_logits"),
        _dev(draft_logits, target_logits.dtype, "draft_logits"),
        _dev(node_token, torch.int32, "node_token"), _dev(parent, torch.int32, "parent"),
        _dev(u_accept, torch.float32, "u_accept"), _dev(u_resample, torch.float32, "u_resample"),
        B, N, V, int(max_depth), ctypes.byref(prm),
        _dev(out_tokens, torch.int32, "out_tokens"),
        _dev(out_accepted_len, torch.int32, "out_accepted_len"),
        _dev(out_status, torch.int32, "out_status"), int(group_size),
        _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(stream))
    _check(st)
    return out_tokens, out_accepted_len, out_status


def resispec_debug_set_group_waits(barrier=None, formation=None) -> None:
    """Testing hook: time limits of row groups in later launches (ticks of the 100 MHz
    device clock): `barrier` for every wait of a formed group for its members' slot
    totals, `formation` for its workgroups to start.  None restores a default (20 ms,
    20 us)."""
    none = (1 << 64) - 1
    _check(lib.resispec_debug_set_group_waits(
        ctypes.c_uint64(none if barrier is None else int(barrier)),
        ctypes.c_uint64(none if formation is None else int(formation))))


def resispec_debug_pool_held() -> int:
    """Testing hook: group states of the library's pool in use, and workgroups counted, on the
    current device, after a synchronisation; 0 unless something went wrong."""
    n = lib.resispec_debug_pool_held()
    if n < 0:
        raise RuntimeError("the pool of group states cannot be read")
    return n


def resispec_debug_fail_pool_launches(n: int) -> None:
    """Testing hook: the next n launches of the pool's groups count as failed."""
    _check(lib.resispec_debug_fail_pool_launches(int(n)))


def resispec_verify_tree_path_group(target_logits, draft_logits, node_token, parent, u_accept,
                                    u_resample, *, temperature, max_depth, mode="resispec",
                                    without_replacement=False, bonus=True, group_size=0,
                                    workspace=None, out_tokens=None, out_accepted_len=None,
                                    out_status=None, stream=None):
    """Path-only schedule with row groups (group_size workgroups per sequence, 0 =
    automatic); same results as resispec_verify_tree_path.  Returns (tokens [B,
    max_depth+1], accepted_len [B], status [B])."""
    import torch
    B, N, V = _tree_common(target_logits, draft_logits, node_token, parent, u_accept, u_resample,
                           max_depth)
    dev = target_logits.device
    if out_tokens is None:
        out_tokens = torch.empty((B, max_depth + 1), dtype=torch.int32, device=dev)
    if out_accepted_len is None:
        out_accepted_len = torch.empty(B, dtype=torch.int32, device=dev)
    if out_status is None:
        out_status = torch.empty(B, dtype=torch.int32, device=dev)
    if workspace is None:
        workspace = torch.empty(max(1, resispec_path_workspace_bytes(B, V)), dtype=torch.uint8,
                                device=dev)
    _shape(out_tokens, (B, max_depth + 1), "out_tokens")
    _shape(out_accepted_len, (B,), "out_accepted_len")
    _shape(out_status, (B,), "out_status")
    prm = _params(target_logits, temperature, mode, without_replacement, bonus)
    st = lib.resispec_verify_tree_path_group(
        _dev(target_logits, target_logits.dtype, "target_logits"),
        _dev(draft_logits, target_logits.dtype, "draft_logits"),
        _dev(node_token, torch.int32, "node_token"), _dev(parent, torch.int32, "parent"),
        _dev(u_accept, torch.float32, "u_accept"), _dev(u_resample, torch.float32, "u_resample"),
        B, N, V, int(max_depth), ctypes.byref(prm),
        _dev(out_tokens, torch.int32, "out_tokens"),
        _dev(out_accepted_len, torch.int32, "out_accepted_len"),
        _dev(out_status, torch.int32, "out_status"), int(group_size),
        _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(stream))
    _check(st)
    return out_tokens, out_accepted_len, out_status


def resispec_draft_candidates(draft_logits, parent, *, temperature, without_replacement=False,
                              seed=0, offset=0, node_token=None, u_accept=None, u_resample=None,
                              out_status=None, stream=None):
    """The draft step on the device: children's candidate tokens drawn from each node's
    draft row, and every node's uniforms (Philox4x32-10 under seed / offset).
    Returns (node_token [B, N], u_accept [B, N], u_resample [B, N], status [B])."""
    import torch
    if draft_logits.dim() != 3:
        raise ValueError("draft_logits must be [B, N, V]")
    B, N, V = draft_logits.shape
    _shape(parent, (B, N), "parent")
    dev = draft_logits.device
    _same_device(draft_logits, parent, node_token, u_accept, u_resample, out_status)
    if node_token is None:
        node_token = torch.empty((B, N), dtype=torch.int32, device=dev)
    if u_accept is None:
        u_accept = torch.empty((B, N), dtype=torch.float32, device=dev)
    if u_resample is None:
        u_resample = torch.empty((B, N), dtype=torch.float32, device=dev)
    if out_status is None:
        out_status = torch.empty(B, dtype=torch.int32, device=dev)
    for t, nm in ((node_token, "node_token"), (u_accept, "u_accept"), (u_resample, "u_resample")):
        _shape(t, (B, N), nm)
    _shape(out_status, (B,), "out_status")
    prm = _params(draft_logits, temperature, "resispec", without_replacement, False)
    st = lib.resispec_draft_candidates(
        _dev(draft_logits, draft_logits.dtype, "draft_logits"), _dev(parent, torch.int32, "parent"),
        B, N, V, ctypes.byref(prm), int(seed) & 0xFFFFFFFFFFFFFFFF, int(offset) & 0xFFFFFFFFFFFFFFFF,
        _dev(node_token, torch.int32, "node_token"), _dev(u_accept, torch.float32, "u_accept"),
        _dev(u_resample, torch.float32, "u_resample"), _dev(out_status, torch.int32, "out_status"),
        _stream(stream))
    _check(st)
    return node_token, u_accept, u_resample, out_status


def resispec_deferred_workspace_bytes(B: int, N: int) -> int:
    return lib.resispec_deferred_workspace_bytes(int(B), int(N))


def _logit_args(target_logits, draft_logits, node_token, parent, u_accept, u_resample):
    import torch
    return (_dev(target_logits, target_logits.dtype, "target_logits"),
            _dev(draft_logits, target_logits.dtype, "draft_logits"),
            _dev(node_token, torch.int32, "node_token"), _dev(parent, torch.int32, "parent"),
            _dev(u_accept, torch.float32, "u_accept"), _dev(u_resample, torch.float32, "u_resample"))


def _tree_outputs(B, max_depth, dev, out_tokens, out_accepted_len, out_status):
    import torch
    if out_tokens is None:
        out_tokens = torch.empty((B, max_depth + 1), dtype=torch.int32, device=dev)
    if out_accepted_len is None:
        out_accepted_len = torch.empty(B, dtype=torch.int32, device=dev)
    if out_status is None:
        out_status = torch.empty(B, dtype=torch.int32, device=dev)
    _shape(out_tokens, (B, max_depth + 1), "out_tokens")
    _shape(out_accepted_len, (B,), "out_accepted_len")
    _shape(out_status, (B,), "out_status")
    return out_tokens, out_accepted_len, out_status


def resispec_verify_tree_deferred(target_logits, draft_logits, node_token, parent, u_accept,
                                  u_resample, *, temperature, max_depth, mode="resispec",
                                  without_replacement=False, bonus=True, out_tokens=None,
                                  out_accepted_len=None, out_status=None, workspace=None,
                                  stream=None):
    """resispec_verify_tree with deferred draws (a row's draw made only where a walk ends);
    returns (tokens [B, max_depth+1], accepted_len [B], status [B])."""
    import torch
    B, N, V = _tree_common(target_logits, draft_logits, node_token, parent, u_accept, u_resample,
                           max_depth)
    dev = target_logits.device
    out_tokens, out_accepted_len, out_status = _tree_outputs(B, max_depth, dev, out_tokens,
                                                             out_accepted_len, out_status)
    if workspace is None:
        workspace = torch.empty(max(resispec_deferred_workspace_bytes(B, N), 1),
                                dtype=torch.uint8, device=dev)
    prm = _params(target_logits, temperature, mode, without_replacement, bonus)
    st = lib.resispec_verify_tree_deferred(
        *_logit_args(target_logits, draft_logits, node_token, parent, u_accept, u_resample),
        B, N, V, int(max_depth), ctypes.byref(prm),
        _dev(out_tokens, torch.int32, "out_tokens"),
        _dev(out_accepted_len, torch.int32, "out_accepted_len"),
        _dev(out_status, torch.int32, "out_status"),
        _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(stream))
    _check(st)
    return out_tokens, out_accepted_len, out_status


def resispec_decide_nodes(target_logits, draft_logits, node_token, parent, u_accept, u_resample,
                          workspace, *, temperature, mode="resispec", without_replacement=False,
                          bonus=True, stream=None):
    """First launch of resispec_verify_tree_deferred: every node's tests into `workspace`
    (resispec_deferred_workspace_bytes), draws deferred where they can be."""
    import torch
    B, N, V = _check_tree_shapes(target_logits, draft_logits, node_token, parent, u_accept,
                                 u_resample)
    prm = _params(target_logits, temperature, mode, without_replacement, bonus)
    st = lib.resispec_decide_nodes(
        *_logit_args(target_logits, draft_logits, node_token, parent, u_accept, u_resample),
        B, N, V, ctypes.byref(prm), _dev(workspace, torch.uint8, "workspace"), workspace.numel(),
        _stream(stream))
    _check(st)


def resispec_walk_draw(target_logits, draft_logits, node_token, parent, u_accept, u_resample,
                       workspace, *, temperature, max_depth, mode="resispec",
                       without_replacement=False, bonus=True, out_tokens=None,
                       out_accepted_len=None, out_status=None, stream=None):
    """Second launch of resispec_verify_tree_deferred: the walks, with the deferred draw
    where a walk ends; returns (tokens, accepted_len, status)."""
    import torch
    B, N, V = _tree_common(target_logits, draft_logits, node_token, parent, u_accept, u_resample,
                           max_depth)
    out_tokens, out_accepted_len, out_status = _tree_outputs(B, max_depth, target_logits.device,
                                                             out_tokens, out_accepted_len,
                                                             out_status)
    prm = _params(target_logits, temperature, mode, without_replacement, bonus)
    st = lib.resispec_walk_draw(
        *_logit_args(target_logits, draft_logits, node_token, parent, u_accept, u_resample),
        B, N, V, int(max_depth), ctypes.byref(prm), _dev(workspace, torch.uint8, "workspace"),
        workspace.numel(), _dev(out_tokens, torch.int32, "out_tokens"),
        _dev(out_accepted_len, torch.int32, "out_accepted_len"),
        _dev(out_status, torch.int32, "out_status"), _stream(stream))
    _check(st)
    return out_tokens, out_accepted_len, out_status


def resispec_verify_nodes(target_logits, draft_logits, node_token, parent, u_accept, u_resample,
                          workspace, *, temperature, mode="resispec", without_replacement=False,
                          bonus=True, stream=None):
    """First stage of resispec_verify_tree: every node's outcome into `workspace`."""
    import torch
    B, N, V = _check_tree_shapes(target_logits, draft_logits, node_token, parent, u_accept,
                                 u_resample)
    prm = _params(target_logits, temperature, mode, without_replacement, bonus)
    st = lib.resispec_verify_nodes(
        _dev(target_logits, target_logits.dtype, "target_logits"),
        _dev(draft_logits, target_logits.dtype, "draft_logits"),
        _dev(node_token, torch.int32, "node_token"), _dev(parent, torch.int32, "parent"),
        _dev(u_accept, torch.float32, "u_accept"), _dev(u_resample, torch.float32, "u_resample"),
        B, N, V, ctypes.byref(prm), _dev(workspace, torch.uint8, "workspace"), workspace.numel(),
        _stream(stream))
    _check(st)


def resispec_walk(node_token, workspace, out_tokens, out_accepted_len, out_status=None, *,
                  max_depth, stream=None):
    """Second stage of resispec_verify_tree: walk every root over the node outcomes."""
    import torch
    B, N = node_token.shape
    _shape(out_tokens, (B, int(max_depth) + 1), "out_tokens")
    _shape(out_accepted_len, (B,), "out_accepted_len")
    if out_status is not None:
        _shape(out_status, (B,), "out_status")
    st = lib.resispec_walk(
        _dev(node_token, torch.int32, "node_token"), B, N, int(max_depth),
        _dev(workspace, torch.uint8, "workspace"), workspace.numel(),
        _dev(out_tokens, torch.int32, "out_tokens"),
        _dev(out_accepted_len, torch.int32, "out_accepted_len"),
        _dev(out_status, torch.int32, "out_status") if out_status is not None else None,
        _stream(stream))
    _check(st)


def resispec_node_outcomes(workspace, B: int, N: int, *, stream=None):
    """Every node's outcome left in `workspace` by resispec_verify_nodes, or by
    resispec_decide_nodes (and resispec_walk_draw, which fills in the nodes it draws for;
    the others report RS_SEQ_DEFERRED): (node_child, node_token, node_status), [B, N]
    int32 each."""
    import torch
    dev = workspace.device
    out = [torch.empty((B, N), dtype=torch.int32, device=dev) for _ in range(3)]
    st = lib.resispec_node_outcomes(_dev(workspace, torch.uint8, "workspace"), workspace.numel(),
                                    int(B), int(N), *[o.data_ptr() for o in out], _stream(stream))
    _check(st)
    return tuple(out)


def resispec_verify_tree_debug(target_logits, draft_logits, node_token, parent, u_accept,
                               u_resample, *, temperature, max_depth, mode="resispec",
                               without_replacement=False, bonus=True, want_residual=False,
                               stream=None):
    """Tree verify that also returns every node's outcome (and optionally the normalised
    distribution each drawing node sampled from)."""
    import torch
    B, N, V = _tree_common(target_logits, draft_logits, node_token, parent, u_accept, u_resample,
                           max_depth)
    dev = target_logits.device
    out_tokens = torch.empty((B, max_depth + 1), dtype=torch.int32, device=dev)
    out_len = torch.empty(B, dtype=torch.int32, device=dev)
    out_status = torch.empty(B, dtype=torch.int32, device=dev)
    node_child = torch.empty((B, N), dtype=torch.int32, device=dev)
    node_tok = torch.empty((B, N), dtype=torch.int32, device=dev)
    node_status = torch.empty((B, N), dtype=torch.int32, device=dev)
    resid = torch.empty((B, N, V), dtype=torch.float32, device=dev) if want_residual else None
    prm = _params(target_logits, temperature, mode, without_replacement, bonus)
    st = lib.resispec_verify_tree_debug(
        _dev(target_logits, target_logits.dtype, "target_logits"),
        _dev(draft_logits, target_logits.dtype, "draft_logits"),
        _dev(node_token, torch.int32, "node_token"), _dev(parent, torch.int32, "parent"),
        _dev(u_accept, torch.float32, "u_accept"), _dev(u_resample, torch.float32, "u_resample"),
        B, N, V, int(max_depth), ctypes.byref(prm), out_tokens.data_ptr(), out_len.data_ptr(),
        out_status.data_ptr(), None, 0, node_child.data_ptr(), node_tok.data_ptr(),
        node_status.data_ptr(), resid.data_ptr() if resid is not None else None, _stream(stream))
    _check(st)
    return {"tokens": out_tokens, "accepted_len": out_len, "status": out_status,
            "node_child": node_child, "node_token": node_tok, "node_status": node_status,
            "residual": resid}


# ----------------------------------------------------------------- sampling --

def _rows(t, name):
    """Rows of a [R, V] or [B, N, V] tensor whose rows lie one stride apart: (pointer,
    stride, leading shape, R, V)."""
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError("%s must be a device tensor" % name)
    if t.dtype is not torch.float32 and t.dtype is not torch.bfloat16:
        raise TypeError("%s must be float32 or bfloat16" % name)
    shape, stride = t.shape, t.stride()
    if len(shape) == 2:
        R, step = shape[0], stride[0]
    elif len(shape) == 3:
        R, step = shape[0] * shape[1], stride[1] if shape[1] > 1 else stride[0]
        if shape[0] > 1 and shape[1] > 1 and stride[0] != shape[1] * stride[1]:
            raise ValueError("%s: all rows must lie one stride apart" % name)
    else:
        raise ValueError("%s must be [R, V] or [B, N, V]" % name)
    V = shape[-1]
    if stride[-1] != 1 and V > 1:
        raise ValueError("%s: the elements of a row must be adjacent" % name)
    if R < 2:
        step = V
    elif step < V:
        raise ValueError("%s: rows must not overlap" % name)
    return t.data_ptr(), step, shape[:-1], R, V


def _overlap(a, a_step, b, b_step, R, V, size):
    """Whether R rows of V elements of `size` bytes at a and b, one step apart, may share
    memory.  Rows of one step can lie between each other (two halves of each row of a
    tensor); of different steps, their whole ranges must be apart."""
    if R == 0 or a + ((R - 1) * a_step + V) * size <= b or b + ((R - 1) * b_step + V) * size <= a:
        return False
    return a_step != b_step or not V * size <= (b - a) % (a_step * size) <= (a_step - V) * size


def _settings(logits, lead, R, temperature, top_k, top_p, min_p):
    """rs_filter of settings that are numbers, or device tensors with an entry a row ([R] or
    [B, N]) or a sequence ([B])."""
    import torch
    f = RsFilter(RS_BF16 if logits.dtype is torch.bfloat16 else RS_F32, 1, 1.0, 0, 1.0, 0.0)
    shape = None
    for v, number, dtype in ((temperature, "temperature", torch.float32), (top_k, "top_k", torch.int32),
                             (top_p, "top_p", torch.float32), (min_p, "min_p", torch.float32)):
        if not isinstance(v, torch.Tensor):
            if number == "top_k" and not -1 << 31 <= v < 1 << 31:   # ctypes would keep its low 32 bits
                raise ValueError("top_k must fit an int32, got %d" % v)
            setattr(f, number, v)
            continue
        if shape is None:
            shape = v.shape
            if shape != lead and shape != lead[:1]:
                raise ValueError("%s has shape %s, expected %s or %s" % (number, tuple(shape), tuple(lead),
                                                                        tuple(lead[:1])))
            f.rows_per_entry = max(1, R // max(1, v.numel()))
        setattr(f, number + "s", _given(v, shape, dtype, logits, number))
    return f


def _given(t, shape, dtype, logits, name):
    """The address of a contiguous tensor on the rows' device."""
    # the usual case, in the fewest looks
    try:
        if (t.dtype is dtype and t.shape == shape and t.get_device() == logits.get_device() >= 0 and
                t.is_contiguous()):
            return t.data_ptr()
    except AttributeError:
        pass
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError("%s must be a device tensor" % name)
    if t.dtype is not dtype:
        raise TypeError("%s must be %s" % (name, dtype))
    if t.shape != shape:
        raise ValueError("%s has shape %s, expected %s" % (name, tuple(t.shape), tuple(shape)))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if t.get_device() != logits.get_device():
        raise ValueError("all tensors must be on one device, got %s" % {t.device, logits.device})
    return t.data_ptr()


def _row_call(logits, stream, call):
    """call(stream handle) with the rows' device current, and `stream`, if given, the one that
    the tensors allocated in it belong to."""
    if stream is None:
        device, raw = _runtime()
        d = logits.get_device()
        if device() == d:
            return call(raw(d))
    import torch
    if stream is None:
        with torch.cuda.device(logits.device):
            return call(_stream(None))
    if stream.device != logits.device:
        raise ValueError("the stream is on %s, the tensors on %s" % (stream.device, logits.device))
    with torch.cuda.stream(stream):
        return call(_stream(stream))


def _handle(like, stream):
    """The current stream's handle where the tensors' device is the current one and no stream is
    given, the usual case; else None, and the call is to be made again by _elsewhere."""
    if stream is None:
        device, raw = _runtime()
        d = like.get_device()
        if device() == d:
            return raw(d)
    return None


def _elsewhere(like, stream, call, *args, **kw):
    """call(*args, **kw) with the tensors' device, and `stream` if given, the current ones."""
    import torch
    if not like.is_cuda:
        raise ValueError("device tensors are required, got %s" % like.device)
    if stream is None:
        with torch.cuda.device(like.device):
            return call(*args, **kw)
    if stream.device != like.device:
        raise ValueError("the stream is on %s, the tensors on %s" % (stream.device, like.device))
    with torch.cuda.stream(stream):
        return call(*args, **kw)


def resispec_sample(logits, u, *, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, out_token=None,
                    out_logprob=None, out_kept=None, out_status=None, stream=None):
    """Draws from rows of logits under temperature, top-k, top-p and min-p, one for each of the
    k uniforms of a row.

    logits: [R, V] or [B, N, V], the rows one stride apart (padding between them is not
    read); u: fp32, the leading shape and k.  Each setting is a number, or a device tensor
    with an entry a row or a sequence (fp32; top_k int32).  top_k 0, top_p 1 and min_p 0 are
    off; top_k 1 is the likeliest token.  Returns (token and log-probability, shaped as u;
    number of elements kept and status, the leading shape)."""
    import torch
    ptr, step, lead, R, V = _rows(logits, "logits")
    if u.dim() != len(lead) + 1 or u.shape[:-1] != lead:
        raise ValueError("u has shape %s, expected %s and the number of draws" % (tuple(u.shape), tuple(lead)))
    shape, dev = u.shape, logits.device
    f = _settings(logits, lead, R, temperature, top_k, top_p, min_p)
    up = _given(u, shape, torch.float32, logits, "u")

    def call(handle):
        tok = torch.empty(shape, dtype=torch.int32, device=dev) if out_token is None else out_token
        lp = torch.empty(shape, dtype=torch.float32, device=dev) if out_logprob is None else out_logprob
        kept = torch.empty(lead, dtype=torch.int32, device=dev) if out_kept is None else out_kept
        st = torch.empty(lead, dtype=torch.int32, device=dev) if out_status is None else out_status
        _check(lib.resispec_sample(ptr, step, up, R, V, shape[-1], ctypes.byref(f),
                                   _given(tok, shape, torch.int32, logits, "out_token"),
                                   _given(lp, shape, torch.float32, logits, "out_logprob"),
                                   _given(kept, lead, torch.int32, logits, "out_kept"),
                                   _given(st, lead, torch.int32, logits, "out_status"), handle))
        return tok, lp, kept, st
    return _row_call(logits, stream, call)


def resispec_filter_logits(logits, *, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, out=None,
                           out_kept=None, out_status=None, stream=None):
    """Rows of logits with -inf outside what their settings (as resispec_sample) keep: target
    and draft rows for the draft step and the verification.  `out` may be `logits` itself.
    Returns (out, number of elements kept, status)."""
    import torch
    ptr, step, lead, R, V = _rows(logits, "logits")
    dev = logits.device
    f = _settings(logits, lead, R, temperature, top_k, top_p, min_p)

    def call(handle):
        y = torch.empty(logits.shape, dtype=logits.dtype, device=dev) if out is None else out
        to, to_step, _, _, _ = _rows(y, "out")
        _shape(y, logits.shape, "out")
        if y.dtype is not logits.dtype:
            raise TypeError("out must be %s" % logits.dtype)
        if y.get_device() != logits.get_device():
            raise ValueError("all tensors must be on one device, got %s" % {y.device, dev})
        if not (to == ptr and to_step == step) and _overlap(ptr, step, to, to_step, R, V, logits.element_size()):
            raise ValueError("out must not overlap logits, unless it is the same rows")
        kept = torch.empty(lead, dtype=torch.int32, device=dev) if out_kept is None else out_kept
        st = torch.empty(lead, dtype=torch.int32, device=dev) if out_status is None else out_status
        _check(lib.resispec_filter_logits(ptr, step, R, V, ctypes.byref(f), to, to_step,
                                          _given(kept, lead, torch.int32, logits, "out_kept"),
                                          _given(st, lead, torch.int32, logits, "out_status"), handle))
        return y, kept, st
    return _row_call(logits, stream, call)


def resispec_token_logprobs(logits, tokens, *, temperature=1.0, out_logprob=None, out_rank=None,
                            out_status=None, stream=None):
    """Log-probabilities, under the temperature softmax of their rows, and ranks of given
    tokens (int32, the leading shape of `logits` and k; -1 = no token, which gives 0 and 0).
    Returns (log-probability, rank, status)."""
    import torch
    ptr, step, lead, R, V = _rows(logits, "logits")
    if tokens.dim() != len(lead) + 1 or tokens.shape[:-1] != lead:
        raise ValueError("tokens has shape %s, expected %s and the number of tokens" %
                         (tuple(tokens.shape), tuple(lead)))
    shape, dev = tokens.shape, logits.device
    f = _settings(logits, lead, R, temperature, 0, 1.0, 0.0)
    ids = _given(tokens, shape, torch.int32, logits, "tokens")

    def call(handle):
        lp = torch.empty(shape, dtype=torch.float32, device=dev) if out_logprob is None else out_logprob
        rank = torch.empty(shape, dtype=torch.int32, device=dev) if out_rank is None else out_rank
        st = torch.empty(lead, dtype=torch.int32, device=dev) if out_status is None else out_status
        _check(lib.resispec_token_logprobs(ptr, step, ids, R, V, shape[-1], ctypes.byref(f),
                                           _given(lp, shape, torch.float32, logits, "out_logprob"),
                                           _given(rank, shape, torch.int32, logits, "out_rank"),
                                           _given(st, lead, torch.int32, logits, "out_status"), handle))
        return lp, rank, st
    return _row_call(logits, stream, call)


# ------------------------------------------------------------------- beams --

def resispec_beam_workspace_bytes(B: int, W: int, V: int) -> int:
    return lib.resispec_beam_workspace_bytes(int(B), int(W), int(V))


def _device(t, name):
    """The number of a tensor's device."""
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError("%s must be a device tensor" % name)
    return t.get_device()


def _at(t, shape, dtype, d, like, name):
    """_given, with the device's number looked up once for a call's tensors."""
    try:
        if t.dtype is dtype and t.shape == shape and t.get_device() == d and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        pass
    return _given(t, shape, dtype, like, name)


def _int32(v, name):
    """A whole number that ctypes will not cut to its low 32 bits."""
    v = int(v)
    if not -1 << 31 <= v < 1 << 31:
        raise ValueError("%s must fit an int32, got %d" % (name, v))
    return v


def resispec_beam_select(logits, scores, *, k=None, temperature=1.0, ended=None, end_token=-1, out_parent=None,
                         out_token=None, out_score=None, out_status=None, workspace=None, stream=None):
    """The k best continuations (default: as many as beams) of each sequence's beams.

    logits: [B, W, V] or [B * W, V], the rows one stride apart; scores: [B, W] fp32, the beams'
    log-probabilities so far, -inf where there is no beam; ended: [B, W] uint8 or bool, beams
    that go on with `end_token` alone, at their score; temperature: a number, or a device
    tensor with an entry a row or a sequence.  Returns (parent beam, token, score, each [B, k],
    best first; status [B])."""
    import torch
    ptr, step, lead, R, V = _rows(logits, "logits")
    if not isinstance(scores, torch.Tensor) or scores.dim() != 2:
        raise ValueError("scores must be a [B, W] tensor")
    shape = scores.shape
    B, W = shape
    if R != B * W or (len(lead) == 2 and lead != shape):
        raise ValueError("logits has rows %s, expected %s" % (tuple(lead), tuple(shape)))
    d = logits.get_device()
    k = W if k is None else _int32(k, "k")
    end_token = _int32(end_token, "end_token")
    if isinstance(temperature, torch.Tensor):
        f = _settings(logits, shape, R, temperature, 0, 1.0, 0.0)
        at = ctypes.addressof(f)
    else:
        f, at = _number_settings(logits.dtype is torch.bfloat16, float(temperature))
    sp = _at(scores, shape, torch.float32, d, logits, "scores")
    ep = None
    if ended is not None:
        if not isinstance(ended, torch.Tensor):
            raise ValueError("ended must be a device tensor")
        ep = _at(ended, shape, torch.bool if ended.dtype is torch.bool else torch.uint8, d, logits, "ended")
    handle = _handle(logits, stream)
    if handle is None:
        return _elsewhere(logits, stream, resispec_beam_select, logits, scores, k=k, temperature=temperature, ended=ended,
                          end_token=end_token, out_parent=out_parent, out_token=out_token, out_score=out_score,
                          out_status=out_status, workspace=workspace)
    i32, to = torch.int32, (B, k)
    if out_parent is None:
        out_parent = torch.empty(to, dtype=i32, device=logits.device)
    if out_token is None:
        out_token = torch.empty(to, dtype=i32, device=logits.device)
    if out_score is None:
        out_score = torch.empty(to, dtype=torch.float32, device=logits.device)
    if out_status is None:
        out_status = torch.empty(B, dtype=i32, device=logits.device)
    if workspace is None:
        workspace = torch.empty(max(1, lib.resispec_beam_workspace_bytes(B, W, V)), dtype=torch.uint8, device=logits.device)
    _check(lib.resispec_beam_select(ptr, step, sp, ep, end_token, B, W, V, k, at,
                                    _at(out_parent, to, i32, d, logits, "out_parent"),
                                    _at(out_token, to, i32, d, logits, "out_token"),
                                    _at(out_score, to, torch.float32, d, logits, "out_score"),
                                    _at(out_status, (B,), i32, d, logits, "out_status"),
                                    _at(workspace, workspace.shape, torch.uint8, d, logits, "workspace"),
                                    workspace.numel(), handle))
    return out_parent, out_token, out_score, out_status


@functools.lru_cache(maxsize=256)
def _number_settings(bf16, temperature):
    f = RsFilter(RS_BF16 if bf16 else RS_F32, 1, temperature, 0, 1.0, 0.0)
    return f, ctypes.addressof(f)


@functools.lru_cache(maxsize=1024)
def _layout(shape, stride, size, page_dim, position_dim, name):
    """(rs_rows, bytes from the first to past the last, its address) of rows in a tensor: the dimensions
    before page_dim are outer, those between it and position_dim inner, those after
    position_dim (without one: after page_dim) the row, which has to lie together."""
    def place(d, what):
        if not -len(shape) <= d < len(shape):
            raise ValueError("%s of %s is %d, of %d dimensions" % (what, name, d, len(shape)))
        return d % len(shape)

    def joined(dims, what):
        n, step = 1, 0
        for d in reversed(dims):
            if shape[d] == 1:
                continue
            if n == 1:
                step = stride[d]
            elif stride[d] != n * step:
                raise ValueError("%s: its %s dimensions must lie one stride apart" % (name, what))
            n *= shape[d]
        return n, step

    page_dim = place(page_dim, "page_dim")
    if min(shape) < 1:
        raise ValueError("%s has shape %s" % (name, shape))
    dims = range(len(shape))
    if position_dim is None:
        at, inner, positions = page_dim, (1, 0), (1, 0)
    else:
        at = place(position_dim, "position_dim")
        if at <= page_dim:
            raise ValueError("%s: the positions must come after the pages or beams" % name)
        inner, positions = joined(dims[page_dim + 1:at], "inner"), joined(dims[at:at + 1], "position")
    outer, pages = joined(dims[:page_dim], "outer"), joined(dims[page_dim:page_dim + 1], "page")
    row, step = joined(dims[at + 1:], "row")
    if row > 1 and step != 1:
        raise ValueError("%s: the elements of a row must be adjacent" % name)
    span = row
    for n, d in sorted((x for x in (outer, pages, inner, positions) if x[0] > 1), key=lambda x: x[1]):
        if d < span:
            raise ValueError("%s: rows must not overlap" % name)
        span += (n - 1) * d
    r = RsRows(outer[0], pages[0], inner[0], positions[0], row * size,
               *(d * size for _, d in (outer, pages, inner, positions)))
    return r, span * size, ctypes.addressof(r)


def _row_layout(t, page_dim, position_dim, name):
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError("%s must be a device tensor" % name)
    return _layout(t.shape, t.stride(), t.element_size(), page_dim, position_dim, name)


def _table(t, rows, like, name):
    """(address, entries from row to row, entries a row) of a block table."""
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError("%s must be a device tensor" % name)
    if t.dtype is not torch.int32:
        raise TypeError("%s must be torch.int32" % name)
    if t.dim() != 2 or t.shape[0] != rows or t.shape[1] < 1:
        raise ValueError("%s has shape %s, expected %d rows" % (name, tuple(t.shape), rows))
    step, n = t.stride(0) if rows > 1 else t.shape[1], t.shape[1]
    if (n > 1 and t.stride(1) != 1) or step < n:
        raise ValueError("%s: the entries of a row must be adjacent, and rows must not overlap" % name)
    if t.get_device() != like.get_device():
        raise ValueError("all tensors must be on one device, got %s" % {t.device, like.device})
    return t.data_ptr(), step, n


@functools.lru_cache(maxsize=1024)
def _interleaved(a, b, between):
    """Whether rows with layouts a and b (bytes of rs_rows) share none, b's first `between` bytes
    after a's, by one step that both repeat: halves of a buffer, every other beam, the two ends
    of rows.  Of steps that are multiples of it only the rest counts."""
    a, b = RsRows.from_buffer_copy(a), RsRows.from_buffer_copy(b)
    steps = [[(n, step) for n, step in ((r.outer, r.outer_stride), (r.pages, r.page_stride), (r.inner, r.inner_stride),
                                        (r.positions, r.position_stride)) if n > 1] for r in (a, b)]
    for whole in {step for x in steps for _, step in x}:
        wide = [r.row_bytes + sum((n - 1) * step for n, step in x if step % whole) for r, x in zip((a, b), steps)]
        if wide[0] <= between % whole <= whole - wide[1]:
            return True
    return False


def _moved_to(src, rows, dst, name, *dims):
    """Where rows go: (address, layout as _layout gives it).  The same rows, or apart from them."""
    if dst is None or dst is src:
        return src.data_ptr(), rows
    to = _row_layout(dst, *dims, name)
    if dst.dtype is not src.dtype:
        raise TypeError("%s must be %s" % (name, src.dtype))
    if dst.get_device() != src.get_device():
        raise ValueError("all tensors must be on one device, got %s" % {dst.device, src.device})
    a, b = src.data_ptr(), dst.data_ptr()
    if a < b + to[1] and b < a + rows[1]:
        x, y = bytes(rows[0]), bytes(to[0])
        if not (a == b and x == y) and not _interleaved(x, y, b - a):
            raise ValueError("%s must be apart from the rows it is taken from, or the same rows" % name)
    return b, to


def _chosen(parent, rows):
    """(B, K) of parent beams, and whether there is nothing to move."""
    import torch
    if not isinstance(parent, torch.Tensor) or parent.dim() != 2:
        raise ValueError("parent must be a [B, K] tensor")
    B, K = parent.shape
    return B, K, B == 0 and parent.is_cuda and rows.is_cuda


def _empty(status, like):
    import torch
    return torch.empty(0, dtype=torch.int32, device=like.device) if status is None else status


def _per_sequence(n, B, name):
    """How many of n beams each of B sequences has."""
    if n % B or n < B:
        raise ValueError("%s has %d beams, parent %d sequences" % (name, n, B))
    return n // B


def resispec_beam_reorder(state, parent, *, beam_dim=0, position_dim=None, lengths=None, out=None, out_status=None,
                          stream=None):
    """The states of the chosen beams: beam k of sequence b becomes beam parent[b, k] (int32 [B,
    K]; -1: stays as it is).  state: any tensor with B * W beams along beam_dim; out: the same
    with B * K, or None for a move in place (K = W).  Its rows may lie between the state's, as
    halves of one buffer do, if both repeat in one step.  lengths (int32 [B], with position_dim):
    only so many positions are moved; where whole states move leave position_dim out, so that
    what lies together moves in one run.  Returns (out, status)."""
    import torch
    B, K, none = _chosen(parent, state)
    if none:
        return (state if out is None else out), _empty(out_status, parent)
    src = _row_layout(state, beam_dim, position_dim, "state")
    d = state.get_device()
    W = _per_sequence(src[0].pages, B, "state")
    pp = _at(parent, parent.shape, torch.int32, d, state, "parent")
    if lengths is not None and position_dim is None:
        raise ValueError("lengths need position_dim")
    if out is None and K != W:
        raise ValueError("a move in place needs as many beams as there are, %d, got %d" % (W, K))
    to, dst = _moved_to(state, src, out, "out", beam_dim, position_dim)
    if dst[0].pages != B * K:
        raise ValueError("out has %d beams, expected %d" % (dst[0].pages, B * K))
    lp = None if lengths is None else _at(lengths, (B,), torch.int32, d, state, "lengths")
    handle = _handle(state, stream)
    if handle is None:
        return _elsewhere(state, stream, resispec_beam_reorder, state, parent, beam_dim=beam_dim, position_dim=position_dim,
                          lengths=lengths, out=out, out_status=out_status)
    if out_status is None:
        out_status = torch.empty(B, dtype=torch.int32, device=state.device)
    _check(lib.resispec_beam_reorder(state.data_ptr(), src[2], to, dst[2], pp, lp, B, W, K,
                                     _at(out_status, (B,), torch.int32, d, state, "out_status"), handle))
    return (state if out is None else out), out_status


def resispec_beam_reorder_paged(cache, block_table, parent, lengths, *, page_dim=0, position_dim=1, out_table=None,
                                out=None, out_status=None, stream=None):
    """resispec_beam_reorder for beams whose positions lie in the pages of a cache: block_table
    is [B * W, pages] int32, lengths [B] int32 positions.  out_table ([B * K, pages]; default:
    block_table, with K = W) says where the chosen beams' positions go, in `out` (default: the
    cache itself; a page may then be in both tables at the same entry of the same sequence).
    Returns (out, status)."""
    import torch
    B, K, none = _chosen(parent, cache)
    if none:
        return (cache if out is None else out), _empty(out_status, parent)
    src = _row_layout(cache, page_dim, position_dim, "cache")
    if not isinstance(block_table, torch.Tensor) or block_table.dim() != 2:
        raise ValueError("block_table must be a [B * W, pages] tensor")
    d = cache.get_device()
    W = _per_sequence(block_table.shape[0], B, "block_table")
    pp = _at(parent, parent.shape, torch.int32, d, cache, "parent")
    tp, tstep, n = _table(block_table, B * W, cache, "block_table")
    if out_table is None:
        if K != W:
            raise ValueError("without out_table there are as many beams as before, %d, got %d" % (W, K))
        op, ostep = tp, tstep
    else:
        op, ostep, on = _table(out_table, B * K, cache, "out_table")
        if on != n:
            raise ValueError("out_table has %d entries a row, block_table %d" % (on, n))
    to, dst = _moved_to(cache, src, out, "out", page_dim, position_dim)
    lp = _at(lengths, (B,), torch.int32, d, cache, "lengths")
    handle = _handle(cache, stream)
    if handle is None:
        return _elsewhere(cache, stream, resispec_beam_reorder_paged, cache, block_table, parent, lengths,
                          page_dim=page_dim, position_dim=position_dim, out_table=out_table, out=out, out_status=out_status)
    if out_status is None:
        out_status = torch.empty(B, dtype=torch.int32, device=cache.device)
    _check(lib.resispec_beam_reorder_paged(cache.data_ptr(), src[2], tp, tstep, to, dst[2], op, ostep, n, pp, lp, B, W, K,
                                           _at(out_status, (B,), torch.int32, d, cache, "out_status"), handle))
    return (cache if out is None else out), out_status


# ------------------------------------------------------------------- cache --

def resispec_plan_cache(kept, added, held, block_table, free_pages, free_count, *, page_size, max_slots=None,
                        out_slots=None, out_positions=None, out_requests=None, out_starts=None, out_held=None,
                        out_free_count=None, out_status=None, stream=None):
    """Pages and slots for a step's new rows.  Request r keeps its first kept[r] positions and
    gets added[r] more; it holds the first held[r] pages of its row of block_table (all int32
    [R]; the table [R, pages]).  free_pages: int32 stack of free page numbers with an entry for
    every page of the cache, the first free_count[0] of them free.  block_table and free_pages
    are brought up to date.  There is room for max_slots new rows (or as out_slots has); out_held
    and out_free_count may be held and free_count.  Returns (slots, positions, requests, each
    [max_slots] with -1 past the last row; starts [R + 1]; held [R]; free_count [1]; status
    [R])."""
    import torch
    if not isinstance(kept, torch.Tensor) or kept.dim() != 1:
        raise ValueError("kept must be a [R] tensor")
    R, like, shape, d = kept.shape[0], kept, kept.shape, _device(kept, "kept")
    kp, ap = _at(kept, shape, torch.int32, d, like, "kept"), _at(added, shape, torch.int32, d, like, "added")
    hp = _at(held, shape, torch.int32, d, like, "held")
    tp, step, n = _table(block_table, R, like, "block_table")
    if not isinstance(free_pages, torch.Tensor) or free_pages.dim() != 1:
        raise ValueError("free_pages must be a [pages] tensor")
    pages = free_pages.shape[0]
    fp = _at(free_pages, (pages,), torch.int32, d, like, "free_pages")
    cp = _at(free_count, (1,), torch.int32, d, like, "free_count")
    if max_slots is None:
        if out_slots is None:
            raise ValueError("max_slots or out_slots is required")
        T = out_slots.shape[0] if out_slots.dim() == 1 else -1
    else:
        T = _int32(max_slots, "max_slots")
    if T < 0:
        raise ValueError("out_slots must be a [T] tensor, max_slots >= 0")
    page_size = _int32(page_size, "page_size")
    handle = _handle(like, stream)
    if handle is None:
        return _elsewhere(like, stream, resispec_plan_cache, kept, added, held, block_table, free_pages, free_count,
                          page_size=page_size, max_slots=T, out_slots=out_slots, out_positions=out_positions,
                          out_requests=out_requests, out_starts=out_starts, out_held=out_held,
                          out_free_count=out_free_count, out_status=out_status)
    i32, dev = torch.int32, kept.device
    if out_slots is None:
        out_slots = torch.empty(T, dtype=i32, device=dev)
    if out_positions is None:
        out_positions = torch.empty(T, dtype=i32, device=dev)
    if out_requests is None:
        out_requests = torch.empty(T, dtype=i32, device=dev)
    if out_starts is None:
        out_starts = torch.empty(R + 1, dtype=i32, device=dev)
    if out_held is None:
        out_held = torch.empty(R, dtype=i32, device=dev)
    if out_free_count is None:
        out_free_count = torch.empty(1, dtype=i32, device=dev)
    if out_status is None:
        out_status = torch.empty(R, dtype=i32, device=dev)
    requests, rows = (R,), (T,)
    _check(lib.resispec_plan_cache(kp, ap, hp, R, page_size, tp, step, n, fp, cp, pages,
                                   _at(out_held, requests, i32, d, like, "out_held"),
                                   _at(out_free_count, (1,), i32, d, like, "out_free_count"),
                                   _at(out_starts, (R + 1,), i32, d, like, "out_starts"), T,
                                   _at(out_slots, rows, i32, d, like, "out_slots"),
                                   _at(out_positions, rows, i32, d, like, "out_positions"),
                                   _at(out_requests, rows, i32, d, like, "out_requests"),
                                   _at(out_status, requests, i32, d, like, "out_status"), handle))
    return out_slots, out_positions, out_requests, out_starts, out_held, out_free_count, out_status


def resispec_accepted_path(parent, node_token, tokens, accepted_len, *, out_path=None, out_status=None, stream=None):
    """The accepted nodes of verified trees: parent and node_token [B, N], and a verification's
    tokens [B, max_depth + 1] and accepted_len [B], all int32.  Returns (path [B, max_depth + 1]:
    the root 0, then the accepted nodes, -1 after the last; status [B])."""
    import torch
    if not isinstance(parent, torch.Tensor) or parent.dim() != 2 or not isinstance(tokens, torch.Tensor) or tokens.dim() != 2:
        raise ValueError("parent must be [B, N], tokens [B, max_depth + 1]")
    B, N = parent.shape
    shape = (B, tokens.shape[1])
    i32, like, d = torch.int32, parent, _device(parent, "parent")
    pp, np_ = _at(parent, (B, N), i32, d, like, "parent"), _at(node_token, (B, N), i32, d, like, "node_token")
    tp, lp = _at(tokens, shape, i32, d, like, "tokens"), _at(accepted_len, (B,), i32, d, like, "accepted_len")
    handle = _handle(like, stream)
    if handle is None:
        return _elsewhere(like, stream, resispec_accepted_path, parent, node_token, tokens, accepted_len, out_path=out_path,
                          out_status=out_status)
    if out_path is None:
        out_path = torch.empty(shape, dtype=i32, device=parent.device)
    if out_status is None:
        out_status = torch.empty(B, dtype=i32, device=parent.device)
    _check(lib.resispec_accepted_path(pp, np_, tp, lp, B, N, shape[1] - 1, _at(out_path, shape, i32, d, like, "out_path"),
                                      _at(out_status, (B,), i32, d, like, "out_status"), handle))
    return out_path, out_status


def resispec_commit_path(cache, slots, path, *, source=None, page_dim=0, position_dim=1, out_status=None, stream=None):
    """The rows of accepted nodes at their places in a paged cache: for every entry path[b, i]
    (int32 [B, depth], ascending, -1 after the last) the node's row goes to slot slots[b, i]
    (int32 [B, N]).  It comes from `source`, laid out as the cache with trees for pages and nodes
    for positions, or, without one, from the node's own slot.  Returns (cache, status)."""
    import torch
    if not isinstance(slots, torch.Tensor) or slots.dim() != 2 or not isinstance(path, torch.Tensor) or path.dim() != 2:
        raise ValueError("slots must be [B, N], path [B, depth]")
    B, N = slots.shape
    rows = _row_layout(cache, page_dim, position_dim, "cache")
    if B == 0 and slots.is_cuda:
        return cache, _empty(out_status, slots)
    i32, d = torch.int32, cache.get_device()
    sp, pp = _at(slots, (B, N), i32, d, cache, "slots"), _at(path, (B, path.shape[1]), i32, d, cache, "path")
    at = rows_of = None
    if source is not None:
        layout, source_span, rows_of = _row_layout(source, page_dim, position_dim, "source")
        at = source.data_ptr()
        if source.dtype is not cache.dtype:
            raise TypeError("source must be %s" % cache.dtype)
        if source.get_device() != cache.get_device():
            raise ValueError("all tensors must be on one device, got %s" % {source.device, cache.device})
        to = cache.data_ptr()
        if at < to + rows[1] and to < at + source_span and not _interleaved(bytes(rows[0]), bytes(layout), at - to):
            raise ValueError("source must be apart from the cache")
        if layout.pages != B or layout.positions != N:
            raise ValueError("source has %d trees of %d nodes, expected %d of %d" % (layout.pages, layout.positions, B, N))
    handle = _handle(cache, stream)
    if handle is None:
        return _elsewhere(cache, stream, resispec_commit_path, cache, slots, path, source=source, page_dim=page_dim,
                          position_dim=position_dim, out_status=out_status)
    if out_status is None:
        out_status = torch.empty(B, dtype=i32, device=cache.device)
    _check(lib.resispec_commit_path(cache.data_ptr(), rows[2], sp, pp, at, rows_of, B, N, path.shape[1],
                                    _at(out_status, (B,), i32, d, cache, "out_status"), handle))
    return cache, out_status
