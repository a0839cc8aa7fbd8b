"""MI355X (gfx950) batch super-tree verification: Python binding of libecho.

The four calls of one verification step live in ``libecho.so`` (HIP kernels
behind a C ABI, declared in ``include/echo.h``).  This module only marshals
arguments: torch device tensors are passed as raw pointers together with the
current HIP stream.  There is no CPU fallback: if the library is missing or
cannot be loaded every call raises.
"""
import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libecho.so")

OK = 0
ERR_INVALID_ARG = -1
ERR_UNSUPPORTED = -2
ERR_WORKSPACE = -3
ERR_HIP = -4

DATA_NAN_LOGQ = 1 << 0
DATA_POS_LOGQ = 1 << 1
DATA_BAD_PARENT = 1 << 2
DATA_TOO_DEEP = 1 << 3
DATA_NOT_CLOSED = 1 << 4
DATA_OVER_CAPACITY = 1 << 5
DATA_BAD_SLOT_PARENT = 1 << 6
DATA_BAD_OFFSETS = 1 << 7
DATA_NO_PAGES = 1 << 8

MAX_DEPTH = 16
MAX_CHECKPOINTS = 16
HEAD_DIM = 128

KV_E4M3 = 0
KV_E5M2 = 1
KV_BLOCK = 32

ROPE_HALF = 0
ROPE_INTERLEAVED = 1
ROPE_MAX_DIM = 1024
ROPE_MAX_ROWS = 16777215
ROPE_SCALINGS = {"plain": 0, "linear": 1, "base": 2, "bands": 3, "smooth": 4}

LATENT_DIM = 512
LATENT_ROPE_DIM = 64

EXPORTS = [
    "echo_gate", "echo_gate_workspace_size", "echo_gate_sparse", "echo_gate_sparse_workspace_size",
    "echo_gate_elastic", "echo_gate_elastic_workspace_size",
    "echo_build_tree_mask", "echo_build_tree_mask_workspace_size",
    "echo_tree_verify_attn", "echo_tree_verify_attn_workspace_size",
    "echo_tree_verify_attn_paged", "echo_accept_logits", "echo_commit_kv",
    "echo_accept", "echo_tree_verify_attn_timed", "echo_tree_verify_attn_paged_timed",
    "echo_probe_stream_read", "echo_gate_noalloc", "echo_verify_step", "echo_status_string",
    "echo_version", "echo_tree_verify_attn_paged_q8",
    "echo_tree_verify_attn_paged_q8_workspace_size", "echo_store_kv_q8", "echo_commit_kv_q8",
    "echo_build_block_tables", "echo_rope", "echo_rope_frequencies", "echo_store_latent",
    "echo_commit_latent", "echo_tree_verify_attn_latent",
    "echo_tree_verify_attn_latent_workspace_size",
]
GATE_SCRATCH_BYTES = 8 << 20

_lib = None
_raw_stream = _device = None  # the current stream's handle, and the current device: set by load()
_int32 = _int64 = _float32 = _float64 = None  # torch's types, and those of 16 bits that hold bf16: too
_bits16 = ()

_P = ctypes.c_void_p
_I32 = ctypes.c_int32
_I64 = ctypes.c_int64
_SZ = ctypes.c_size_t
_F32 = ctypes.c_float
_F64 = ctypes.c_double

_SIGS = {
    "echo_gate": (_I32, [_P, _P, _P, _I32, _I32, _I32, _P, _P, _P, _P, _SZ, _P, _P]),
    "echo_gate_workspace_size": (_SZ, [_I32, _I32, _I32]),
    "echo_gate_noalloc": (_I32, [_P, _P, _P, _I32, _I32, _I32, _P, _P, _P, _P, _P]),
    "echo_gate_sparse": (_I32, [_P, _P, _P, _I32, _I32, _I32, _P, _P, _I32, _P, _P, _P, _P, _P,
                                _SZ, _P, _P]),
    "echo_gate_sparse_workspace_size": (_SZ, [_I32, _I32, _I32]),
    "echo_gate_elastic": (_I32, [_P, _P, _P, _I32, _I32, _I32, _P, _P, _I32, _I32, _I32, _P, _P,
                                 _P, _P, _P, _SZ, _P, _P]),
    "echo_gate_elastic_workspace_size": (_SZ, [_I32, _I32, _I32]),
    "echo_build_tree_mask": (_I32, [_P, _P, _P, _P, _P, _P, _I32, _I32, _I32, _P, _P, _P, _P, _P, _P,
                                    _I32, _P, _SZ, _P, _P]),
    "echo_build_tree_mask_workspace_size": (_SZ, [_I32, _I32, _I32]),
    "echo_tree_verify_attn": (_I32, [_P, _P, _P, _P, _P, _P, _I64, _P, _P, _I32, _I32, _I32, _I32,
                                     _I32, _I32, _F32, _P, _P, _P, _SZ, _P, _P]),
    "echo_tree_verify_attn_workspace_size": (_SZ, [_I32, _I32, _I32, _I32, _I32]),
    "echo_accept": (_I32, [_P, _P, _P, _P, _I32, _I32, _I32, _P, _P, _P, _P, _P]),
    "echo_tree_verify_attn_paged": (_I32, [_P, _P, _P, _P, _P, _I64, _I32, _P, _I32, _P, _P, _P,
                                           _I32, _I32, _I32, _I32, _I32, _I32, _F32, _P, _P, _P,
                                           _SZ, _P, _P]),
    "echo_accept_logits": (_I32, [_P, _P, _P, _P, _I64, _I32, _I32, _I32, _P, _P, _P, _P, _P,
                                  _P]),
    "echo_commit_kv": (_I32, [_P, _P, _P, _I32, _P, _P, _I32, _I32, _I32, _P, _P, _I64, _I32, _P,
                              _I32, _P, _P, _P]),
    "echo_tree_verify_attn_timed": (_I32, [_P, _P, _P, _P, _P, _P, _I64, _P, _P, _I32, _I32, _I32,
                                           _I32, _I32, _I32, _F32, _P, _P, _P, _SZ, _P, _P, _P,
                                           _P]),
    "echo_tree_verify_attn_paged_timed": (_I32, [_P, _P, _P, _P, _P, _I64, _I32, _P, _I32, _P, _P,
                                                 _P, _I32, _I32, _I32, _I32, _I32, _I32, _F32, _P,
                                                 _P, _P, _SZ, _P, _P, _P, _P]),
    "echo_probe_stream_read": (_I32, [_P, _P, _I64, _I32, _I32, _P, _P]),
    "echo_verify_step": (_I32, [_P, _P, _P, _P, _I32, _I32, _I32, _P, _P, _P, _P, _SZ,
                                _P, _P, _P, _P, _P, _P, _P, _P, _I32,
                                _P, _P, _P, _P, _P, _P, _I64, _I32, _I32, _I32, _I32, _F32, _P,
                                _P, _P, _SZ,
                                _P, _I32, _P, _P, _P, _P, _P]),
    "echo_tree_verify_attn_paged_q8": (_I32, [_P, _P, _P, _I32, _P, _P, _P, _P, _I64, _I32, _P,
                                              _I32, _P, _P, _P, _I32, _I32, _I32, _I32, _I32,
                                              _I32, _F32, _P, _P, _P, _SZ, _P, _P]),
    "echo_tree_verify_attn_paged_q8_workspace_size": (_SZ, [_I32, _I32, _I32, _I32, _I32, _I32]),
    "echo_store_kv_q8": (_I32, [_P, _P, _I64, _I64, _P, _I32, _I32, _I32, _I32, _P, _P, _P, _P,
                                _I64, _I32, _P, _P]),
    "echo_commit_kv_q8": (_I32, [_P, _P, _P, _I32, _P, _P, _I32, _I32, _I32, _I32, _I32, _P, _P,
                                 _P, _P, _I64, _I32, _P, _I32, _P, _P, _P, _P]),
    "echo_build_block_tables": (_I32, [_P, _I32, _I32, _P, _I32, _P, _P, _P, _I32, _P, _P, _P,
                                       _P, _I32, _P, _P, _P]),
    "echo_rope": (_I32, [_P, _I64, _I64, _P, _I64, _I64, _I32, _P, _I64, _I64, _P, _I64, _I64,
                         _I32, _P, _I32, _P, _I32, _I32, _P, _F32, _P, _P]),
    "echo_rope_frequencies": (_I32, [_I32, _F64, _I32, _F64, _F64, _F64, _F64, _P, _P]),
    "echo_store_latent": (_I32, [_P, _I64, _P, _F32, _P, _P, _F32, _I32, _I32, _P, _I32, _I32, _P,
                                 _P, _P, _I64, _I32, _P, _P]),
    "echo_tree_verify_attn_latent": (_I32, [_P, _P, _P, _I64, _I32, _P, _I32, _P, _P, _P, _I32,
                                            _I32, _I32, _I32, _I32, _I32, _F32, _P, _P, _P, _SZ,
                                            _P, _P]),
    "echo_tree_verify_attn_latent_workspace_size": (_SZ, [_I32, _I32, _I32, _I32, _I32, _I32]),
    "echo_commit_latent": (_I32, [_P, _P, _P, _I32, _P, _I32, _I32, _I32, _I32, _P, _I64, _I32,
                                  _P, _I32, _P, _P, _P, _P]),
    "echo_status_string": (ctypes.c_char_p, [_I32]),
    "echo_version": (ctypes.c_char_p, []),
}


class EchoError(RuntimeError):
    pass


def load(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libecho (once).  Raises if it has not been built."""
    global _lib, _raw_stream, _device, _int32, _int64, _float32, _float64, _bits16
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise EchoError(f"{path} is missing: build it with "
                        "`python -m paper_2604_09603_amd.build` (there is no CPU fallback)")
    # torch ships its own HIP runtime under the same soname; load it first so that the
    # library and torch's streams and allocations share one runtime instance
    import torch
    # (a torch without GPU support has no streams, but the calls' refusals work there too)
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    _device = torch.cuda.current_device
    _int32, _int64, _float32, _float64 = torch.int32, torch.int64, torch.float32, torch.float64
    _bits16 = (torch.bfloat16, torch.int16, torch.uint16)
    lib = ctypes.CDLL(path)
    for name, (res, args) in _SIGS.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def _ptr(t):
    if t is None:
        return None
    return t.data_ptr()


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None:  # the current one; its handle alone is 2.4 us cheaper than its object
        return _raw_stream(_device())
    import torch
    return torch.cuda.current_stream().cuda_stream


def _check(code: int, what: str):
    if code != OK:
        raise EchoError(f"{what}: {load().echo_status_string(code).decode()} ({code})")


def _event(e):
    return ctypes.c_void_p(e.cuda_event)


def echo_probe_stream_read(k, v, rows, heads, mode, sink, stream=None, check=True):
    """Measurement helper: read two [rows, heads, 128] bf16 tensors once (mode 0: plain
    vector loads; mode 1: the attention's tile copies into LDS)."""
    code = load().echo_probe_stream_read(_ptr(k), _ptr(v), int(rows), int(heads), int(mode),
                                         _ptr(sink), _stream(stream))
    if check:
        _check(code, "echo_probe_stream_read")
    return code


def version() -> str:
    return load().echo_version().decode()


def status_string(code: int) -> str:
    return load().echo_status_string(code).decode()


def gate_workspace_size(R, N, budget) -> int:
    return int(load().echo_gate_workspace_size(R, N, budget))


def build_tree_mask_workspace_size(R, N, budget) -> int:
    return int(load().echo_build_tree_mask_workspace_size(R, N, budget))


def tree_verify_attn_workspace_size(R, max_rows, hq, hkv, head_dim=HEAD_DIM) -> int:
    return int(load().echo_tree_verify_attn_workspace_size(R, max_rows, hq, hkv, head_dim))


def echo_gate(cand_offsets, parent, logq, R, N, budget, path_score, selected, num_selected,
              workspace, status=None, stream=None, check=True):
    """Path scores and global top-B selection (eq. 5, eq. 4).  Device tensors."""
    code = load().echo_gate(_ptr(cand_offsets), _ptr(parent), _ptr(logq), R, N, budget,
                            _ptr(path_score), _ptr(selected), _ptr(num_selected), _ptr(workspace),
                            workspace.numel() * workspace.element_size(), _ptr(status),
                            _stream(stream))
    if check:
        _check(code, "echo_gate")
    return code


def echo_gate_noalloc(cand_offsets, parent, logq, R, N, budget, path_score, selected,
                      num_selected, status=None, stream=None, check=True):
    """echo_gate with the library's fixed per-device workspace (no allocation;
    overlapping calls on one device race)."""
    code = load().echo_gate_noalloc(_ptr(cand_offsets), _ptr(parent), _ptr(logq), R, N, budget,
                                    _ptr(path_score), _ptr(selected), _ptr(num_selected),
                                    _ptr(status), _stream(stream))
    if check:
        _check(code, "echo_gate_noalloc")
    return code


def echo_gate_sparse(cand_offsets, parent, logq, R, N, budget, sig_depth, log_tau, path_score,
                     selected, num_selected, workspace, trunc_depth=None, status=None,
                     stream=None, check=True):
    """Sparse checkpoint gating (eq. 6-7) then the global top-B.  ``sig_depth`` and
    ``log_tau`` are host sequences (checkpoint depths and ln tau); the rest are
    device tensors."""
    n = len(sig_depth)
    if len(log_tau) != n:
        raise ValueError("sig_depth and log_tau differ in length")
    depths = (ctypes.c_int32 * max(n, 1))(*[int(x) for x in sig_depth])
    taus = (ctypes.c_float * max(n, 1))(*[float(x) for x in log_tau])
    code = load().echo_gate_sparse(_ptr(cand_offsets), _ptr(parent), _ptr(logq), R, N, budget,
                                   ctypes.cast(depths, _P), ctypes.cast(taus, _P), n,
                                   _ptr(path_score), _ptr(selected), _ptr(num_selected),
                                   _ptr(trunc_depth), _ptr(workspace),
                                   workspace.numel() * workspace.element_size(), _ptr(status),
                                   _stream(stream))
    if check:
        _check(code, "echo_gate_sparse")
    return code


def gate_elastic_workspace_size(R, N, budget) -> int:
    return int(load().echo_gate_elastic_workspace_size(R, N, budget))


def echo_gate_elastic(cand_offsets, parent, logq, R, N, budget, sig_depth, log_tau, w_topk, w_max,
                      path_score, selected, num_selected, workspace, trunc_depth=None,
                      status=None, stream=None, check=True):
    """Alg. 1's elastic budget scheduler as a selection.  ``sig_depth`` and
    ``log_tau`` are host sequences; the rest are device tensors."""
    n = len(sig_depth)
    if len(log_tau) != n:
        raise ValueError("sig_depth and log_tau differ in length")
    depths = (ctypes.c_int32 * max(n, 1))(*[int(x) for x in sig_depth])
    taus = (ctypes.c_float * max(n, 1))(*[float(x) for x in log_tau])
    code = load().echo_gate_elastic(_ptr(cand_offsets), _ptr(parent), _ptr(logq), R, N, budget,
                                    ctypes.cast(depths, _P), ctypes.cast(taus, _P), n, w_topk,
                                    w_max, _ptr(path_score), _ptr(selected), _ptr(num_selected),
                                    _ptr(trunc_depth), _ptr(workspace),
                                    workspace.numel() * workspace.element_size(), _ptr(status),
                                    _stream(stream))
    if check:
        _check(code, "echo_gate_elastic")
    return code


def echo_build_tree_mask(cand_offsets, parent, token, selected, root_token, prefix_len, R, N,
                         budget, q_offsets, slot_cand, slot_parent, slot_token, position_ids,
                         tree_mask, mask_words, workspace=None, status=None, stream=None,
                         check=True):
    """Flatten & pack the selection into verify slots.  Device tensors."""
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    code = load().echo_build_tree_mask(
        _ptr(cand_offsets), _ptr(parent), _ptr(token), _ptr(selected), _ptr(root_token),
        _ptr(prefix_len), R, N, budget, _ptr(q_offsets), _ptr(slot_cand), _ptr(slot_parent),
        _ptr(slot_token), _ptr(position_ids), _ptr(tree_mask), mask_words, _ptr(workspace),
        ws_bytes, _ptr(status), _stream(stream))
    if check:
        _check(code, "echo_build_tree_mask")
    return code


def echo_tree_verify_attn(q, k_new, v_new, k_cache, v_cache, kv_offsets, kv_rows, q_offsets,
                          tree_mask, mask_words, R, max_rows, hq, hkv, head_dim, sm_scale, out,
                          lse, workspace, status=None, stream=None, check=True):
    """Tree-masked GQA verification attention.  bf16 inputs as int16/uint16/bfloat16 tensors."""
    code = load().echo_tree_verify_attn(
        _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(k_cache), _ptr(v_cache), _ptr(kv_offsets),
        int(kv_rows), _ptr(q_offsets), _ptr(tree_mask), mask_words, R, max_rows, hq, hkv, head_dim,
        float(sm_scale), _ptr(out), _ptr(lse), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _ptr(status), _stream(stream))
    if check:
        _check(code, "echo_tree_verify_attn")
    return code


def echo_tree_verify_attn_timed(q, k_new, v_new, k_cache, v_cache, kv_offsets, kv_rows, q_offsets,
                                tree_mask, mask_words, R, max_rows, hq, hkv, head_dim, sm_scale,
                                out, lse, workspace, ev_start, ev_stop, status=None, stream=None,
                                check=True):
    """echo_tree_verify_attn with two torch.cuda.Event objects recorded around its
    main kernel on its stream (measurement only)."""
    code = load().echo_tree_verify_attn_timed(
        _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(k_cache), _ptr(v_cache), _ptr(kv_offsets),
        int(kv_rows), _ptr(q_offsets), _ptr(tree_mask), mask_words, R, max_rows, hq, hkv, head_dim,
        float(sm_scale), _ptr(out), _ptr(lse), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _ptr(status), _event(ev_start),
        _event(ev_stop), _stream(stream))
    if check:
        _check(code, "echo_tree_verify_attn_timed")
    return code


def echo_accept(q_offsets, slot_parent, slot_token, target_token, R, max_rows, max_depth,
                accept_len, accept_slots, bonus_token, status=None, stream=None, check=True):
    """Greedy acceptance of the longest matching path per request."""
    code = load().echo_accept(_ptr(q_offsets), _ptr(slot_parent), _ptr(slot_token),
                              _ptr(target_token), R, max_rows, max_depth, _ptr(accept_len),
                              _ptr(accept_slots), _ptr(bonus_token), _ptr(status),
                              _stream(stream))
    if check:
        _check(code, "echo_accept")
    return code


def echo_verify_step(cand_offsets, parent, logq, token, R, N, budget, path_score, selected,
                     num_selected, gate_workspace, root_token, prefix_len, q_offsets, slot_cand,
                     slot_parent, slot_token, position_ids, tree_mask, mask_words, q, k_new, v_new,
                     k_cache, v_cache, kv_offsets, kv_rows, max_rows, hq, hkv, head_dim, sm_scale,
                     out, lse, attn_workspace, target_token, max_depth, accept_len, accept_slots,
                     bonus_token, status=None, stream=None, check=True):
    """The four stages of a step in one call (gate, flatten & pack, attention over a
    contiguous cache, acceptance); the arguments of the four calls in order."""
    code = load().echo_verify_step(
        _ptr(cand_offsets), _ptr(parent), _ptr(logq), _ptr(token), R, N, budget, _ptr(path_score),
        _ptr(selected), _ptr(num_selected), _ptr(gate_workspace),
        gate_workspace.numel() * gate_workspace.element_size(), _ptr(root_token),
        _ptr(prefix_len), _ptr(q_offsets), _ptr(slot_cand), _ptr(slot_parent), _ptr(slot_token),
        _ptr(position_ids), _ptr(tree_mask), mask_words, _ptr(q), _ptr(k_new), _ptr(v_new),
        _ptr(k_cache), _ptr(v_cache), _ptr(kv_offsets), int(kv_rows), max_rows, hq, hkv, head_dim,
        float(sm_scale), _ptr(out), _ptr(lse), _ptr(attn_workspace),
        attn_workspace.numel() * attn_workspace.element_size(), _ptr(target_token), max_depth,
        _ptr(accept_len), _ptr(accept_slots), _ptr(bonus_token), _ptr(status), _stream(stream))
    if check:
        _check(code, "echo_verify_step")
    return code


def echo_tree_verify_attn_paged(q, k_new, v_new, k_pages, v_pages, page_size, block_table,
                                prefix_len, q_offsets, tree_mask, mask_words, R, max_rows, hq,
                                hkv, head_dim, sm_scale, out, lse, workspace, status=None,
                                stream=None, check=True):
    """Verification attention over a paged KV cache.  Device tensors; k_pages is
    [num_pages, page_size, Hkv, 128] bf16 bits, block_table [R, max_pages]."""
    code = load().echo_tree_verify_attn_paged(
        _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(k_pages), _ptr(v_pages), k_pages.shape[0],
        page_size, _ptr(block_table), block_table.shape[1], _ptr(prefix_len), _ptr(q_offsets),
        _ptr(tree_mask), mask_words, R, max_rows, hq, hkv, head_dim, sm_scale, _ptr(out),
        _ptr(lse), _ptr(workspace), workspace.numel() * workspace.element_size(), _ptr(status),
        _stream(stream))
    if check:
        _check(code, "echo_tree_verify_attn_paged")
    return code


def echo_tree_verify_attn_paged_timed(q, k_new, v_new, k_pages, v_pages, page_size, block_table,
                                      prefix_len, q_offsets, tree_mask, mask_words, R, max_rows,
                                      hq, hkv, head_dim, sm_scale, out, lse, workspace, ev_start,
                                      ev_stop, status=None, stream=None, check=True):
    """echo_tree_verify_attn_paged with events around its main kernel (measurement only)."""
    code = load().echo_tree_verify_attn_paged_timed(
        _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(k_pages), _ptr(v_pages), k_pages.shape[0],
        page_size, _ptr(block_table), block_table.shape[1], _ptr(prefix_len), _ptr(q_offsets),
        _ptr(tree_mask), mask_words, R, max_rows, hq, hkv, head_dim, sm_scale, _ptr(out),
        _ptr(lse), _ptr(workspace), workspace.numel() * workspace.element_size(), _ptr(status),
        _event(ev_start), _event(ev_stop), _stream(stream))
    if check:
        _check(code, "echo_tree_verify_attn_paged_timed")
    return code


def echo_accept_logits(q_offsets, slot_parent, slot_token, logits, R, max_rows, max_depth,
                       target_token, accept_len, accept_slots, bonus_token, status=None,
                       stream=None, check=True):
    """Target argmax of bf16 logits [max_rows, V] followed by greedy acceptance."""
    code = load().echo_accept_logits(_ptr(q_offsets), _ptr(slot_parent), _ptr(slot_token),
                                     _ptr(logits), logits.shape[1], R, max_rows, max_depth,
                                     _ptr(target_token), _ptr(accept_len), _ptr(accept_slots),
                                     _ptr(bonus_token), _ptr(status), _stream(stream))
    if check:
        _check(code, "echo_accept_logits")
    return code


def echo_commit_kv(q_offsets, accept_len, accept_slots, max_depth, k_new, v_new, R, max_rows,
                   hkv, k_pages, v_pages, page_size, block_table, prefix_len, status=None,
                   stream=None, check=True):
    """Append each request's root and accepted slots to its paged KV cache."""
    code = load().echo_commit_kv(_ptr(q_offsets), _ptr(accept_len), _ptr(accept_slots),
                                 max_depth, _ptr(k_new), _ptr(v_new), R, max_rows, hkv,
                                 _ptr(k_pages), _ptr(v_pages), k_pages.shape[0], page_size,
                                 _ptr(block_table), block_table.shape[1], _ptr(prefix_len),
                                 _ptr(status), _stream(stream))
    if check:
        _check(code, "echo_commit_kv")
    return code


def tree_verify_attn_paged_q8_workspace_size(R, max_rows, hq, hkv, max_pages,
                                             head_dim=HEAD_DIM) -> int:
    return int(load().echo_tree_verify_attn_paged_q8_workspace_size(R, max_rows, hq, hkv,
                                                                    head_dim, max_pages))


def echo_tree_verify_attn_paged_q8(q, k_new, v_new, kv_format, k_pages, v_pages, k_scale, v_scale,
                                   page_size, block_table, prefix_len, q_offsets, tree_mask,
                                   mask_words, R, max_rows, hq, hkv, head_dim, sm_scale, out, lse,
                                   workspace, status=None, stream=None, check=True):
    """Verification attention over an 8-bit paged KV cache.  Device tensors; k_pages is
    [num_pages, Hkv, page_size, 128] bytes, k_scale [num_pages, Hkv, page_size / 32] float32,
    out [max_rows, Hq, 128] bf16 bits."""
    code = load().echo_tree_verify_attn_paged_q8(
        _ptr(q), _ptr(k_new), _ptr(v_new), kv_format, _ptr(k_pages), _ptr(v_pages), _ptr(k_scale),
        _ptr(v_scale), k_pages.shape[0], page_size, _ptr(block_table), block_table.shape[1],
        _ptr(prefix_len), _ptr(q_offsets), _ptr(tree_mask), mask_words, R, max_rows, hq, hkv,
        head_dim, float(sm_scale), _ptr(out), _ptr(lse), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _ptr(status), _stream(stream))
    if check:
        _check(code, "echo_tree_verify_attn_paged_q8")
    return code


def echo_store_kv_q8(k, v, slot_map, num_rows, hkv, head_dim, kv_format, k_pages, v_pages, k_scale,
                     v_scale, page_size, status=None, stream=None, check=True):
    """Quantise rows into an 8-bit paged KV cache at the slots of a slot map.  Device tensors;
    k and v are [num_rows, Hkv, 128] bf16 bits whose rows may be strided (parts of one
    projection's output), slot_map int64."""
    ks, vs = k.stride(), v.stride()
    if ks[-1] != 1 or vs[-1] != 1 or (hkv > 1 and (ks[-2] != head_dim or vs[-2] != head_dim)):
        raise ValueError("the heads of a row of k and v must be contiguous")
    # (the stride of a dimension of size 1 says nothing)
    code = load().echo_store_kv_q8(
        _ptr(k), _ptr(v), ks[0] if k.shape[0] > 1 else hkv * head_dim,
        vs[0] if v.shape[0] > 1 else hkv * head_dim, _ptr(slot_map), num_rows, hkv, head_dim,
        kv_format, _ptr(k_pages), _ptr(v_pages), _ptr(k_scale), _ptr(v_scale), k_pages.shape[0],
        page_size, _ptr(status), _stream(stream))
    if check:
        _check(code, "echo_store_kv_q8")
    return code


def echo_commit_kv_q8(q_offsets, accept_len, accept_slots, max_depth, k_new, v_new, R, max_rows,
                      hkv, head_dim, kv_format, k_pages, v_pages, k_scale, v_scale, page_size,
                      block_table, prefix_len, new_len, status=None, stream=None, check=True):
    """Append each request's root and accepted slots to its 8-bit paged KV cache; new_len may
    be prefix_len."""
    code = load().echo_commit_kv_q8(
        _ptr(q_offsets), _ptr(accept_len), _ptr(accept_slots), max_depth, _ptr(k_new), _ptr(v_new),
        R, max_rows, hkv, head_dim, kv_format, _ptr(k_pages), _ptr(v_pages), _ptr(k_scale),
        _ptr(v_scale), k_pages.shape[0], page_size, _ptr(block_table), block_table.shape[1],
        _ptr(prefix_len), _ptr(new_len), _ptr(status), _stream(stream))
    if check:
        _check(code, "echo_commit_kv_q8")
    return code


def echo_build_block_tables(want_len, R, page_size, block_table, num_held, num_held_out,
                            free_pages, num_free, num_free_out, row_offsets=None, row_start=None,
                            slot_map=None, status=None, stream=None, check=True):
    """Block tables (and the slot map of new rows, if given) from the requests' lengths.
    Device tensors; block_table is [R, max_pages] int32, free_pages the stack of free pages,
    slot_map int64."""
    code = load().echo_build_block_tables(
        _ptr(want_len), R, page_size, _ptr(block_table), block_table.shape[1], _ptr(num_held),
        _ptr(num_held_out), _ptr(free_pages), free_pages.numel(), _ptr(num_free),
        _ptr(num_free_out), _ptr(row_offsets), _ptr(row_start),
        0 if slot_map is None else slot_map.numel(), _ptr(slot_map), _ptr(status),
        _stream(stream))
    if check:
        _check(code, "echo_build_block_tables")
    return code


def _dense(name, t, dtype, n):
    """Refuse a tensor whose elements are not n or more of dtype, one after another."""
    if t is not None and (t.dtype is not dtype or t.numel() < n or not t.is_contiguous()):
        raise ValueError(f"{name}: {n} contiguous elements of {dtype}, not {tuple(t.shape)} of {t.dtype}")


def _dense_bits16(name, t, n):
    if t is not None and (t.dtype not in _bits16 or t.numel() < n or not t.is_contiguous()):
        raise ValueError(f"{name}: {n} contiguous bf16, not {tuple(t.shape)} of {t.dtype}")


def _head_strides(t, rows, heads, rot_dim):
    """Row and head strides of [rows, heads, rot_dim] (the stride of a dimension of size 1 says
    nothing)."""
    if t is None:
        return 0, 0
    shape, stride = t.shape, t.stride()
    if len(shape) != 3 or stride[2] != 1 or shape[1] != heads or shape[2] != rot_dim or shape[0] < rows:
        raise ValueError("q and k are [rows, heads, rot_dim] with contiguous dims")
    return stride[0] if shape[0] > 1 else 0, stride[1] if heads > 1 else rot_dim


def echo_rope(q, q_out, k, k_out, positions, num_rows, hq, hk, rot_dim, layout, inv_freq, scale,
              row_count=None, status=None, stream=None, check=True):
    """Rotary positions of queries and keys.  Device tensors; q and k (k may be None with hk 0)
    are [rows, heads, rot_dim] bf16 bits, views of the rotated part of each head with any
    strides; q_out may be q and k_out k; positions int32, inv_freq float64 [rot_dim / 2]."""
    qr, qh = _head_strides(q, num_rows, hq, rot_dim)
    qor, qoh = _head_strides(q_out, num_rows, hq, rot_dim)
    kr, kh = _head_strides(k, num_rows, hk, rot_dim)
    kor, koh = _head_strides(k_out, num_rows, hk, rot_dim)
    lib = load()
    _dense("positions", positions, _int32, num_rows)
    _dense("inv_freq", inv_freq, _float64, rot_dim // 2)
    code = lib.echo_rope(_ptr(q), qr, qh, _ptr(q_out), qor, qoh, hq, _ptr(k), kr, kh, _ptr(k_out),
                         kor, koh, hk, _ptr(positions), num_rows, _ptr(row_count), rot_dim, layout,
                         _ptr(inv_freq), scale, _ptr(status), _stream(stream))
    if check:
        _check(code, "echo_rope")
    return code


def echo_rope_frequencies(rot_dim, base, scaling="plain", factor=1.0, original_len=0.0,
                          low_turns=1.0, high_turns=32.0):
    """Inverse frequencies of rotary positions (a list of rot_dim / 2 floats, for a float64 tensor)
    and the factor on cosines and sines.  Computed on the host."""
    f = (ctypes.c_double * max(int(rot_dim) // 2, 1))()
    scale = ctypes.c_float()
    _check(load().echo_rope_frequencies(rot_dim, base, ROPE_SCALINGS[scaling], factor, original_len,
                                        low_turns, high_turns, ctypes.cast(f, _P),
                                        ctypes.addressof(scale)), "echo_rope_frequencies")
    return list(f), scale.value


def echo_store_latent(kv, norm_weight, eps, positions, inv_freq, rope_scale, layout, num_rows,
                      latent_dim, rope_dim, latent_new, slot_map, pages, page_size, row_count=None,
                      status=None, stream=None, check=True):
    """Normalise and rotate rows into the latent paged cache (slot_map, pages), beside a draft
    tree (latent_new), or both.  Device tensors; kv is [num_rows, 576] bf16 bits whose rows may
    be strided, norm_weight [512] bf16 bits or None, inv_freq float64 [32] or None, slot_map
    int64."""
    lib = load()
    s, shape, row = kv.stride(), kv.shape, latent_dim + rope_dim
    if len(s) != 2 or s[1] != 1 or shape[0] < num_rows or shape[1] < row or kv.dtype not in _bits16:
        raise ValueError("kv is [num_rows, latent_dim + rope_dim] bf16 with contiguous dims")
    _dense_bits16("norm_weight", norm_weight, latent_dim)
    if inv_freq is not None:
        _dense("positions", positions, _int32, num_rows)
        _dense("inv_freq", inv_freq, _float64, rope_dim // 2)
    _dense_bits16("latent_new", latent_new, num_rows * row)
    num_pages = 0
    if slot_map is not None:
        _dense("slot_map", slot_map, _int64, num_rows)
        num_pages = 0 if pages is None else pages.shape[0]
        _dense_bits16("pages", pages, num_pages * page_size * row)
    code = lib.echo_store_latent(
        _ptr(kv), s[0] if shape[0] > 1 else row, _ptr(norm_weight), eps, _ptr(positions),
        _ptr(inv_freq), rope_scale, layout, num_rows, _ptr(row_count), latent_dim, rope_dim,
        _ptr(latent_new), _ptr(slot_map), _ptr(pages), num_pages, page_size, _ptr(status),
        _stream(stream))
    if check:
        _check(code, "echo_store_latent")
    return code


def tree_verify_attn_latent_workspace_size(R, max_rows, hq, max_pages, latent_dim=LATENT_DIM,
                                           rope_dim=LATENT_ROPE_DIM) -> int:
    return int(load().echo_tree_verify_attn_latent_workspace_size(R, max_rows, hq, latent_dim,
                                                                  rope_dim, max_pages))


def echo_tree_verify_attn_latent(q, latent_new, pages, page_size, block_table, prefix_len,
                                 q_offsets, tree_mask, mask_words, R, max_rows, hq, latent_dim,
                                 rope_dim, sm_scale, out, lse, workspace, status=None,
                                 stream=None, check=True):
    """Verification attention over a latent paged cache (absorbed form).  Device tensors; q is
    [max_rows, Hq, 576] bf16 bits, latent_new [max_rows, 576], pages [num_pages, page_size, 576],
    out [max_rows, Hq, 512]."""
    lib = load()
    row, rows = latent_dim + rope_dim, max_rows * hq
    num_pages, max_pages = pages.shape[0], block_table.shape[1]
    for name, t, n in (("q", q, rows * row), ("latent_new", latent_new, max_rows * row),
                       ("pages", pages, num_pages * page_size * row), ("out", out, rows * latent_dim)):
        _dense_bits16(name, t, n)
    for name, t, n in (("block_table", block_table, R * max_pages), ("prefix_len", prefix_len, R),
                       ("q_offsets", q_offsets, R + 1)):
        _dense(name, t, _int32, n)
    if tree_mask.element_size() != 4 or tree_mask.numel() < max_rows * mask_words or not tree_mask.is_contiguous():
        raise ValueError("tree_mask is [max_rows, mask_words] words of 32 bits")
    _dense("lse", lse, _float32, rows)
    code = lib.echo_tree_verify_attn_latent(
        _ptr(q), _ptr(latent_new), _ptr(pages), num_pages, page_size, _ptr(block_table), max_pages,
        _ptr(prefix_len), _ptr(q_offsets), _ptr(tree_mask), mask_words, R, max_rows, hq, latent_dim,
        rope_dim, float(sm_scale), _ptr(out), _ptr(lse), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _ptr(status), _stream(stream))
    if check:
        _check(code, "echo_tree_verify_attn_latent")
    return code


def echo_commit_latent(q_offsets, accept_len, accept_slots, max_depth, latent_new, R, max_rows,
                       latent_dim, rope_dim, pages, page_size, block_table, prefix_len, new_len,
                       status=None, stream=None, check=True):
    """Append each request's root and accepted rows to its latent paged cache; new_len may be
    prefix_len."""
    code = load().echo_commit_latent(
        _ptr(q_offsets), _ptr(accept_len), _ptr(accept_slots), max_depth, _ptr(latent_new), R,
        max_rows, latent_dim, rope_dim, _ptr(pages), pages.shape[0], page_size, _ptr(block_table),
        block_table.shape[1], _ptr(prefix_len), _ptr(new_len), _ptr(status), _stream(stream))
    if check:
        _check(code, "echo_commit_latent")
    return code
