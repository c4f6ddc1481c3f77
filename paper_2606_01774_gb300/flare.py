"""Thin ctypes binding of ``libflare.so`` (declared in ``include/flare.h``).

Argument marshalling only: every function takes torch tensors that already
live on the current CUDA device (or None for nullable arguments), passes their
data pointers and the stream to the C entry point of the same name, and
returns the ``flare_status`` code.  No arithmetic of the method happens here,
and there is no fallback: if the library is missing or was built for another
machine, loading it raises.
"""
from __future__ import annotations

import ctypes
import re
import struct
from pathlib import Path

_PKG = Path(__file__).resolve().parent
LIB_PATH = _PKG / "libflare.so"
HEADER = _PKG.parent / "include" / "flare.h"

FLARE_OK = 0
FLARE_ERR_INVALID_ARGUMENT = 1
FLARE_ERR_UNSUPPORTED = 2
FLARE_ERR_CUDA = 3
FLARE_ERR_DEVICE_STATUS = 4

FLARE_DT_BF16 = 0
FLARE_DT_F32 = 1
FLARE_MASK_BLOCK_BIDIR = 0
FLARE_MASK_BLOCK_CAUSAL = 1
FLARE_MASK_ROW_TYPE_UNIFORM = 2
FLARE_MASK_ROW_TYPE_PER_REQUEST = 3
FLARE_ROW_CAUSAL = 0
FLARE_ROW_BIDIR = 1
FLARE_ACT_NONE = 0
FLARE_ACT_SILU = 1
FLARE_ACT_SIGMOID = 2
FLARE_ROTARY_HALF = 0
FLARE_ROTARY_INTERLEAVED = 1
FLARE_ROTARY_PLAIN = 0
FLARE_ROTARY_LINEAR = 1
FLARE_ROTARY_BASE = 2
FLARE_ROTARY_BY_PARTS = 3

FLARE_DEV_BAD_SLOT = 0x1
FLARE_DEV_BAD_PAGE = 0x2
FLARE_DEV_BAD_PREFIX_LEN = 0x4
FLARE_DEV_BAD_ACCEPT_LEN = 0x8
FLARE_DEV_WAIT_TIMEOUT = 0x10
FLARE_DEV_BAD_VERIFY_LEN = 0x20
FLARE_DEV_BAD_TREE = 0x40
FLARE_DEV_BAD_LOGITS = 0x80
FLARE_DEV_BAD_HISTORY = 0x100
FLARE_DEV_BAD_PENALTY = 0x200

FLARE_VERIFY_GREEDY = 0
FLARE_VERIFY_SAMPLE = 1


class FlareError(RuntimeError):
    def __init__(self, status, what=""):
        self.status = status
        super().__init__(f"{what}: {flare_status_string(status)}" if what else
                         flare_status_string(status))


class flare_linear_desc(ctypes.Structure):
    _fields_ = [("num_requests", ctypes.c_int32), ("block_len", ctypes.c_int32),
                ("num_qk_heads", ctypes.c_int32), ("num_v_heads", ctypes.c_int32),
                ("head_dim_k", ctypes.c_int32), ("head_dim_v", ctypes.c_int32),
                ("num_state_slots", ctypes.c_int32), ("act_dtype", ctypes.c_int),
                ("scale", ctypes.c_float)]


class flare_conv_desc(ctypes.Structure):
    _fields_ = [("num_requests", ctypes.c_int32), ("block_len", ctypes.c_int32),
                ("channels", ctypes.c_int32), ("width", ctypes.c_int32),
                ("num_state_slots", ctypes.c_int32), ("act_dtype", ctypes.c_int),
                ("activation", ctypes.c_int)]


class flare_two_stream_desc(ctypes.Structure):
    _fields_ = [("num_seqs", ctypes.c_int32), ("seq_len", ctypes.c_int32),
                ("chunk_len", ctypes.c_int32), ("block_len", ctypes.c_int32),
                ("num_qk_heads", ctypes.c_int32), ("num_v_heads", ctypes.c_int32),
                ("head_dim_k", ctypes.c_int32), ("head_dim_v", ctypes.c_int32),
                ("act_dtype", ctypes.c_int), ("scale", ctypes.c_float)]


class flare_tree_verify_desc(ctypes.Structure):
    _fields_ = [("num_requests", ctypes.c_int32), ("num_nodes", ctypes.c_int32),
                ("vocab_size", ctypes.c_int32), ("logits_dtype", ctypes.c_int),
                ("mode", ctypes.c_int), ("inv_temperature", ctypes.c_float)]


class flare_rotary_freq_desc(ctypes.Structure):
    _fields_ = [("rotary_dim", ctypes.c_int32), ("scaling", ctypes.c_int),
                ("base", ctypes.c_double), ("factor", ctypes.c_double),
                ("original_len", ctypes.c_double), ("low_turns", ctypes.c_double),
                ("high_turns", ctypes.c_double)]


class flare_rotary_desc(ctypes.Structure):
    _fields_ = [("num_requests", ctypes.c_int32), ("block_len", ctypes.c_int32),
                ("num_tokens", ctypes.c_int32), ("num_q_heads", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("rotary_dim", ctypes.c_int32), ("layout", ctypes.c_int),
                ("inverse", ctypes.c_int32), ("act_dtype", ctypes.c_int),
                ("amplitude", ctypes.c_float), ("q_stride", ctypes.c_int64),
                ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64),
                ("page_size", ctypes.c_int32), ("num_pages", ctypes.c_int32),
                ("max_pages_per_req", ctypes.c_int32)]


class flare_tree_logits_desc(ctypes.Structure):
    _fields_ = [("num_requests", ctypes.c_int32), ("num_nodes", ctypes.c_int32),
                ("vocab_size", ctypes.c_int32), ("logits_dtype", ctypes.c_int),
                ("max_history", ctypes.c_int32), ("max_bias", ctypes.c_int32)]


class flare_block_norm_desc(ctypes.Structure):
    _fields_ = [("num_tokens", ctypes.c_int32), ("width", ctypes.c_int32),
                ("group", ctypes.c_int32), ("shared_weight", ctypes.c_int32),
                ("post_norm", ctypes.c_int32), ("pre_norm", ctypes.c_int32),
                ("gate_act", ctypes.c_int), ("act_dtype", ctypes.c_int),
                ("eps", ctypes.c_float), ("residual_scale", ctypes.c_float),
                ("x_stride", ctypes.c_int64), ("gate_stride", ctypes.c_int64)]


class flare_softmax_desc(ctypes.Structure):
    _fields_ = [("num_requests", ctypes.c_int32), ("block_len", ctypes.c_int32),
                ("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("num_pages", ctypes.c_int32), ("max_pages_per_req", ctypes.c_int32),
                ("act_dtype", ctypes.c_int), ("scale", ctypes.c_float),
                ("mask_mode", ctypes.c_int), ("row_type", ctypes.c_void_p)]


_lib = None


def load() -> ctypes.CDLL:
    """Load libflare.so (raises OSError if it is missing: there is no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    if not LIB_PATH.exists():
        raise OSError(f"{LIB_PATH} is missing; build it with paper_2606_01774_gb300.build.build()")
    lib = ctypes.CDLL(str(LIB_PATH))
    P, S, I32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32
    lin = ctypes.POINTER(flare_linear_desc)
    smx = ctypes.POINTER(flare_softmax_desc)
    cnv = ctypes.POINTER(flare_conv_desc)
    tsd = ctypes.POINTER(flare_two_stream_desc)
    tvd = ctypes.POINTER(flare_tree_verify_desc)
    frq = ctypes.POINTER(flare_rotary_freq_desc)
    rot = ctypes.POINTER(flare_rotary_desc)
    tld = ctypes.POINTER(flare_tree_logits_desc)
    bnd = ctypes.POINTER(flare_block_norm_desc)
    sigs = {
        "flare_short_conv": [cnv] + [P] * 9,
        "flare_two_stream_fwd": [tsd] + [P] * 13,
        "flare_block_linear_attn": [lin] + [P] * 10,
        "flare_commit_state": [lin] + [P] * 11,
        "flare_verify_linear_attn": [lin, I32] + [P] * 12,
        "flare_verify_commit": [lin, I32, I32] + [P] * 7,
        "flare_softmax_workspace_size": [smx, ctypes.POINTER(S)],
        "flare_block_softmax_attn": [smx] + [P] * 10 + [S, P, P],
        "flare_block_softmax_attn_noalloc": [smx] + [P] * 11,
        "flare_append_kv": [smx] + [P] * 9,
        "flare_tree_softmax_workspace_size": [smx, ctypes.POINTER(S)],
        "flare_tree_softmax_attn": [smx] + [P] * 12 + [S, P, P],
        "flare_tree_linear_attn": [lin] + [P] * 12,
        "flare_tree_verify_workspace_size": [tvd, ctypes.POINTER(S)],
        "flare_tree_verify": [tvd] + [P] * 12 + [S, P, P],
        "flare_tree_commit_state": [lin] + [P] * 11,
        "flare_tree_append_kv": [smx, I32] + [P] * 10,
        "flare_rotary_table": [frq, P, P],
        "flare_rotary": [rot] + [P] * 12,
        "flare_rotary_append_kv": [rot] + [P] * 15,
        "flare_tree_logits": [tld] + [P] * 17,
        "flare_block_norm": [bnd] + [P] * 8,
        "flare_block_norm_bwd_workspace_size": [bnd, ctypes.POINTER(S)],
        "flare_block_norm_bwd": [bnd] + [P] * 13 + [S, P],
        "flare_debug_gather_prefix": [smx, P, P, P, P, I32, P, P, P, P],
        "flare_debug_wait_timeout": [P, ctypes.c_uint64, P],
        "flare_read_status": [P, P, ctypes.POINTER(I32)],
    }
    for name, args in sigs.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = ctypes.c_int
    lib.flare_launch_count.argtypes = []
    lib.flare_launch_count.restype = ctypes.c_uint64
    lib.flare_status_string.argtypes = [ctypes.c_int]
    lib.flare_status_string.restype = ctypes.c_char_p
    _lib = lib
    return lib


def declared_functions():
    """Names of the entry points declared in include/flare.h."""
    text = HEADER.read_text()
    return sorted(set(re.findall(r"^\s*(?:const\s+)?[\w\s\*]*?\b(flare_\w+)\s*\(", text, re.M)))


def _p(t):
    if t is None:
        return None
    return ctypes.c_void_p(t.data_ptr())


def _current_stream():
    """Handle of the current device's current stream."""
    global _current_stream
    from torch import _C

    # the raw handle: building a torch.cuda.Stream object costs 3 us a call
    def _current_stream(device=_C._cuda_getDevice, raw=_C._cuda_getCurrentRawStream):
        return raw(device())

    return _current_stream()


def _stream(stream):
    if stream is None:
        return _current_stream()
    return ctypes.c_void_p(getattr(stream, "cuda_stream", stream))


def flare_launch_count() -> int:
    return int(load().flare_launch_count())


def flare_status_string(status: int) -> str:
    return load().flare_status_string(int(status)).decode()


def check(status: int, what: str = "") -> None:
    if status != FLARE_OK:
        raise FlareError(status, what)


def flare_block_linear_attn(desc, q, k, v, log_decay, beta, state_pool, state_slot, out,
                            dev_status, stream=None) -> int:
    return load().flare_block_linear_attn(
        ctypes.byref(desc), _p(q), _p(k), _p(v), _p(log_decay), _p(beta), _p(state_pool),
        _p(state_slot), _p(out), _p(dev_status), _stream(stream))


def flare_commit_state(desc, q, k, v, log_decay, beta, state_pool, state_slot, accept_len,
                       causal_out, dev_status, stream=None) -> int:
    return load().flare_commit_state(
        ctypes.byref(desc), _p(q), _p(k), _p(v), _p(log_decay), _p(beta), _p(state_pool),
        _p(state_slot), _p(accept_len), _p(causal_out), _p(dev_status), _stream(stream))


def flare_verify_linear_attn(desc, max_verify, q, k, v, log_decay, beta, state_pool,
                             state_slot, verify_len, out, verify_states, dev_status,
                             stream=None) -> int:
    return load().flare_verify_linear_attn(
        ctypes.byref(desc), int(max_verify), _p(q), _p(k), _p(v), _p(log_decay), _p(beta),
        _p(state_pool), _p(state_slot), _p(verify_len), _p(out), _p(verify_states),
        _p(dev_status), _stream(stream))


def flare_verify_commit(desc, max_verify, verify_states, state_pools, state_slot, accept,
                        verify_len, dev_status, stream=None) -> int:
    """verify_states, state_pools: sequences of per-layer device tensors; their
    data pointers are passed as host arrays."""
    n = len(state_pools)
    recs = (ctypes.c_void_p * n)(*[None if t is None else t.data_ptr() for t in verify_states])
    pools = (ctypes.c_void_p * n)(*[t.data_ptr() for t in state_pools])
    return load().flare_verify_commit(
        ctypes.byref(desc), int(max_verify), n, recs, pools, _p(state_slot), _p(accept),
        _p(verify_len), _p(dev_status), _stream(stream))


def flare_short_conv(desc, x, conv_state, state_slot, weight, bias, accept_len, out,
                     dev_status, stream=None) -> int:
    return load().flare_short_conv(
        ctypes.byref(desc), _p(x), _p(conv_state), _p(state_slot), _p(weight), _p(bias),
        _p(accept_len), _p(out), _p(dev_status), _stream(stream))


def flare_two_stream_fwd(desc, chunk_states, k, v, log_decay, beta, q_noisy, k_noisy, v_noisy,
                         log_decay_noisy, beta_noisy, out_noisy, dev_status, stream=None) -> int:
    return load().flare_two_stream_fwd(
        ctypes.byref(desc), _p(chunk_states), _p(k), _p(v), _p(log_decay), _p(beta), _p(q_noisy),
        _p(k_noisy), _p(v_noisy), _p(log_decay_noisy), _p(beta_noisy), _p(out_noisy),
        _p(dev_status), _stream(stream))


def flare_softmax_workspace_size(desc) -> int:
    n = ctypes.c_size_t(0)
    check(load().flare_softmax_workspace_size(ctypes.byref(desc), ctypes.byref(n)),
          "flare_softmax_workspace_size")
    return int(n.value)


def flare_block_softmax_attn(desc, q, k_blk, v_blk, k_pool, v_pool, page_table, prefix_len,
                             out, lse, workspace, workspace_bytes, dev_status, stream=None) -> int:
    return load().flare_block_softmax_attn(
        ctypes.byref(desc), _p(q), _p(k_blk), _p(v_blk), _p(k_pool), _p(v_pool), _p(page_table),
        _p(prefix_len), _p(out), _p(lse), _p(workspace), int(workspace_bytes), _p(dev_status),
        _stream(stream))


def flare_append_kv(desc, k_blk, v_blk, k_pool, v_pool, page_table, prefix_len, append_len,
                    dev_status, stream=None) -> int:
    return load().flare_append_kv(
        ctypes.byref(desc), _p(k_blk), _p(v_blk), _p(k_pool), _p(v_pool), _p(page_table),
        _p(prefix_len), _p(append_len), _p(dev_status), _stream(stream))


FLARE_NOALLOC_SCRATCH_BYTES = 64 * 1024 * 1024


def flare_block_softmax_attn_noalloc(desc, q, k_blk, v_blk, k_pool, v_pool, page_table,
                                     prefix_len, out, lse, dev_status, stream=None) -> int:
    return load().flare_block_softmax_attn_noalloc(
        ctypes.byref(desc), _p(q), _p(k_blk), _p(v_blk), _p(k_pool), _p(v_pool), _p(page_table),
        _p(prefix_len), _p(out), _p(lse), _p(dev_status), _stream(stream))


def _c(t):
    """Data pointer of a tensor that must be contiguous."""
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("the tree calls take contiguous tensors")
    return t.data_ptr()


def flare_tree_softmax_workspace_size(desc) -> int:
    n = ctypes.c_size_t(0)
    check(load().flare_tree_softmax_workspace_size(ctypes.byref(desc), ctypes.byref(n)),
          "flare_tree_softmax_workspace_size")
    return int(n.value)


def flare_tree_softmax_attn(desc, q, k_blk, v_blk, k_pool, v_pool, page_table, prefix_len, parent,
                            node_len, out, lse, workspace, workspace_bytes, dev_status,
                            stream=None) -> int:
    return load().flare_tree_softmax_attn(
        ctypes.byref(desc), _c(q), _c(k_blk), _c(v_blk), _c(k_pool), _c(v_pool), _c(page_table),
        _c(prefix_len), _c(parent), _c(node_len), _c(out), _c(lse), _c(workspace),
        int(workspace_bytes), _c(dev_status), _stream(stream))


def flare_tree_linear_attn(desc, q, k, v, log_decay, beta, state_pool, state_slot, parent,
                           node_len, out, dev_status, stream=None) -> int:
    return load().flare_tree_linear_attn(
        ctypes.byref(desc), _c(q), _c(k), _c(v), _c(log_decay), _c(beta), _c(state_pool),
        _c(state_slot), _c(parent), _c(node_len), _c(out), _c(dev_status), _stream(stream))


def flare_tree_verify_workspace_size(desc) -> int:
    n = ctypes.c_size_t(0)
    check(load().flare_tree_verify_workspace_size(ctypes.byref(desc), ctypes.byref(n)),
          "flare_tree_verify_workspace_size")
    return int(n.value)


def flare_tree_verify(desc, logits, draft_probs, token, parent, node_len, uniform, noise, path,
                      path_len, next_token, node_logp, workspace, workspace_bytes, dev_status,
                      stream=None) -> int:
    return load().flare_tree_verify(
        ctypes.byref(desc), _c(logits), _c(draft_probs), _c(token), _c(parent), _c(node_len),
        _c(uniform), _c(noise), _c(path), _c(path_len), _c(next_token), _c(node_logp),
        _c(workspace), int(workspace_bytes), _c(dev_status), _stream(stream))


def flare_tree_commit_state(desc, k, v, log_decay, beta, state_pool, src_slot, dst_slot, path,
                            path_len, dev_status, stream=None) -> int:
    return load().flare_tree_commit_state(
        ctypes.byref(desc), _c(k), _c(v), _c(log_decay), _c(beta), _c(state_pool), _c(src_slot),
        _c(dst_slot), _c(path), _c(path_len), _c(dev_status), _stream(stream))


def _pointers(*lists):
    """Host arrays of the tensors' data pointers, as bytes (half the time of ctypes arrays)."""
    from torch import Tensor

    for tensors in lists:
        if not all(map(Tensor.is_contiguous, tensors)):
            raise ValueError("the tree calls take contiguous tensors")
    form = f"{len(lists[0])}P"
    return [struct.pack(form, *map(Tensor.data_ptr, tensors)) for tensors in lists]


def flare_tree_append_kv(desc, k_blk, v_blk, k_pool, v_pool, page_table, prefix_len, path,
                         path_len, dev_status, stream=None) -> int:
    """k_blk, v_blk, k_pool, v_pool: sequences of per-layer device tensors, of one length; their
    data pointers are passed as host arrays."""
    n = len(k_pool)
    if not len(k_blk) == len(v_blk) == len(v_pool) == n:
        raise ValueError("one k_blk, v_blk, k_pool and v_pool per layer")
    return load().flare_tree_append_kv(
        ctypes.byref(desc), n, *_pointers(k_blk, v_blk, k_pool, v_pool), _c(page_table),
        _c(prefix_len), _c(path), _c(path_len), _c(dev_status), _stream(stream))


def _device():
    """Index of the current device."""
    global _device
    from torch import _C

    _device = _C._cuda_getDevice
    return _device()


def _dense(device, *tensors):
    """Data pointers of contiguous tensors on the current device, None for None."""
    there = [t for t in tensors if t is not None]
    if not all(map(_is_contiguous, there)):
        raise ValueError("only the rows of q, k, v, x, gate and their gradients may be strided")
    for at in map(_get_device, there):
        if at != device:
            raise ValueError("tensors must be on the current device")
    return [None if t is None else t.data_ptr() for t in tensors]


def _is_contiguous(t):
    global _is_contiguous, _get_device
    from torch import Tensor

    _is_contiguous, _get_device = Tensor.is_contiguous, Tensor.get_device
    return t.is_contiguous()


def _get_device(t):
    return t.get_device()


def _rows(t, step, inner, device):
    """Data pointer of rows `step` elements apart (0: dense), a row's elements contiguous.

    The rows are all leading dimensions but the last `inner`."""
    if t is None:
        return None
    if t.get_device() != device:
        raise ValueError("tensors must be on the current device")
    strides = t.stride()  # 0 over rows: one row repeated, not dense
    if step and len(strides) == inner + 1 and strides[0] == step and (
            strides[-1] == 1 and (inner == 1 or strides[1] == t.shape[2])):
        return t.data_ptr()
    if not step and t.is_contiguous():
        return t.data_ptr()
    dense = 1
    for i in range(t.dim() - 1, -1, -1):
        if i == t.dim() - inner - 1:
            dense = step or dense
        if t.shape[i] > 1 and t.stride(i) != dense:
            raise ValueError("strides other than the descriptor's")
        dense *= t.shape[i]
    return t.data_ptr()


def flare_rotary_table(desc, table, stream=None) -> int:
    return load().flare_rotary_table(ctypes.byref(desc), *_dense(_device(), table),
                                     _stream(stream))


def _in_place(out, source):
    return out is not None and source is not None and out.data_ptr() == source.data_ptr()


def flare_rotary(desc, q, k, table, position, prefix_len, token_len, parent, token_start, q_out,
                 k_out, dev_status, stream=None) -> int:
    """q, k (and the outputs written in place) have rows q_stride and k_stride apart."""
    dev = _device()
    qs, ks = desc.q_stride, desc.k_stride
    q_at, k_at = _rows(q, qs, 2, dev), _rows(k, ks, 2, dev)
    q_to = k_to = None
    if _in_place(q_out, q):
        q_to, q_out = _rows(q_out, qs, 2, dev), None
    if _in_place(k_out, k):
        k_to, k_out = _rows(k_out, ks, 2, dev), None
    *ins, qo, ko, status = _dense(dev, table, position, prefix_len, token_len, parent, token_start,
                                  q_out, k_out, dev_status)
    return load().flare_rotary(ctypes.byref(desc), q_at, k_at, *ins, q_to or qo, k_to or ko, status,
                               _stream(stream))


def flare_rotary_append_kv(desc, q, k, v, table, position, prefix_len, token_len, token_start,
                           page_table, q_out, k_out, k_pool, v_pool, dev_status,
                           stream=None) -> int:
    dev = _device()
    qs, ks = desc.q_stride, desc.k_stride
    q_at, k_at, v_at = _rows(q, qs, 2, dev), _rows(k, ks, 2, dev), _rows(v, desc.v_stride, 2, dev)
    q_to = k_to = None
    if _in_place(q_out, q):
        q_to, q_out = _rows(q_out, qs, 2, dev), None
    if _in_place(k_out, k):
        k_to, k_out = _rows(k_out, ks, 2, dev), None
    *ins, qo, ko, kp, vp, status = _dense(dev, table, position, prefix_len, token_len, token_start,
                                          page_table, q_out, k_out, k_pool, v_pool, dev_status)
    return load().flare_rotary_append_kv(ctypes.byref(desc), q_at, k_at, v_at, *ins, q_to or qo,
                                         k_to or ko, kp, vp, status, _stream(stream))


def flare_tree_logits(desc, logits, history, history_len, output_start, token, parent, node_len,
                      repetition, presence, frequency, bias_token, bias_value, bias_len, mask,
                      out, dev_status, stream=None) -> int:
    return load().flare_tree_logits(
        ctypes.byref(desc),
        *_dense(_device(), logits, history, history_len, output_start, token, parent, node_len,
                repetition, presence, frequency, bias_token, bias_value, bias_len, mask, out,
                dev_status), _stream(stream))


def flare_block_norm(desc, x, gate, residual, post_weight, pre_weight, y, h, stream=None) -> int:
    dev = _device()
    return load().flare_block_norm(
        ctypes.byref(desc), _rows(x, desc.x_stride, 1, dev), _rows(gate, desc.gate_stride, 1, dev),
        *_dense(dev, residual, post_weight, pre_weight, y, h), _stream(stream))


def flare_block_norm_bwd_workspace_size(desc) -> int:
    n = ctypes.c_size_t(0)
    check(load().flare_block_norm_bwd_workspace_size(ctypes.byref(desc), ctypes.byref(n)),
          "flare_block_norm_bwd_workspace_size")
    return int(n.value)


def flare_block_norm_bwd(desc, x, gate, residual, post_weight, pre_weight, dy, dh, dx, dgate,
                         dresidual, dpost_weight, dpre_weight, workspace, workspace_bytes,
                         stream=None) -> int:
    """dx and dgate have their inputs' strides."""
    dev = _device()
    xs, gs = desc.x_stride, desc.gate_stride
    (res, w_post, w_pre, dy, dh, dres, dw_post, dw_pre, work) = _dense(
        dev, residual, post_weight, pre_weight, dy, dh, dresidual, dpost_weight, dpre_weight,
        workspace)
    return load().flare_block_norm_bwd(
        ctypes.byref(desc), _rows(x, xs, 1, dev), _rows(gate, gs, 1, dev), res, w_post, w_pre, dy,
        dh, _rows(dx, xs, 1, dev), _rows(dgate, gs, 1, dev), dres, dw_post, dw_pre, work,
        int(workspace_bytes), _stream(stream))


def flare_debug_gather_prefix(desc, k_pool, v_pool, page_table, prefix_len, request, k_out,
                              v_out, dev_status, stream=None) -> int:
    return load().flare_debug_gather_prefix(
        ctypes.byref(desc), _p(k_pool), _p(v_pool), _p(page_table), _p(prefix_len),
        int(request), _p(k_out), _p(v_out), _p(dev_status), _stream(stream))


def flare_debug_wait_timeout(dev_status, limit_ns, stream=None) -> int:
    return load().flare_debug_wait_timeout(_p(dev_status), int(limit_ns), _stream(stream))


def flare_read_status(dev_status, stream=None):
    """Returns (status, bits)."""
    bits = ctypes.c_int32(0)
    st = load().flare_read_status(_p(dev_status), _stream(stream), ctypes.byref(bits))
    return st, int(bits.value)


# ---------------------------------------------------------------- descriptors


def linear_desc(num_requests, block_len, num_qk_heads, num_v_heads, head_dim_k, head_dim_v,
                num_state_slots, act_dtype, scale) -> flare_linear_desc:
    return flare_linear_desc(num_requests, block_len, num_qk_heads, num_v_heads, head_dim_k,
                             head_dim_v, num_state_slots, act_dtype, scale)


def conv_desc(num_requests, block_len, channels, width, num_state_slots, act_dtype,
              activation=FLARE_ACT_SILU) -> flare_conv_desc:
    return flare_conv_desc(num_requests, block_len, channels, width, num_state_slots, act_dtype,
                           activation)


def two_stream_desc(num_seqs, seq_len, chunk_len, block_len, num_qk_heads, num_v_heads,
                    head_dim_k, head_dim_v, act_dtype, scale) -> flare_two_stream_desc:
    return flare_two_stream_desc(num_seqs, seq_len, chunk_len, block_len, num_qk_heads,
                                 num_v_heads, head_dim_k, head_dim_v, act_dtype, scale)


def tree_verify_desc(num_requests, num_nodes, vocab_size, logits_dtype,
                     mode=FLARE_VERIFY_SAMPLE, inv_temperature=1.0) -> flare_tree_verify_desc:
    return flare_tree_verify_desc(num_requests, num_nodes, vocab_size, logits_dtype, mode,
                                  inv_temperature)


def rotary_freq_desc(rotary_dim, base=10000.0, scaling=FLARE_ROTARY_PLAIN, factor=1.0,
                     original_len=0.0, low_turns=1.0, high_turns=32.0) -> flare_rotary_freq_desc:
    return flare_rotary_freq_desc(rotary_dim, scaling, base, factor, original_len, low_turns,
                                  high_turns)


def rotary_desc(num_requests, block_len, num_tokens, num_q_heads, num_kv_heads, head_dim,
                rotary_dim, act_dtype, layout=FLARE_ROTARY_HALF, inverse=0, amplitude=1.0,
                q_stride=0, k_stride=0, v_stride=0, page_size=0, num_pages=0,
                max_pages_per_req=0) -> flare_rotary_desc:
    """Padded rows read block_len, packed ones num_tokens; the page fields are the append's."""
    return flare_rotary_desc(num_requests, block_len, num_tokens, num_q_heads, num_kv_heads,
                             head_dim, rotary_dim, layout, inverse, act_dtype, amplitude, q_stride,
                             k_stride, v_stride, page_size, num_pages, max_pages_per_req)


def tree_logits_desc(num_requests, num_nodes, vocab_size, logits_dtype, max_history=0,
                     max_bias=0) -> flare_tree_logits_desc:
    return flare_tree_logits_desc(num_requests, num_nodes, vocab_size, logits_dtype, max_history,
                                  max_bias)


def block_norm_desc(num_tokens, width, act_dtype, group=0, shared_weight=0, post_norm=1,
                    pre_norm=1, gate_act=FLARE_ACT_NONE, eps=1e-6, residual_scale=1.0, x_stride=0,
                    gate_stride=0) -> flare_block_norm_desc:
    return flare_block_norm_desc(num_tokens, width, group, shared_weight, post_norm, pre_norm,
                                 gate_act, act_dtype, eps, residual_scale, x_stride, gate_stride)


def softmax_desc(num_requests, block_len, num_q_heads, num_kv_heads, head_dim, page_size,
                 num_pages, max_pages_per_req, act_dtype, scale,
                 mask_mode=FLARE_MASK_BLOCK_BIDIR, row_type=None) -> flare_softmax_desc:
    """row_type: uint8 device tensor ([B] or [R,B]) for the ROW_TYPE mask modes;
    the caller keeps it alive while the descriptor is in use."""
    return flare_softmax_desc(num_requests, block_len, num_q_heads, num_kv_heads, head_dim,
                              page_size, num_pages, max_pages_per_req, act_dtype, scale, mask_mode,
                              None if row_type is None else row_type.data_ptr())
