"""ctypes binding of the C-ABI in include/dc.h -- argument marshalling only.

Every function has the name and argument order of its C counterpart.  Device
buffers are torch tensors (or raw integer device addresses); the stream defaults
to torch's current HIP stream.  No step of the path is computed here, and there is
no CPU fallback: if ``libdc.so`` has not been built, loading raises.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from typing import Optional, Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdc.so")

DC_MAX_SEQ = 16384
DC_MAX_SEQ_LARGE = 1 << 20
DC_MAX_SHARDS = 1024
DC_MAX_FIELDS = 8
DC_MAX_SRC_SHARDS = 16
DC_REPACK_NOALLOC_WS_BYTES = 8 << 20
DC_MAX_VOCAB = 1 << 24
DC_MAX_DIM = 65536
DC_MAX_TOP = 64
DC_MAX_HEAD_ROWS = 1 << 22
DC_MAX_TENSORS = 65536
DC_STATE_BLOCK = 256
DC_NO_TOKEN = -1

DC_OK = 0
DC_ERR_INVALID_ARG = 1
DC_ERR_NOT_DIVISIBLE = 2
DC_ERR_UNSUPPORTED_SIZE = 3
DC_ERR_WORKSPACE = 4
DC_ERR_HIP = 5
DC_ERR_SEQ_EXCEEDS_BUDGET = 6
DC_ERR_ZERO_LENGTH_SEQ = 7
DC_ERR_OVERFLOW = 8
DC_ERR_BAD_LAYOUT = 9
DC_ERR_TOKEN_RANGE = 10

DC_F32, DC_BF16, DC_F16, DC_E4M3 = range(4)

EXPORTS = ("dc_workspace_bytes", "dc_balance", "dc_group_advantage", "dc_plan", "dc_gather",
           "dc_repack", "dc_scatter_workspace_bytes", "dc_scatter", "dc_gae", "dc_balance_group_advantage",
           "dc_gather_advantage", "dc_balance_workspace_bytes", "dc_balance_ws", "dc_repack_noalloc", "dc_balance_plan_group_advantage", "dc_gather_timed",
           "dc_token_logprob_workspace_bytes", "dc_token_logprob", "dc_token_logprob_backward",
           "dc_head_logprob_workspace_bytes", "dc_head_logprob", "dc_head_logprob_backward_workspace_bytes", "dc_head_logprob_backward",
           "dc_residual_norm", "dc_residual_norm_backward_workspace_bytes", "dc_residual_norm_backward",
           "dc_embedding", "dc_embedding_backward_workspace_bytes", "dc_embedding_backward",
           "dc_adamw_table_bytes", "dc_adamw_table", "dc_adamw", "dc_strerror")


class dc_params(C.Structure):
    _fields_ = [("n_seq", C.c_int32), ("n_shards", C.c_int32), ("cap", C.c_int32),
                ("align_tokens", C.c_int32), ("token_budget", C.c_int64), ("eps", C.c_double),
                ("ddof", C.c_int32), ("reserved", C.c_int32)]


class dc_source(C.Structure):
    _fields_ = [("n_src_shards", C.c_int32), ("reserved", C.c_int32),
                ("shard_seq_off", C.POINTER(C.c_int32)), ("shard_tokens", C.POINTER(C.c_int64)),
                ("d_src_tok_off", C.c_void_p)]


class dc_field(C.Structure):
    _fields_ = [("src_base", C.POINTER(C.c_void_p)), ("d_dst", C.c_void_p),
                ("elem_bytes", C.c_int32), ("reserved", C.c_int32)]


class dc_matrix(C.Structure):
    _fields_ = [("d_data", C.c_void_p), ("n_rows", C.c_int64), ("n_cols", C.c_int64), ("row_stride", C.c_int64),
                ("type", C.c_int32), ("reserved", C.c_int32)]


class dc_norm_params(C.Structure):
    _fields_ = [("eps", C.c_double), ("residual_scale", C.c_double), ("block_scale", C.c_double),
                ("gate_rows", C.c_int32), ("reserved", C.c_int32)]


class dc_adamw_tensor(C.Structure):
    _fields_ = [("d_param", C.c_void_p), ("d_master", C.c_void_p), ("d_grad", C.c_void_p), ("d_exp_avg", C.c_void_p),
                ("d_exp_avg_sq", C.c_void_p), ("d_exp_avg_scale", C.c_void_p), ("d_exp_avg_sq_scale", C.c_void_p),
                ("n", C.c_int64), ("weight_decay", C.c_double), ("param_type", C.c_int32), ("grad_type", C.c_int32),
                ("state_type", C.c_int32), ("reserved", C.c_int32)]


class dc_adamw_params(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double),
                ("step", C.c_int64)]


class DcError(RuntimeError):
    def __init__(self, code: int, where: str):
        super().__init__(f"{where}: {strerror(code)} (dc_status {code})")
        self.code = code


_lib = None


def load() -> C.CDLL:
    """Load libdc.so.  Raises if the HIP library has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2507_13833_amd.build` (hipcc, gfx950); there is no fallback")
        lib = C.CDLL(LIB_PATH)
        lib.dc_workspace_bytes.restype = C.c_size_t
        lib.dc_workspace_bytes.argtypes = [C.POINTER(dc_params), C.c_int64]
        lib.dc_strerror.restype = C.c_char_p
        lib.dc_strerror.argtypes = [C.c_int]
        vp = C.c_void_p
        lib.dc_balance.restype = C.c_int
        lib.dc_balance.argtypes = [C.POINTER(dc_params), vp, vp, vp, vp, vp, vp, vp]
        lib.dc_balance_workspace_bytes.restype = C.c_size_t
        lib.dc_balance_workspace_bytes.argtypes = [C.POINTER(dc_params)]
        lib.dc_balance_ws.restype = C.c_int
        lib.dc_balance_ws.argtypes = [C.POINTER(dc_params), vp, vp, vp, vp, vp, vp, C.c_size_t, vp, vp]
        lib.dc_group_advantage.restype = C.c_int
        lib.dc_group_advantage.argtypes = [C.POINTER(dc_params), C.POINTER(dc_source), vp, vp, vp, C.c_int32,
                                           C.POINTER(vp), vp, C.POINTER(vp), vp, vp]
        lib.dc_plan.restype = C.c_int
        lib.dc_plan.argtypes = [C.POINTER(dc_params), C.POINTER(dc_source), vp, vp, vp, C.c_int64,
                                vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp, vp]
        lib.dc_gather.restype = C.c_int
        lib.dc_gather.argtypes = [C.POINTER(dc_params), C.POINTER(dc_source), C.POINTER(dc_field), C.c_int32,
                                  C.c_int64, vp, vp, C.c_size_t, vp, vp]
        lib.dc_gather_timed.restype = C.c_int
        lib.dc_gather_timed.argtypes = [C.POINTER(dc_params), C.POINTER(dc_source), C.POINTER(dc_field), C.c_int32,
                                        C.c_int64, vp, vp, C.c_size_t, vp, vp, vp, vp]
        lib.dc_gather_advantage.restype = C.c_int
        lib.dc_gather_advantage.argtypes = [C.POINTER(dc_params), C.POINTER(dc_source), C.POINTER(dc_field), C.c_int32,
                                            C.c_int32, vp, vp, vp, C.c_int64, vp, vp, C.c_size_t, vp, vp]
        lib.dc_repack.restype = C.c_int
        lib.dc_repack.argtypes = [C.POINTER(dc_params), C.POINTER(dc_source), vp, vp, vp,
                                  C.POINTER(dc_field), C.c_int32, C.c_int64,
                                  vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp, vp]
        lib.dc_repack_noalloc.restype = C.c_int
        lib.dc_repack_noalloc.argtypes = [C.POINTER(dc_params), C.POINTER(dc_source), vp, vp, vp,
                                          C.POINTER(dc_field), C.c_int32, C.c_int64,
                                          vp, vp, vp, vp, vp, vp, vp, vp]
        lib.dc_scatter_workspace_bytes.restype = C.c_size_t
        lib.dc_scatter_workspace_bytes.argtypes = [C.POINTER(dc_params), C.POINTER(dc_source)]
        lib.dc_scatter.restype = C.c_int
        lib.dc_scatter.argtypes = [C.POINTER(dc_params), C.POINTER(dc_source), vp, vp, C.POINTER(dc_field), C.c_int32,
                                   C.c_int64, vp, vp, C.c_size_t, vp, vp]
        lib.dc_gae.restype = C.c_int
        lib.dc_gae.argtypes = [C.POINTER(dc_params), C.POINTER(dc_source), vp, vp, C.POINTER(vp), C.POINTER(vp),
                               C.POINTER(vp), C.POINTER(vp), C.c_double, C.c_double, C.c_double,
                               C.POINTER(vp), C.POINTER(vp), vp, vp]
        lib.dc_balance_group_advantage.restype = C.c_int
        lib.dc_balance_group_advantage.argtypes = [C.POINTER(dc_params), C.POINTER(dc_source), vp, vp, vp, vp, vp, vp, vp,
                                                   C.c_int32, C.POINTER(vp), vp, C.POINTER(vp), vp, vp]
        lib.dc_balance_plan_group_advantage.restype = C.c_int
        lib.dc_balance_plan_group_advantage.argtypes = [C.POINTER(dc_params), C.POINTER(dc_source), vp, vp, vp, vp, vp, vp, vp,
                                                        C.c_int32, C.POINTER(vp), vp, C.POINTER(vp), C.c_int64,
                                                        vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp, vp]
        mp = C.POINTER(dc_matrix)
        lib.dc_token_logprob_workspace_bytes.restype = C.c_size_t
        lib.dc_token_logprob_workspace_bytes.argtypes = [mp, C.c_int32]
        lib.dc_token_logprob.restype = C.c_int
        lib.dc_token_logprob.argtypes = [mp, C.c_double, vp, vp, C.c_int32, vp, vp, vp, vp, vp, vp, C.c_size_t, vp, vp]
        lib.dc_token_logprob_backward.restype = C.c_int
        lib.dc_token_logprob_backward.argtypes = [mp, C.c_double, vp, vp, vp, vp, vp, vp, mp, vp, vp]
        lib.dc_head_logprob_workspace_bytes.restype = C.c_size_t
        lib.dc_head_logprob_workspace_bytes.argtypes = [mp, mp, C.c_int32]
        lib.dc_head_logprob.restype = C.c_int
        lib.dc_head_logprob.argtypes = [mp, mp, C.c_double, vp, vp, C.c_int32, vp, vp, vp, vp, vp, vp, C.c_size_t, vp, vp]
        lib.dc_head_logprob_backward_workspace_bytes.restype = C.c_size_t
        lib.dc_head_logprob_backward_workspace_bytes.argtypes = [mp, mp, mp]
        lib.dc_head_logprob_backward.restype = C.c_int
        lib.dc_head_logprob_backward.argtypes = [mp, mp, C.c_double, vp, vp, vp, vp, vp, vp, mp, C.c_int32, mp, vp, C.c_size_t, vp, vp]
        np_ = C.POINTER(dc_norm_params)
        lib.dc_residual_norm.restype = C.c_int
        lib.dc_residual_norm.argtypes = [mp, mp, mp, mp, mp, np_, mp, mp, vp, vp]
        lib.dc_residual_norm_backward_workspace_bytes.restype = C.c_size_t
        lib.dc_residual_norm_backward_workspace_bytes.argtypes = [mp]
        lib.dc_residual_norm_backward.restype = C.c_int
        lib.dc_residual_norm_backward.argtypes = [mp, mp, mp, mp, mp, np_, vp, mp, mp, mp, mp, C.c_int32, mp, mp, mp, vp, C.c_size_t, vp]
        lib.dc_embedding.restype = C.c_int
        lib.dc_embedding.argtypes = [mp, vp, C.c_double, mp, vp, vp]
        lib.dc_embedding_backward_workspace_bytes.restype = C.c_size_t
        lib.dc_embedding_backward_workspace_bytes.argtypes = [mp, mp]
        lib.dc_embedding_backward.restype = C.c_int
        lib.dc_embedding_backward.argtypes = [mp, vp, C.c_double, C.c_int32, mp, vp, C.c_size_t, vp, vp]
        tp = C.POINTER(dc_adamw_tensor)
        lib.dc_adamw_table_bytes.restype = C.c_size_t
        lib.dc_adamw_table_bytes.argtypes = [tp, C.c_int32]
        lib.dc_adamw_table.restype = C.c_int
        lib.dc_adamw_table.argtypes = [tp, C.c_int32, vp, C.c_size_t, vp]
        lib.dc_adamw.restype = C.c_int
        lib.dc_adamw.argtypes = [tp, C.c_int32, C.POINTER(dc_adamw_params), vp, vp, C.c_size_t, vp, vp]
        _lib = lib
    return _lib


def strerror(code: int) -> str:
    return load().dc_strerror(int(code)).decode()


def _ptr(x) -> Optional[int]:
    """Device address of a torch tensor (or pass an int / None through)."""
    if x is None or isinstance(x, int):
        return x
    if not x.is_cuda:
        raise TypeError("expected a device tensor")
    if not x.is_contiguous():
        raise TypeError("expected a contiguous tensor")
    return x.data_ptr()


_raw_stream = None


def _stream(stream) -> Optional[int]:
    if stream is None:
        # the current stream's handle without the Stream object that torch.cuda.current_stream() builds round it
        # (1.5 us of a call that takes 8)
        global _raw_stream
        if _raw_stream is None:
            import torch
            _raw_stream = torch._C._cuda_getCurrentRawStream, torch.cuda.current_device
        return _raw_stream[0](_raw_stream[1]()) or None
    if isinstance(stream, int):
        return stream or None
    return stream.cuda_stream or None


def make_params(n_seq: int, n_shards: int, token_budget: int, eps: float = 1e-6, ddof: int = 1,
                cap: int = 0, align_tokens: int = 1) -> dc_params:
    return dc_params(n_seq, n_shards, cap, align_tokens, token_budget, eps, ddof, 0)


class Source:
    """Keeps the host arrays of a dc_source alive next to the struct."""

    def __init__(self, shard_seq_off: Sequence[int], shard_tokens: Sequence[int], d_src_tok_off):
        n = len(shard_tokens)
        self._seq_off = (C.c_int32 * (n + 1))(*[int(v) for v in shard_seq_off])
        self._tokens = (C.c_int64 * n)(*[int(v) for v in shard_tokens])
        self._keep = d_src_tok_off
        self.struct = dc_source(n, 0, C.cast(self._seq_off, C.POINTER(C.c_int32)),
                                C.cast(self._tokens, C.POINTER(C.c_int64)), _ptr(d_src_tok_off))
        self.n_src_shards = n


_ARRAYS = tuple(C.c_void_p * n for n in range(DC_MAX_SRC_SHARDS + 1))       # array types by length


def _ptr_array(items: Optional[Sequence]) -> Optional[C.Array]:
    """Host array of device addresses; None (a null pointer) stays None."""
    if items is None:
        return None
    n = len(items)
    return (_ARRAYS[n] if n <= DC_MAX_SRC_SHARDS else C.c_void_p * n)(*[_ptr(t) for t in items])


class Fields:
    """Host array of dc_field built from (src tensors per rollout shard, dst tensor, elem_bytes)."""

    def __init__(self, specs: Sequence[tuple]):
        self._src_arrays = []
        self._keep = specs
        self.array = (dc_field * max(1, len(specs)))()
        for i, (srcs, dst, elem_bytes) in enumerate(specs):
            arr = _ptr_array(srcs)
            self._src_arrays.append(arr)
            self.array[i] = dc_field(C.cast(arr, C.POINTER(C.c_void_p)), _ptr(dst), int(elem_bytes), 0)
        self.n = len(specs)


def _check(rc: int, where: str) -> None:
    if rc != DC_OK:
        raise DcError(rc, where)


def dc_workspace_bytes(prm: dc_params, dst_capacity_tokens: int) -> int:
    return int(load().dc_workspace_bytes(C.byref(prm), int(dst_capacity_tokens)))


def dc_balance(prm: dc_params, d_seq_len, d_perm, d_shard_seq_off, d_shard_of_seq, d_shard_load,
               d_status, stream=None) -> None:
    _check(load().dc_balance(C.byref(prm), _ptr(d_seq_len), _ptr(d_perm), _ptr(d_shard_seq_off),
                             _ptr(d_shard_of_seq), _ptr(d_shard_load), _ptr(d_status), _stream(stream)),
           "dc_balance")


def dc_balance_workspace_bytes(prm: dc_params) -> int:
    return int(load().dc_balance_workspace_bytes(C.byref(prm)))


def dc_balance_ws(prm: dc_params, d_seq_len, d_perm, d_shard_seq_off, d_shard_of_seq, d_shard_load,
                  d_ws, ws_bytes: int, d_status, stream=None) -> None:
    _check(load().dc_balance_ws(C.byref(prm), _ptr(d_seq_len), _ptr(d_perm), _ptr(d_shard_seq_off),
                                _ptr(d_shard_of_seq), _ptr(d_shard_load), _ptr(d_ws), int(ws_bytes), _ptr(d_status),
                                _stream(stream)),
           "dc_balance_ws")


def dc_group_advantage(prm: dc_params, src: Source, d_seq_len, d_reward, d_group_off, n_groups: int,
                       mask_src: Optional[Sequence], d_adv_seq, adv_tok_src: Optional[Sequence],
                       d_status, stream=None) -> None:
    _check(load().dc_group_advantage(C.byref(prm), C.byref(src.struct), _ptr(d_seq_len), _ptr(d_reward),
                                     _ptr(d_group_off), int(n_groups),
                                     _ptr_array(mask_src), _ptr(d_adv_seq), _ptr_array(adv_tok_src),
                                     _ptr(d_status), _stream(stream)),
           "dc_group_advantage")


def dc_plan(prm: dc_params, src: Source, d_seq_len, d_perm, d_shard_seq_off, dst_capacity_tokens: int,
            d_dst_tok_off, d_shard_tok_off, d_shard_mb_off, d_mb_seq_off, d_cu_seqlens, d_n_mb,
            d_ws, ws_bytes: int, d_status, stream=None) -> None:
    _check(load().dc_plan(C.byref(prm), C.byref(src.struct), _ptr(d_seq_len), _ptr(d_perm), _ptr(d_shard_seq_off),
                          int(dst_capacity_tokens), _ptr(d_dst_tok_off), _ptr(d_shard_tok_off),
                          _ptr(d_shard_mb_off), _ptr(d_mb_seq_off), _ptr(d_cu_seqlens), _ptr(d_n_mb),
                          _ptr(d_ws), int(ws_bytes), _ptr(d_status), _stream(stream)),
           "dc_plan")


def dc_gather(prm: dc_params, src: Source, fields: Fields, dst_capacity_tokens: int, d_dst_tok_off,
              d_ws, ws_bytes: int, d_status, stream=None) -> None:
    _check(load().dc_gather(C.byref(prm), C.byref(src.struct), fields.array, fields.n, int(dst_capacity_tokens),
                            _ptr(d_dst_tok_off), _ptr(d_ws), int(ws_bytes), _ptr(d_status), _stream(stream)),
           "dc_gather")


def _event(ev) -> Optional[int]:
    """Raw hipEvent_t of a torch.cuda.Event that has been recorded at least once (torch creates the HIP event at
    its first record), or of an integer handle; None stays None."""
    if ev is None:
        return None
    if isinstance(ev, int):
        return ev or None
    h = ev.cuda_event
    h = getattr(h, "value", h)
    if not h:
        raise ValueError("the event has no HIP handle yet: record it once before passing it")
    return int(h)


def dc_gather_timed(prm: dc_params, src: Source, fields: Fields, dst_capacity_tokens: int, d_dst_tok_off,
                    d_ws, ws_bytes: int, d_status, event_begins, event_ends, stream=None) -> None:
    _check(load().dc_gather_timed(C.byref(prm), C.byref(src.struct), fields.array, fields.n, int(dst_capacity_tokens),
                                  _ptr(d_dst_tok_off), _ptr(d_ws), int(ws_bytes), _ptr(d_status), _stream(stream),
                                  _event(event_begins), _event(event_ends)),
           "dc_gather_timed")


def dc_gather_advantage(prm: dc_params, src: Source, fields: Fields, mask_field: int, d_perm, d_adv_seq,
                        d_adv_tok_dst, dst_capacity_tokens: int, d_dst_tok_off, d_ws, ws_bytes: int, d_status,
                        stream=None) -> None:
    _check(load().dc_gather_advantage(C.byref(prm), C.byref(src.struct), fields.array, fields.n, int(mask_field),
                                      _ptr(d_perm), _ptr(d_adv_seq), _ptr(d_adv_tok_dst), int(dst_capacity_tokens),
                                      _ptr(d_dst_tok_off), _ptr(d_ws), int(ws_bytes), _ptr(d_status),
                                      _stream(stream)),
           "dc_gather_advantage")


def dc_repack(prm: dc_params, src: Source, d_seq_len, d_perm, d_shard_seq_off, fields: Fields,
              dst_capacity_tokens: int, d_dst_tok_off, d_shard_tok_off, d_shard_mb_off, d_mb_seq_off,
              d_cu_seqlens, d_n_mb, d_ws, ws_bytes: int, d_status, stream=None) -> None:
    _check(load().dc_repack(C.byref(prm), C.byref(src.struct), _ptr(d_seq_len), _ptr(d_perm), _ptr(d_shard_seq_off),
                            fields.array, fields.n, int(dst_capacity_tokens), _ptr(d_dst_tok_off),
                            _ptr(d_shard_tok_off), _ptr(d_shard_mb_off), _ptr(d_mb_seq_off), _ptr(d_cu_seqlens),
                            _ptr(d_n_mb), _ptr(d_ws), int(ws_bytes), _ptr(d_status), _stream(stream)),
           "dc_repack")


def dc_repack_noalloc(prm: dc_params, src: Source, d_seq_len, d_perm, d_shard_seq_off, fields: Fields,
                      dst_capacity_tokens: int, d_dst_tok_off, d_shard_tok_off, d_shard_mb_off, d_mb_seq_off,
                      d_cu_seqlens, d_n_mb, d_status, stream=None) -> None:
    _check(load().dc_repack_noalloc(C.byref(prm), C.byref(src.struct), _ptr(d_seq_len), _ptr(d_perm),
                                    _ptr(d_shard_seq_off), fields.array, fields.n, int(dst_capacity_tokens),
                                    _ptr(d_dst_tok_off), _ptr(d_shard_tok_off), _ptr(d_shard_mb_off),
                                    _ptr(d_mb_seq_off), _ptr(d_cu_seqlens), _ptr(d_n_mb), _ptr(d_status),
                                    _stream(stream)),
           "dc_repack_noalloc")


def dc_scatter_workspace_bytes(prm: dc_params, src: Source) -> int:
    return int(load().dc_scatter_workspace_bytes(C.byref(prm), C.byref(src.struct)))


def dc_scatter(prm: dc_params, src: Source, d_seq_len, d_perm, fields: Fields, dst_capacity_tokens: int,
               d_dst_tok_off, d_ws, ws_bytes: int, d_status, stream=None) -> None:
    """fields: as for dc_gather, with the roles swapped (dst = training arena read, srcs = rollout buffers written)."""
    _check(load().dc_scatter(C.byref(prm), C.byref(src.struct), _ptr(d_seq_len), _ptr(d_perm), fields.array, fields.n,
                             int(dst_capacity_tokens), _ptr(d_dst_tok_off), _ptr(d_ws), int(ws_bytes),
                             _ptr(d_status), _stream(stream)),
           "dc_scatter")


def dc_gae(prm: dc_params, src: Source, d_seq_len, d_reward, value_src: Sequence, mask_src: Sequence,
           logp_src: Optional[Sequence], ref_src: Optional[Sequence], gamma: float, lam: float, kl_coef: float,
           adv_tok_src: Sequence, ret_tok_src: Sequence, d_status, stream=None) -> None:
    _check(load().dc_gae(C.byref(prm), C.byref(src.struct), _ptr(d_seq_len), _ptr(d_reward), _ptr_array(value_src),
                         _ptr_array(mask_src), _ptr_array(logp_src), _ptr_array(ref_src), float(gamma), float(lam),
                         float(kl_coef), _ptr_array(adv_tok_src), _ptr_array(ret_tok_src), _ptr(d_status),
                         _stream(stream)),
           "dc_gae")


def dc_balance_group_advantage(prm: dc_params, src: Source, d_seq_len, d_perm, d_shard_seq_off, d_shard_of_seq,
                               d_shard_load, d_reward, d_group_off, n_groups: int, mask_src: Optional[Sequence],
                               d_adv_seq, adv_tok_src: Optional[Sequence], d_status, stream=None) -> None:
    _check(load().dc_balance_group_advantage(
        C.byref(prm), C.byref(src.struct), _ptr(d_seq_len), _ptr(d_perm), _ptr(d_shard_seq_off), _ptr(d_shard_of_seq),
        _ptr(d_shard_load), _ptr(d_reward), _ptr(d_group_off), int(n_groups),
        _ptr_array(mask_src), _ptr(d_adv_seq), _ptr_array(adv_tok_src), _ptr(d_status), _stream(stream)),
        "dc_balance_group_advantage")


def dc_balance_plan_group_advantage(prm: dc_params, src: Source, d_seq_len, d_perm, d_shard_seq_off, d_shard_of_seq,
                                    d_shard_load, d_reward, d_group_off, n_groups: int, mask_src: Optional[Sequence],
                                    d_adv_seq, adv_tok_src: Optional[Sequence], dst_capacity_tokens: int, d_dst_tok_off,
                                    d_shard_tok_off, d_shard_mb_off, d_mb_seq_off, d_cu_seqlens, d_n_mb, d_ws,
                                    ws_bytes: int, d_status, stream=None) -> None:
    _check(load().dc_balance_plan_group_advantage(
        C.byref(prm), C.byref(src.struct), _ptr(d_seq_len), _ptr(d_perm), _ptr(d_shard_seq_off), _ptr(d_shard_of_seq),
        _ptr(d_shard_load), _ptr(d_reward), _ptr(d_group_off), int(n_groups),
        _ptr_array(mask_src), _ptr(d_adv_seq), _ptr_array(adv_tok_src), int(dst_capacity_tokens), _ptr(d_dst_tok_off),
        _ptr(d_shard_tok_off), _ptr(d_shard_mb_off), _ptr(d_mb_seq_off), _ptr(d_cu_seqlens), _ptr(d_n_mb),
        _ptr(d_ws), int(ws_bytes), _ptr(d_status), _stream(stream)),
        "dc_balance_plan_group_advantage")


# ---- the actor's update on the packed training layout ----

@functools.lru_cache(maxsize=None)
def _dtypes() -> dict:
    import torch
    return {name: getattr(torch, name) for name in ("float32", "bfloat16", "float16", "float8_e4m3fn", "int32", "uint8")}


@functools.lru_cache(maxsize=None)
def _types() -> dict:
    d = _dtypes()
    return {d["float32"]: DC_F32, d["bfloat16"]: DC_BF16, d["float16"]: DC_F16, d["float8_e4m3fn"]: DC_E4M3}


def _dc_type(dtype) -> int:
    try:
        return _types()[dtype]
    except KeyError:
        raise TypeError(f"no dc_type for {dtype}") from None


def make_matrix(t) -> dc_matrix:
    """dc_matrix of a device tensor [rows, columns] whose columns are neighbours; rows may be any distance apart from the
    number of columns up.  The struct holds the address only: the tensor has to outlive the calls."""
    if not t.is_cuda:
        raise TypeError("expected a device tensor")
    if t.dim() != 2:
        raise TypeError("expected a tensor of two dimensions")
    rows, cols = t.shape
    stride, step = t.stride()
    if rows <= 1:
        stride = cols
    if (step != 1 and cols > 1) or stride < cols:
        raise TypeError("expected rows of neighbouring elements that do not overlap")
    return dc_matrix(t.data_ptr() or None, rows, cols, stride, _dc_type(t.dtype), 0)


def _vec(x, n: int, dtype: str, what: str) -> Optional[int]:
    """Device address of a tensor of at least n elements of one type, both checked (an int or None passes through)."""
    if x is None or isinstance(x, int):
        return x
    # (one test where all is well: a call of the smallest sizes takes as long on the host as on the device)
    if x.is_cuda and x.dtype is _dtypes()[dtype] and x.is_contiguous() and x.numel() >= n:
        return x.data_ptr()
    if x.dtype is not _dtypes()[dtype]:
        raise TypeError(f"{what}: expected {dtype}, got {x.dtype}")
    if x.numel() < n:
        raise ValueError(f"{what}: {x.numel()} elements, {n} are needed")
    return _ptr(x)


_F32, _I32, _U8 = "float32", "int32", "uint8"


def dc_token_logprob_workspace_bytes(logits: dc_matrix, n_top: int) -> int:
    return int(load().dc_token_logprob_workspace_bytes(C.byref(logits), int(n_top)))


def dc_token_logprob(logits: dc_matrix, temperature: float, d_token, d_mask, n_top: int, d_logprob, d_row_stat, d_entropy,
                     d_top_token, d_top_logprob, d_ws, ws_bytes: int, d_status, stream=None) -> None:
    n, k = logits.n_rows, int(n_top)
    _check(load().dc_token_logprob(C.byref(logits), float(temperature), _vec(d_token, n, _I32, "d_token"),
                                   _vec(d_mask, n, _U8, "d_mask"), k, _vec(d_logprob, n, _F32, "d_logprob"),
                                   _vec(d_row_stat, 2 * n, _F32, "d_row_stat"), _vec(d_entropy, n, _F32, "d_entropy"),
                                   _vec(d_top_token, n * k, _I32, "d_top_token"),
                                   _vec(d_top_logprob, n * k, _F32, "d_top_logprob"), _ptr(d_ws), int(ws_bytes),
                                   _ptr(d_status), _stream(stream)),
           "dc_token_logprob")


def dc_token_logprob_backward(logits: dc_matrix, temperature: float, d_token, d_mask, d_row_stat, d_entropy, d_grad_logprob,
                              d_grad_entropy, grad_logits: dc_matrix, d_status, stream=None) -> None:
    n = logits.n_rows
    _check(load().dc_token_logprob_backward(C.byref(logits), float(temperature), _vec(d_token, n, _I32, "d_token"),
                                            _vec(d_mask, n, _U8, "d_mask"), _vec(d_row_stat, 2 * n, _F32, "d_row_stat"),
                                            _vec(d_entropy, n, _F32, "d_entropy"),
                                            _vec(d_grad_logprob, n, _F32, "d_grad_logprob"),
                                            _vec(d_grad_entropy, n, _F32, "d_grad_entropy"), C.byref(grad_logits),
                                            _ptr(d_status), _stream(stream)),
           "dc_token_logprob_backward")


def _ref(m: Optional[dc_matrix]):
    """A matrix by reference; None (a null pointer) stays None."""
    return None if m is None else C.byref(m)


def dc_head_logprob_workspace_bytes(hidden: dc_matrix, weight: dc_matrix, n_top: int) -> int:
    return int(load().dc_head_logprob_workspace_bytes(C.byref(hidden), C.byref(weight), int(n_top)))


def dc_head_logprob(hidden: dc_matrix, weight: dc_matrix, temperature: float, d_token, d_mask, n_top: int, d_logprob, d_row_stat,
                    d_entropy, d_top_token, d_top_logprob, d_ws, ws_bytes: int, d_status, stream=None) -> None:
    n, k = hidden.n_rows, int(n_top)
    _check(load().dc_head_logprob(C.byref(hidden), C.byref(weight), float(temperature), _vec(d_token, n, _I32, "d_token"),
                                  _vec(d_mask, n, _U8, "d_mask"), k, _vec(d_logprob, n, _F32, "d_logprob"),
                                  _vec(d_row_stat, 2 * n, _F32, "d_row_stat"), _vec(d_entropy, n, _F32, "d_entropy"),
                                  _vec(d_top_token, n * k, _I32, "d_top_token"),
                                  _vec(d_top_logprob, n * k, _F32, "d_top_logprob"), _ptr(d_ws), int(ws_bytes),
                                  _ptr(d_status), _stream(stream)),
           "dc_head_logprob")


def dc_head_logprob_backward_workspace_bytes(hidden: dc_matrix, weight: dc_matrix, grad_weight: Optional[dc_matrix]) -> int:
    return int(load().dc_head_logprob_backward_workspace_bytes(C.byref(hidden), C.byref(weight), _ref(grad_weight)))


def dc_head_logprob_backward(hidden: dc_matrix, weight: dc_matrix, temperature: float, d_token, d_mask, d_row_stat, d_entropy,
                             d_grad_logprob, d_grad_entropy, grad_hidden: Optional[dc_matrix], accumulate: bool,
                             grad_weight: Optional[dc_matrix], d_ws, ws_bytes: int, d_status, stream=None) -> None:
    n = hidden.n_rows
    _check(load().dc_head_logprob_backward(C.byref(hidden), C.byref(weight), float(temperature), _vec(d_token, n, _I32, "d_token"),
                                           _vec(d_mask, n, _U8, "d_mask"), _vec(d_row_stat, 2 * n, _F32, "d_row_stat"),
                                           _vec(d_entropy, n, _F32, "d_entropy"),
                                           _vec(d_grad_logprob, n, _F32, "d_grad_logprob"),
                                           _vec(d_grad_entropy, n, _F32, "d_grad_entropy"), _ref(grad_hidden),
                                           int(bool(accumulate)), _ref(grad_weight), _ptr(d_ws), int(ws_bytes), _ptr(d_status),
                                           _stream(stream)),
           "dc_head_logprob_backward")


def make_norm(eps: float = 1e-6, residual_scale: float = 1.0, block_scale: float = 1.0,
              gate_rows: bool = False) -> dc_norm_params:
    return dc_norm_params(eps, residual_scale, block_scale, int(bool(gate_rows)), 0)


def dc_residual_norm(block: dc_matrix, post_weight: Optional[dc_matrix], gate: Optional[dc_matrix], residual: dc_matrix,
                     pre_weight: Optional[dc_matrix], prm: dc_norm_params, residual_out: dc_matrix, out: Optional[dc_matrix],
                     d_row_stat=None, stream=None) -> None:
    _check(load().dc_residual_norm(C.byref(block), _ref(post_weight), _ref(gate), C.byref(residual), _ref(pre_weight),
                                   C.byref(prm), C.byref(residual_out), _ref(out),
                                   _vec(d_row_stat, 2 * block.n_rows, _F32, "d_row_stat"), _stream(stream)),
           "dc_residual_norm")


def dc_residual_norm_backward_workspace_bytes(block: dc_matrix) -> int:
    return int(load().dc_residual_norm_backward_workspace_bytes(C.byref(block)))


def dc_residual_norm_backward(block: dc_matrix, post_weight: Optional[dc_matrix], gate: Optional[dc_matrix],
                              residual_out: Optional[dc_matrix], pre_weight: Optional[dc_matrix], prm: dc_norm_params, d_row_stat,
                              grad_residual_out: Optional[dc_matrix], grad_out: Optional[dc_matrix], grad_block: Optional[dc_matrix],
                              grad_residual: Optional[dc_matrix], accumulate: bool, grad_post_weight: Optional[dc_matrix],
                              grad_gate: Optional[dc_matrix], grad_pre_weight: Optional[dc_matrix], d_ws, ws_bytes: int,
                              stream=None) -> None:
    _check(load().dc_residual_norm_backward(C.byref(block), _ref(post_weight), _ref(gate), _ref(residual_out), _ref(pre_weight),
                                            C.byref(prm), _vec(d_row_stat, 2 * block.n_rows, _F32, "d_row_stat"),
                                            _ref(grad_residual_out), _ref(grad_out), _ref(grad_block), _ref(grad_residual),
                                            int(bool(accumulate)), _ref(grad_post_weight), _ref(grad_gate), _ref(grad_pre_weight),
                                            _ptr(d_ws), int(ws_bytes), _stream(stream)),
           "dc_residual_norm_backward")


def dc_embedding(weight: dc_matrix, d_token, scale: float, out: dc_matrix, d_status, stream=None) -> None:
    _check(load().dc_embedding(C.byref(weight), _vec(d_token, out.n_rows, _I32, "d_token"), float(scale),
                               C.byref(out), _ptr(d_status), _stream(stream)),
           "dc_embedding")


def dc_embedding_backward_workspace_bytes(grad_out: dc_matrix, grad_weight: dc_matrix) -> int:
    return int(load().dc_embedding_backward_workspace_bytes(C.byref(grad_out), C.byref(grad_weight)))


def dc_embedding_backward(grad_out: dc_matrix, d_token, scale: float, accumulate: bool, grad_weight: dc_matrix, d_ws,
                          ws_bytes: int, d_status, stream=None) -> None:
    _check(load().dc_embedding_backward(C.byref(grad_out), _vec(d_token, grad_out.n_rows, _I32, "d_token"), float(scale),
                                        int(bool(accumulate)), C.byref(grad_weight), _ptr(d_ws), int(ws_bytes),
                                        _ptr(d_status), _stream(stream)),
           "dc_embedding_backward")


class AdamwTensors:
    """Host array of dc_adamw_tensor, and the tensors it points into, which it keeps whatever becomes of the dicts.  items:
    dicts with param, grad, exp_avg, exp_avg_sq and, where there are any, master, exp_avg_scale, exp_avg_sq_scale,
    weight_decay."""

    _SCALES = ("exp_avg_scale", "exp_avg_sq_scale")

    def __init__(self, items: Sequence[dict]):
        items = self._keep = [dict(it) for it in items]
        self.n = len(items)
        self.array = (dc_adamw_tensor * max(1, self.n))()
        for i, it in enumerate(items):
            param, n = it["param"], it["param"].numel()
            blocks = -(-n // DC_STATE_BLOCK)
            for name in ("master", "grad", "exp_avg", "exp_avg_sq", *self._SCALES):
                t = it.get(name)
                if t is not None and t.numel() != (blocks if name in self._SCALES else n):
                    raise ValueError(f"tensor {i}: {name} has {t.numel()} elements, param {n}")
                if t is not None and (name == "master" or name in self._SCALES) and _dc_type(t.dtype) != DC_F32:
                    raise TypeError(f"tensor {i}: {name} is not float32")
            if _dc_type(it["exp_avg"].dtype) != _dc_type(it["exp_avg_sq"].dtype):
                raise TypeError(f"tensor {i}: the two states differ in type")
            at = lambda name: (_ptr(it[name]) or None) if it.get(name) is not None else None  # noqa: E731
            self.array[i] = dc_adamw_tensor(
                at("param"), at("master"), at("grad"), at("exp_avg"), at("exp_avg_sq"), at("exp_avg_scale"),
                at("exp_avg_sq_scale"), n, float(it.get("weight_decay", 0.0)), _dc_type(param.dtype),
                _dc_type(it["grad"].dtype), _dc_type(it["exp_avg"].dtype), 0)


def make_adamw(lr: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8, step: int = 1) -> dc_adamw_params:
    return dc_adamw_params(lr, beta1, beta2, eps, step)


def dc_adamw_table_bytes(tensors: AdamwTensors) -> int:
    return int(load().dc_adamw_table_bytes(tensors.array, tensors.n))


def dc_adamw_table(tensors: AdamwTensors, d_table, table_bytes: int, stream=None) -> None:
    _check(load().dc_adamw_table(tensors.array, tensors.n, _ptr(d_table), int(table_bytes), _stream(stream)),
           "dc_adamw_table")


def dc_adamw(tensors: AdamwTensors, prm: dc_adamw_params, d_grad_scale, d_table, table_bytes: int, d_status,
             stream=None) -> None:
    _check(load().dc_adamw(tensors.array, tensors.n, C.byref(prm), _vec(d_grad_scale, 1, _F32, "d_grad_scale"),
                           _ptr(d_table), int(table_bytes), _ptr(d_status), _stream(stream)),
           "dc_adamw")
