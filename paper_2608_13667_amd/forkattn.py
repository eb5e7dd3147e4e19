"""ctypes binding of libforkattn.so (include/forkattn.h), argument marshalling only.

Every step of the computation runs in the library's HIP kernels; this module
turns torch device tensors into raw pointers and the current torch stream into a
hipStream_t.  Importing it fails loudly when the library has not been built.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libforkattn.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is not built: run paper_2608_13667_amd.build.build() "
                      "(or __graft_entry__.build()) first")
_lib = C.CDLL(LIB_PATH)

FKA_OK, FKA_ERR_INVALID_ARG, FKA_ERR_UNSUPPORTED, FKA_ERR_HIP, FKA_ERR_NOMEM = 0, -1, -2, -3, -4
ERR_SUFFIX_CLAMPED, ERR_APPEND_NO_ROOM, ERR_BAD_PAGE, ERR_BAD_SCHEDULE = 1, 2, 4, 8


class Heads(C.Structure):
    _fields_ = [("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("softmax_scale", C.c_float)]


class ContigDesc(C.Structure):
    _fields_ = [("n_branches", C.c_int32), ("prefix_len", C.c_int32), ("suffix_cap", C.c_int32),
                ("max_suffix_len", C.c_int32), ("share_prefix", C.c_int32), ("rounds", C.c_int32),
                ("blocks", C.c_int32)]


class PagedDesc(C.Structure):
    _fields_ = [("n_seqs", C.c_int32), ("n_groups", C.c_int32), ("page_size", C.c_int32),
                ("max_pages_per_seq", C.c_int32), ("n_pool_pages", C.c_int32), ("max_suffix_len", C.c_int32),
                ("share_prefix", C.c_int32), ("rounds", C.c_int32), ("blocks", C.c_int32)]


class PrefillDesc(C.Structure):
    _fields_ = [("n_branches", C.c_int32), ("n_tokens", C.c_int32), ("prefix_len", C.c_int32),
                ("suffix_cap", C.c_int32), ("max_suffix_len", C.c_int32), ("blocks", C.c_int32)]


class PrefillPagedDesc(C.Structure):
    _fields_ = [("n_branches", C.c_int32), ("n_tokens", C.c_int32), ("prefix_len", C.c_int32),
                ("page_size", C.c_int32), ("max_pages_per_seq", C.c_int32), ("n_pool_pages", C.c_int32),
                ("max_suffix_len", C.c_int32), ("blocks", C.c_int32)]


class PlanInfo(C.Structure):
    _fields_ = [("n_items", C.c_int32), ("n_units", C.c_int32), ("waves_per_block", C.c_int32),
                ("n_blocks", C.c_int32), ("rounds", C.c_int32), ("n_slots", C.c_int32), ("slot_rows", C.c_int32),
                ("static_split", C.c_int32), ("units_per_block", C.c_int32),
                ("workspace_bytes", C.c_size_t)]


class Slot(C.Structure):
    _fields_ = [("slot", C.c_int32), ("seq0", C.c_int32), ("nseq", C.c_int32), ("kv_head", C.c_int32),
                ("rows", C.c_int32), ("prefix_begin", C.c_int32), ("prefix_end", C.c_int32),
                ("suffix_begin", C.c_int32), ("suffix_end", C.c_int32), ("prefix_len", C.c_int32)]


class RotateDesc(C.Structure):
    _fields_ = [("n_seqs", C.c_int32), ("n_tokens", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("rotary_dim", C.c_int32), ("interleaved", C.c_int32), ("max_len", C.c_int32),
                ("advance", C.c_int32), ("eps", C.c_float), ("q_stride", C.c_int64), ("k_stride", C.c_int64),
                ("v_stride", C.c_int64)]


class MxDesc(C.Structure):
    _fields_ = [("n_seqs", C.c_int32), ("n_groups", C.c_int32), ("max_tiles_per_group", C.c_int32),
                ("n_pool_tiles", C.c_int32), ("suffix_cap", C.c_int32), ("max_suffix_len", C.c_int32), ("blocks", C.c_int32)]


MX_TILE = 128  # tokens of a 4-bit tile

_vp = C.c_void_p
_sig = {
    "fka_version": ([], C.c_int),
    "fka_last_error": ([], C.c_char_p),
    "fka_plan_create_contig": ([C.POINTER(Heads), C.POINTER(ContigDesc), C.POINTER(_vp)], C.c_int),
    "fka_plan_create_paged": ([C.POINTER(Heads), C.POINTER(PagedDesc), _vp, _vp, C.POINTER(_vp)], C.c_int),
    "fka_fork_decode": ([_vp] * 10, C.c_int),
    "fka_append_kv": ([_vp] * 7, C.c_int),
    "fka_fork_step": ([_vp] * 12, C.c_int),
    "fka_fork_decode_paged": ([_vp] * 9, C.c_int),
    "fka_fork_step_paged": ([_vp] * 11, C.c_int),
    "fka_append_kv_paged": ([_vp] * 8, C.c_int),
    "fka_gather_paged": ([_vp, C.c_int32, _vp, _vp, _vp, C.c_int32, _vp, _vp, _vp], C.c_int),
    "fka_gather_paged_range": ([_vp, C.c_int32, C.c_int32, C.c_int32, _vp, _vp, _vp, _vp, _vp, _vp], C.c_int),
    "fka_plan_get_info": ([_vp, C.POINTER(PlanInfo)], C.c_int),
    "fka_plan_create_prefill": ([C.POINTER(Heads), C.POINTER(PrefillDesc), C.POINTER(_vp)], C.c_int),
    "fka_prefill": ([_vp] * 10, C.c_int),
    "fka_plan_create_prefill_paged": ([C.POINTER(Heads), C.POINTER(PrefillPagedDesc), C.POINTER(_vp)], C.c_int),
    "fka_prefill_paged": ([_vp] * 9, C.c_int),
    "fka_fork_decode_noalloc": ([C.POINTER(Heads), C.POINTER(ContigDesc)] + [_vp] * 10, C.c_int),
    "fka_plan_slots": ([_vp, _vp, _vp, C.c_int32, C.POINTER(C.c_int32)], C.c_int),
    "fka_partials": ([_vp] * 10, C.c_int),
    "fka_partials_paged": ([_vp] * 9, C.c_int),
    "fka_lse_merge": ([C.c_int32, C.c_int32, C.c_int32, _vp, _vp, _vp, _vp, _vp], C.c_int),
    "fka_plan_device_error": ([_vp, C.POINTER(C.c_int32)], C.c_int),
    "fka_read_probe": ([_vp, C.c_size_t, C.c_int32, C.c_int32, C.c_int32, _vp, _vp], C.c_int),
    "fka_plan_destroy": ([_vp], None),
    "fka_pool_create": ([C.c_int32, C.POINTER(_vp)], C.c_int),
    "fka_pool_destroy": ([_vp], None),
    "fka_pool_free_pages": ([_vp], C.c_int32),
    "fka_pool_refcount": ([_vp, C.c_int32], C.c_int32),
    "fka_pool_alloc": ([_vp, C.c_int32, _vp], C.c_int),
    "fka_pool_retain": ([_vp, C.c_int32, _vp], C.c_int),
    "fka_pool_release": ([_vp, C.c_int32, _vp], C.c_int),
    "fka_pool_fork": ([_vp, _vp, C.c_int32, _vp, C.c_int32, C.c_int32, C.c_int32], C.c_int),
    "fka_pool_reserve": ([_vp, _vp, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.POINTER(C.c_int32)], C.c_int),
    "fka_pool_drop": ([_vp, _vp, C.c_int32, C.c_int32], C.c_int),
    "fka_pool_promote": ([_vp, _vp, C.c_int32, C.c_int32, C.c_int32, C.c_int32, _vp, C.POINTER(C.c_int32)],
                         C.c_int),
    "fka_scatter_pages": ([_vp, _vp, C.c_int32, C.c_int32, _vp, C.c_int32, C.c_int32, C.c_int32, _vp, _vp, _vp, _vp],
                          C.c_int),
    "fka_rotate_append": ([C.POINTER(RotateDesc)] + [_vp] * 10 + [C.c_int32, _vp, _vp, _vp], C.c_int),
    "fka_rotate_append_paged": ([C.POINTER(RotateDesc)] + [_vp] * 12 + [C.c_int32, C.c_int32, _vp, _vp, _vp], C.c_int),
    "fka_mx_tile_bytes": ([C.c_int32, C.c_int32], C.c_size_t),
    "fka_mx_pack": ([C.c_int32] * 4 + [_vp, _vp, C.c_int32, _vp, _vp, C.c_int32, _vp, _vp], C.c_int),
    "fka_mx_unpack": ([C.c_int32] * 4 + [_vp, _vp, C.c_int32, _vp, _vp, C.c_int32, _vp, _vp], C.c_int),
    "fka_plan_create_mx": ([C.POINTER(Heads), C.POINTER(MxDesc), _vp, _vp, C.POINTER(_vp)], C.c_int),
    "fka_fork_decode_mx": ([_vp] * 10, C.c_int),
    "fka_fork_step_mx": ([_vp] * 12, C.c_int),
    "fka_key_weights": ([C.POINTER(Heads), C.c_int32, C.c_int32, _vp, _vp, _vp, C.c_int32, _vp, C.c_int32, C.c_float, _vp],
                        C.c_int),
    "fka_evict_bytes": ([C.c_int32, C.c_int32], C.c_size_t),
    "fka_evict": ([C.c_int32] * 6 + [_vp, _vp, C.c_int32, _vp, C.c_int32] + [_vp] * 5 + [C.c_size_t, _vp], C.c_int),
}
for _name, (_args, _res) in _sig.items():
    _f = getattr(_lib, _name)
    _f.argtypes = _args
    _f.restype = _res

EXPORTED = tuple(_sig)


class FkaError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"status {status}: {msg}")
        self.status = status


def _check(status: int):
    if status != FKA_OK:
        raise FkaError(status, _lib.fka_last_error().decode())


def last_error() -> str:
    return _lib.fka_last_error().decode()


def version() -> int:
    return _lib.fka_version()


_KIND_DTYPES = {"bf16": torch.bfloat16, "i32": torch.int32, "f32": torch.float32, "f64": torch.float64, "u8": torch.uint8}


def _p(t: Optional[torch.Tensor], kind: Optional[str] = None, device: Optional[int] = None):
    """Device pointer of a contiguous tensor on the plan's GPU, of the dtype the C ABI expects
    for this argument (bf16 q/K/V, int32 lengths and page tables, fp32 outputs)."""
    # A plain tensor on the plan's GPU passes all the checks below in one expression and goes to the
    # C call as a plain integer: 0.26 us against 0.35 with the checks in turn and a c_void_p made,
    # ten times in a step.  Anything else, and every error, goes through the checks in turn.
    if (type(t) is torch.Tensor and device is not None and t.is_cuda and t.get_device() == device
            and t.dtype is _KIND_DTYPES.get(kind) and t.is_contiguous()):
        return t.data_ptr()
    if t is None:
        return None
    if not isinstance(t, torch.Tensor):
        raise ValueError("expected a torch tensor")
    if not t.is_cuda:
        raise ValueError("tensor must be on the GPU (the library reads device memory)")
    if device is not None and t.get_device() != device:
        raise ValueError(f"tensor is on cuda:{t.get_device()}, the plan's device is cuda:{device}")
    if kind is not None and t.dtype != _KIND_DTYPES[kind]:
        raise ValueError(f"tensor must be {kind}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    return _vp(t.data_ptr())


# The current stream's handle without building a torch.cuda.Stream object (2.9 us of a call's 12);
# torch.cuda.current_stream() where this torch does not have it.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    if stream is None:
        if _raw_stream is not None and _current_device is not None and torch.cuda.is_initialized():
            return _raw_stream(_current_device())
        stream = torch.cuda.current_stream()
    return _vp(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


class Plan:
    """A fork plan: the static work schedule and the device workspace (see fka_plan_create_*)."""

    def __init__(self, handle: int, paged: bool, heads: Heads, n_seqs: int):
        self._h = _vp(handle)
        self.device = torch.cuda.current_device() if torch.cuda.is_available() else None
        self.paged = paged
        self.heads = heads
        self.n_seqs = n_seqs
        self._mx = None  # of a plan over 4-bit tiles: the pool's shape, entries of the tile table

    @classmethod
    def contig(cls, n_q_heads, n_kv_heads, head_dim, n_branches, prefix_len, suffix_cap, max_suffix_len,
               share_prefix=True, rounds=0, softmax_scale=0.0, blocks=0) -> "Plan":
        h = Heads(n_q_heads, n_kv_heads, head_dim, softmax_scale)
        d = ContigDesc(n_branches, prefix_len, suffix_cap, max_suffix_len, int(bool(share_prefix)), rounds, blocks)
        out = _vp()
        _check(_lib.fka_plan_create_contig(C.byref(h), C.byref(d), C.byref(out)))
        return cls(out.value, False, h, n_branches)

    @classmethod
    def paged_plan(cls, n_q_heads, n_kv_heads, head_dim, group_start, group_prefix_len, max_pages_per_seq,
                   n_pool_pages, max_suffix_len, share_prefix=True, rounds=0, softmax_scale=0.0,
                   page_size=16, blocks=0) -> "Plan":
        gs = np.ascontiguousarray(group_start, np.int32)
        gl = np.ascontiguousarray(group_prefix_len, np.int32)
        h = Heads(n_q_heads, n_kv_heads, head_dim, softmax_scale)
        d = PagedDesc(int(gs[-1]), len(gl), page_size, max_pages_per_seq, n_pool_pages, max_suffix_len,
                      int(bool(share_prefix)), rounds, blocks)
        out = _vp()
        _check(_lib.fka_plan_create_paged(C.byref(h), C.byref(d), gs.ctypes.data_as(_vp), gl.ctypes.data_as(_vp),
                                          C.byref(out)))
        return cls(out.value, True, h, int(gs[-1]))

    @classmethod
    def prefill_plan(cls, n_q_heads, n_kv_heads, head_dim, n_branches, n_tokens, prefix_len, suffix_cap,
                     max_suffix_len, softmax_scale=0.0, blocks=0) -> "Plan":
        """An instruction-prefill plan (fka_plan_create_prefill): n_tokens per branch."""
        h = Heads(n_q_heads, n_kv_heads, head_dim, softmax_scale)
        d = PrefillDesc(n_branches, n_tokens, prefix_len, suffix_cap, max_suffix_len, blocks)
        out = _vp()
        _check(_lib.fka_plan_create_prefill(C.byref(h), C.byref(d), C.byref(out)))
        return cls(out.value, False, h, n_branches * n_tokens)

    @classmethod
    def prefill_paged_plan(cls, n_q_heads, n_kv_heads, head_dim, n_branches, n_tokens, prefix_len, max_pages_per_seq,
                           n_pool_pages, max_suffix_len, softmax_scale=0.0, blocks=0, page_size=16) -> "Plan":
        """A paged instruction-prefill plan (fka_plan_create_prefill_paged): n_tokens per branch."""
        h = Heads(n_q_heads, n_kv_heads, head_dim, softmax_scale)
        d = PrefillPagedDesc(n_branches, n_tokens, prefix_len, page_size, max_pages_per_seq, n_pool_pages,
                             max_suffix_len, blocks)
        out = _vp()
        _check(_lib.fka_plan_create_prefill_paged(C.byref(h), C.byref(d), C.byref(out)))
        return cls(out.value, True, h, n_branches * n_tokens)

    def prefill_paged(self, q, k_pool, v_pool, page_table, suffix_len, out, out_lse=None, stream=None):
        """fka_prefill_paged: q bf16 [N][n][Hq][d], page_table int32 [N][max_pages] -> out fp32 [N][n][Hq][d]."""
        d = self.device
        _check(_lib.fka_prefill_paged(self._h, _p(q, "bf16", d), _p(k_pool, "bf16", d), _p(v_pool, "bf16", d),
                                      _p(page_table, "i32", d), _p(suffix_len, "i32", d), _p(out, "f32", d),
                                      _p(out_lse, "f32", d), _stream(stream)))

    def prefill(self, q, prefix_k, prefix_v, suffix_k, suffix_v, suffix_len, out, out_lse=None, stream=None):
        """fka_prefill: q bf16 [N][n][Hq][d] -> out fp32 [N][n][Hq][d], out_lse fp32 [N][n][Hq]."""
        d = self.device
        _check(_lib.fka_prefill(self._h, _p(q, "bf16", d), _p(prefix_k, "bf16", d), _p(prefix_v, "bf16", d),
                                _p(suffix_k, "bf16", d), _p(suffix_v, "bf16", d), _p(suffix_len, "i32", d),
                                _p(out, "f32", d), _p(out_lse, "f32", d), _stream(stream)))

    @classmethod
    def mx_plan(cls, n_q_heads, n_kv_heads, head_dim, group_start, group_prefix_len, suffix_cap, max_suffix_len, *, n_pool_tiles,
                max_tiles=None, softmax_scale=0.0, blocks=0) -> "Plan":
        """A decode plan over 4-bit prefix tiles and contiguous suffixes (fka_plan_create_mx); max_tiles is the
        tile table's width (default: the longest prefix's tiles)."""
        gs = np.ascontiguousarray(group_start, np.int32)
        gl = np.ascontiguousarray(group_prefix_len, np.int32)
        if gs.ndim != 1 or gl.shape != (len(gs) - 1,):
            raise ValueError("group_start must have one entry more than group_prefix_len")
        if max_tiles is None:
            max_tiles = max(1, -(-int(gl.max(initial=0)) // MX_TILE))
        h = Heads(n_q_heads, n_kv_heads, head_dim, softmax_scale)
        d = MxDesc(int(gs[-1]), len(gl), max_tiles, n_pool_tiles, suffix_cap, max_suffix_len, blocks)
        out = _vp()
        _check(_lib.fka_plan_create_mx(C.byref(h), C.byref(d), gs.ctypes.data_as(_vp), gl.ctypes.data_as(_vp), C.byref(out)))
        plan = cls(out.value, False, h, int(gs[-1]))
        plan._mx = (n_pool_tiles, n_kv_heads, 136 * head_dim), len(gl) * max_tiles
        return plan

    def _mx_tiles(self, tiles, tile_table):
        if self._mx is None:
            return  # refused by the call
        want, entries = self._mx
        got = () if tiles is None else tiles.shape
        if want != got and want[0] and (len(got) != 3 or got[0] < want[0] or got[1:] != want[1:]):
            raise ValueError(f"tiles must be uint8 {list(want)}, the pool that the plan was made for")
        if tile_table is not None and tile_table.numel() < entries:
            raise ValueError(f"tile_table must have {entries} entries, the plan's groups x max_tiles")

    def decode_mx(self, q, tiles, suffix_k, suffix_v, suffix_len, out, out_lse=None, tile_table=None, stream=None):
        """fka_fork_decode_mx: tiles uint8 [pool][Hkv][136 d], tile_table int32 [groups][max_tiles] or None."""
        self._mx_tiles(tiles, tile_table)
        d = self.device
        _check(_lib.fka_fork_decode_mx(self._h, _p(q, "bf16", d), _p(tiles, "u8", d), _p(tile_table, "i32", d),
                                       _p(suffix_k, "bf16", d), _p(suffix_v, "bf16", d), _p(suffix_len, "i32", d),
                                       _p(out, "f32", d), _p(out_lse, "f32", d), _stream(stream)))

    def step_mx(self, q, k_new, v_new, tiles, suffix_k, suffix_v, suffix_len, out, out_lse=None, tile_table=None, stream=None):
        """fka_fork_step_mx: append and decode."""
        self._mx_tiles(tiles, tile_table)
        d = self.device
        _check(_lib.fka_fork_step_mx(self._h, _p(q, "bf16", d), _p(k_new, "bf16", d), _p(v_new, "bf16", d), _p(tiles, "u8", d),
                                     _p(tile_table, "i32", d), _p(suffix_k, "bf16", d), _p(suffix_v, "bf16", d),
                                     _p(suffix_len, "i32", d), _p(out, "f32", d), _p(out_lse, "f32", d), _stream(stream)))

    def close(self):
        if self._h is not None and self._h.value:
            _lib.fka_plan_destroy(self._h)
        self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def handle(self):
        return self._h

    def info(self) -> PlanInfo:
        i = PlanInfo()
        _check(_lib.fka_plan_get_info(self._h, C.byref(i)))
        return i

    def slots(self, suffix_len) -> list:
        """The partial slots a decode writes for these (host) suffix lengths (fka_plan_slots)."""
        import numpy as np
        sl = np.ascontiguousarray(suffix_len, np.int32)
        if sl.shape != (self.n_seqs,):
            raise ValueError(f"suffix_len must have shape ({self.n_seqs},)")
        n = C.c_int32(0)
        _check(_lib.fka_plan_slots(self._h, sl.ctypes.data_as(_vp), None, 0, C.byref(n)))
        arr = (Slot * max(1, n.value))()
        _check(_lib.fka_plan_slots(self._h, sl.ctypes.data_as(_vp), C.cast(arr, _vp), n.value, C.byref(n)))
        return [{f: getattr(arr[i], f) for f, _ in Slot._fields_} for i in range(n.value)]

    def device_error(self) -> int:
        v = C.c_int32(0)
        _check(_lib.fka_plan_device_error(self._h, C.byref(v)))
        return v.value

    # ---- contiguous
    def decode(self, q, prefix_k, prefix_v, suffix_k, suffix_v, suffix_len, out, out_lse=None, stream=None):
        d = self.device
        _check(_lib.fka_fork_decode(self._h, _p(q, "bf16", d), _p(prefix_k, "bf16", d), _p(prefix_v, "bf16", d),
                                    _p(suffix_k, "bf16", d), _p(suffix_v, "bf16", d), _p(suffix_len, "i32", d),
                                    _p(out, "f32", d), _p(out_lse, "f32", d), _stream(stream)))

    def append(self, k_new, v_new, suffix_k, suffix_v, suffix_len, stream=None):
        d = self.device
        _check(_lib.fka_append_kv(self._h, _p(k_new, "bf16", d), _p(v_new, "bf16", d), _p(suffix_k, "bf16", d),
                                  _p(suffix_v, "bf16", d), _p(suffix_len, "i32", d), _stream(stream)))

    def step(self, q, k_new, v_new, prefix_k, prefix_v, suffix_k, suffix_v, suffix_len, out, out_lse=None,
             stream=None):
        d = self.device
        _check(_lib.fka_fork_step(self._h, _p(q, "bf16", d), _p(k_new, "bf16", d), _p(v_new, "bf16", d),
                                  _p(prefix_k, "bf16", d), _p(prefix_v, "bf16", d), _p(suffix_k, "bf16", d),
                                  _p(suffix_v, "bf16", d), _p(suffix_len, "i32", d), _p(out, "f32", d),
                                  _p(out_lse, "f32", d), _stream(stream)))

    def partials(self, q, prefix_k, prefix_v, suffix_k, suffix_v, suffix_len, part_o, part_lse, stream=None):
        d = self.device
        _check(_lib.fka_partials(self._h, _p(q, "bf16", d), _p(prefix_k, "bf16", d), _p(prefix_v, "bf16", d),
                                 _p(suffix_k, "bf16", d), _p(suffix_v, "bf16", d), _p(suffix_len, "i32", d),
                                 _p(part_o, "f32", d), _p(part_lse, "f32", d), _stream(stream)))

    # ---- paged
    def partials_paged(self, q, k_pool, v_pool, page_table, suffix_len, part_o, part_lse, stream=None):
        d = self.device
        _check(_lib.fka_partials_paged(self._h, _p(q, "bf16", d), _p(k_pool, "bf16", d), _p(v_pool, "bf16", d),
                                       _p(page_table, "i32", d), _p(suffix_len, "i32", d), _p(part_o, "f32", d),
                                       _p(part_lse, "f32", d), _stream(stream)))

    def decode_paged(self, q, k_pool, v_pool, page_table, suffix_len, out, out_lse=None, stream=None):
        d = self.device
        _check(_lib.fka_fork_decode_paged(self._h, _p(q, "bf16", d), _p(k_pool, "bf16", d), _p(v_pool, "bf16", d),
                                          _p(page_table, "i32", d), _p(suffix_len, "i32", d), _p(out, "f32", d),
                                          _p(out_lse, "f32", d), _stream(stream)))

    def step_paged(self, q, k_new, v_new, k_pool, v_pool, page_table, suffix_len, out, out_lse=None, stream=None):
        d = self.device
        _check(_lib.fka_fork_step_paged(self._h, _p(q, "bf16", d), _p(k_new, "bf16", d), _p(v_new, "bf16", d),
                                        _p(k_pool, "bf16", d), _p(v_pool, "bf16", d), _p(page_table, "i32", d),
                                        _p(suffix_len, "i32", d), _p(out, "f32", d), _p(out_lse, "f32", d),
                                        _stream(stream)))

    def append_paged(self, k_new, v_new, k_pool, v_pool, page_table, suffix_len, stream=None):
        d = self.device
        _check(_lib.fka_append_kv_paged(self._h, _p(k_new, "bf16", d), _p(v_new, "bf16", d), _p(k_pool, "bf16", d),
                                        _p(v_pool, "bf16", d), _p(page_table, "i32", d), _p(suffix_len, "i32", d),
                                        _stream(stream)))

    def gather_paged_range(self, seq, begin, out_len, k_pool, v_pool, page_table, k_out, v_out, stream=None):
        d = self.device
        _check(_lib.fka_gather_paged_range(self._h, int(seq), int(begin), int(out_len), _p(k_pool, "bf16", d),
                                           _p(v_pool, "bf16", d), _p(page_table, "i32", d), _p(k_out, "bf16", d),
                                           _p(v_out, "bf16", d), _stream(stream)))

    def gather_paged(self, seq, k_pool, v_pool, page_table, out_len, k_out, v_out, stream=None):
        d = self.device
        _check(_lib.fka_gather_paged(self._h, int(seq), _p(k_pool, "bf16", d), _p(v_pool, "bf16", d),
                                     _p(page_table, "i32", d), int(out_len), _p(k_out, "bf16", d),
                                     _p(v_out, "bf16", d), _stream(stream)))


def _host_i32(a: np.ndarray) -> _vp:
    if a.dtype != np.int32 or not a.flags["C_CONTIGUOUS"] or not a.flags["WRITEABLE"]:
        raise ValueError("host page ids must be a writeable C-contiguous int32 array")
    return _vp(a.ctypes.data)


class Pool:
    """Page pool of a paged K/V store (host bookkeeping; see fka_pool_* in forkattn.h).  Page
    tables are host numpy int32 arrays [rows][max_pages] with -1 for no page."""

    def __init__(self, n_pages: int):
        h = _vp()
        _check(_lib.fka_pool_create(int(n_pages), C.byref(h)))
        self._h = h

    def close(self):
        if self._h:
            _lib.fka_pool_destroy(self._h)
            self._h = _vp()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def free_pages(self) -> int:
        return _lib.fka_pool_free_pages(self._h)

    def refcount(self, page: int) -> int:
        return _lib.fka_pool_refcount(self._h, int(page))

    def alloc(self, n: int) -> np.ndarray:
        ids = np.empty(int(n), np.int32)
        _check(_lib.fka_pool_alloc(self._h, int(n), _host_i32(ids)))
        return ids

    def retain(self, ids: np.ndarray):
        ids = np.ascontiguousarray(ids, np.int32)
        _check(_lib.fka_pool_retain(self._h, ids.size, _host_i32(ids)))

    def release(self, ids: np.ndarray):
        ids = np.ascontiguousarray(ids, np.int32)
        _check(_lib.fka_pool_release(self._h, ids.size, _host_i32(ids)))

    def fork(self, prefix_pages: np.ndarray, table: np.ndarray, first: int, n: int):
        prefix_pages = np.ascontiguousarray(prefix_pages, np.int32)
        _check(_lib.fka_pool_fork(self._h, _host_i32(prefix_pages), prefix_pages.size, _host_i32(table),
                                  table.shape[1], int(first), int(n)))

    def reserve(self, table: np.ndarray, seq: int, prefix_len: int, suffix_len: int) -> int:
        n_new = C.c_int32(0)
        _check(_lib.fka_pool_reserve(self._h, _host_i32(table), table.shape[1], int(seq), int(prefix_len),
                                     int(suffix_len), C.byref(n_new)))
        return n_new.value

    def drop(self, table: np.ndarray, seq: int):
        _check(_lib.fka_pool_drop(self._h, _host_i32(table), table.shape[1], int(seq)))

    def promote(self, table: np.ndarray, seq: int, prefix_len: int, suffix_len: int):
        """Returns (dense page ids, first position to rewrite)."""
        n = (int(prefix_len) + int(suffix_len) + 15) // 16
        dense = np.full(max(n, 1), -1, np.int32)
        frm = C.c_int32(0)
        _check(_lib.fka_pool_promote(self._h, _host_i32(table), table.shape[1], int(seq), int(prefix_len),
                                     int(suffix_len), _host_i32(dense), C.byref(frm)))
        return dense[:n], frm.value


def scatter_pages(k_src, v_src, frm, page_row, n_pool_pages, k_pool, v_pool, err=None, stream=None):
    """Positions [frm, frm + n) held in k_src / v_src bf16 [Hkv][n][d] -> pool pages of page_row (device int32)."""
    Hkv, n, d = k_src.shape
    _check(_lib.fka_scatter_pages(_p(k_src, "bf16"), _p(v_src, "bf16"), int(frm) + n, int(frm), _p(page_row, "i32"), Hkv, d, int(n_pool_pages),
                                  _p(k_pool, "bf16"), _p(v_pool, "bf16"), _p(err, "i32"), _stream(stream)))


def read_probe(buf, blocks, threads, unroll, sink, stream=None):
    """Read-only streaming probe over the device tensor buf (fka_read_probe)."""
    _check(_lib.fka_read_probe(_p(buf), buf.numel() * buf.element_size(), int(blocks), int(threads), int(unroll),
                               _p(sink), _stream(stream)))


def decode_noalloc(n_q_heads, n_kv_heads, head_dim, prefix_len, suffix_cap, max_suffix_len, q, prefix_k, prefix_v,
                   suffix_k, suffix_v, suffix_len, out, out_lse=None, err=None, rounds=0, softmax_scale=0.0, blocks=0,
                   stream=None):
    """fka_fork_decode_noalloc: a shared-prefix decode without a plan, on the library's static scratch
    (the sizes are those of Plan.contig with share_prefix=True; n_branches is q's first dimension)."""
    dev = q.get_device() if isinstance(q, torch.Tensor) and q.is_cuda else None
    h = Heads(n_q_heads, n_kv_heads, head_dim, softmax_scale)
    d = ContigDesc(q.shape[0], prefix_len, suffix_cap, max_suffix_len, 1, rounds, blocks)
    _check(_lib.fka_fork_decode_noalloc(C.byref(h), C.byref(d), _p(q, "bf16", dev), _p(prefix_k, "bf16", dev),
                                        _p(prefix_v, "bf16", dev), _p(suffix_k, "bf16", dev), _p(suffix_v, "bf16", dev),
                                        _p(suffix_len, "i32", dev), _p(out, "f32", dev), _p(out_lse, "f32", dev),
                                        _p(err, "i32", dev), _stream(stream)))


def lse_merge(part_o, part_lse, out, out_lse=None, stream=None):
    """part_o fp32 [P][R][d], part_lse fp32 [P][R] -> out fp32 [R][d], out_lse fp32 [R]."""
    P, R, d = part_o.shape
    _check(_lib.fka_lse_merge(R, P, d, _p(part_o, "f32"), _p(part_lse, "f32"), _p(out, "f32"), _p(out_lse, "f32"), _stream(stream)))


def _token_rows(t, shape, what):
    """Token stride (elements) of q, k or v [N][n][heads][d]: any view whose tokens lie evenly apart."""
    N, n, heads, d = shape
    seq, step, head, elem = t.stride()
    if elem != 1 or (head != d and heads > 1):
        raise ValueError(f"{what} must be [N][n][heads][d] with the heads of a token dense")
    if n == 1:
        return seq if N > 1 else heads * d
    if N > 1 and seq != n * step:
        raise ValueError(f"the tokens of {what} must lie evenly apart")
    return step


def _on_current(t):
    """The device of t, which has to be the current one: a call without a plan launches on the current device's stream."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError("tensor must be on the GPU (the library reads device memory)")
    dev = t.get_device()
    current = torch.cuda.current_device() if _current_device is None else _current_device()
    if dev != current:
        raise ValueError(f"tensor is on cuda:{dev}, the current device is cuda:{current}")
    return dev


def _strided(t, dev):
    if t.dtype is torch.bfloat16 and t.get_device() == dev:  # -1 on the CPU
        return t.data_ptr()
    if not t.is_cuda or t.dtype is not torch.bfloat16:
        raise ValueError("expected a bf16 tensor on the GPU")
    raise ValueError(f"tensor is on cuda:{t.get_device()}, q is on cuda:{dev}")


def _rotate_desc(q, k, v, positions, freq, q_out, q_weight, k_weight, eps, interleaved, advance):
    for t in (q, k, v, positions, q_out):
        if not isinstance(t, torch.Tensor):
            raise ValueError("expected a torch tensor")
    shape, kv = q.shape, k.shape
    if len(shape) != 4 or len(kv) != 4 or v.dim() != 4:
        raise ValueError("q, k and v must be [N][n][heads][d]")
    steps = _token_rows(q, shape, "q"), _token_rows(k, kv, "k"), _token_rows(v, v.shape, "v")
    N, n, Hq, d = shape
    if (kv[0], kv[1], kv[3]) != (N, n, d) or v.shape != kv:
        raise ValueError("k and v must be [N][n][Hkv][d] with q's N, n and d")
    if q_out.shape != shape or positions.numel() != N * n:
        raise ValueError("q_out must have q's shape, positions N n entries")
    if (q_weight is not None and q_weight.shape != (d,)) or (k_weight is not None and k_weight.shape != (d,)):
        raise ValueError("a norm weight must be [d]")
    return RotateDesc(N, n, Hq, kv[2], d, 0 if freq is None else 2 * freq.numel(), 1 if interleaved else 0, 0,
                      1 if advance else 0, eps, *steps)


def _check_lens(suffix_len, N):
    if suffix_len is not None and suffix_len.numel() != N:
        raise ValueError("suffix_len must have an entry per sequence")


def rotate_append(q, k, v, positions, freq, q_out, suffix_k, suffix_v, suffix_len=None, *, q_weight=None, k_weight=None,
                  eps=1e-6, interleaved=False, max_len=None, advance=False, err=None, stream=None):
    """fka_rotate_append: q, k, v bf16 [N][n][heads][d] (views of a joint projection output allowed), positions int32 [N][n],
    freq fp64 [rotary_dim / 2] or None -> q_out, and rows of suffix_k / suffix_v bf16 [N][Hkv][cap][d]."""
    desc = _rotate_desc(q, k, v, positions, freq, q_out, q_weight, k_weight, eps, interleaved, advance)
    N, _, Hkv, d = k.shape
    rows = suffix_k.shape
    cap = rows[2] if len(rows) == 4 else -1
    if rows != (N, Hkv, cap, d) or suffix_v.shape != rows:
        raise ValueError("suffix_k and suffix_v must be [N][Hkv][cap][d]")
    _check_lens(suffix_len, N)
    desc.max_len = cap if max_len is None else max_len
    dev = _on_current(q)
    _check(_lib.fka_rotate_append(C.byref(desc), _strided(q, dev), _strided(k, dev), _strided(v, dev), _p(q_weight, "bf16", dev),
                                  _p(k_weight, "bf16", dev), _p(freq, "f64", dev), _p(positions, "i32", dev),
                                  _p(q_out, "bf16", dev), _p(suffix_k, "bf16", dev), _p(suffix_v, "bf16", dev), cap,
                                  _p(suffix_len, "i32", dev), _p(err, "i32", dev), _stream(stream)))


def rotate_append_paged(q, k, v, positions, freq, q_out, k_pool, v_pool, page_table, prefix_len, suffix_len=None, *,
                        q_weight=None, k_weight=None, eps=1e-6, interleaved=False, max_len=None, advance=False, err=None,
                        stream=None):
    """fka_rotate_append_paged: as rotate_append, into the pages of page_table int32 [N][max_pages] behind prefix_len int32 [N]."""
    desc = _rotate_desc(q, k, v, positions, freq, q_out, q_weight, k_weight, eps, interleaved, advance)
    N, _, Hkv, d = k.shape
    if k_pool.dim() != 4 or k_pool.shape[1:] != (Hkv, 16, d) or v_pool.shape != k_pool.shape:
        raise ValueError("k_pool and v_pool must be [pages][Hkv][16][d]")
    if page_table.dim() != 2 or page_table.shape[0] != N or prefix_len.numel() != N:
        raise ValueError("page_table must have a row, prefix_len an entry per sequence")
    _check_lens(suffix_len, N)
    desc.max_len = 16 * page_table.shape[1] if max_len is None else max_len
    dev = _on_current(q)
    _check(_lib.fka_rotate_append_paged(C.byref(desc), _strided(q, dev), _strided(k, dev), _strided(v, dev),
                                        _p(q_weight, "bf16", dev), _p(k_weight, "bf16", dev), _p(freq, "f64", dev),
                                        _p(positions, "i32", dev), _p(q_out, "bf16", dev), _p(k_pool, "bf16", dev),
                                        _p(v_pool, "bf16", dev), _p(page_table, "i32", dev), _p(prefix_len, "i32", dev),
                                        page_table.shape[1], k_pool.shape[0], _p(suffix_len, "i32", dev), _p(err, "i32", dev),
                                        _stream(stream)))


def mx_tile_bytes(n_kv_heads, head_dim) -> int:
    """Bytes of one 4-bit tile (128 tokens) of all KV heads."""
    return _lib.fka_mx_tile_bytes(n_kv_heads, head_dim)


def _mx_sizes(k, v, tiles, tile_row, frm, length):
    if k.dim() != 3 or v.shape != k.shape:
        raise ValueError("k and v must be [Hkv][cap][d]")
    Hkv, cap, d = k.shape
    if tiles.dim() != 3 or tiles.shape[1:] != (Hkv, 136 * d):
        raise ValueError("tiles must be uint8 [pool][Hkv][136 d]")
    length = int(frm) + cap if length is None else int(length)
    if tile_row is not None and tile_row.numel() < -(-length // MX_TILE):
        raise ValueError("tile_row is shorter than the prefix's tiles")
    return Hkv, cap, d, length


def mx_pack(k, v, tiles, *, tile_row=None, frm=0, length=None, err=None, stream=None):
    """fka_mx_pack: positions [frm, length) held in k, v bf16 [Hkv][cap][d] -> tiles uint8 [pool][Hkv][136 d]."""
    Hkv, cap, d, length = _mx_sizes(k, v, tiles, tile_row, frm, length)
    dev = _on_current(tiles)
    _check(_lib.fka_mx_pack(Hkv, d, int(frm), length, _p(k, "bf16", dev), _p(v, "bf16", dev), cap, _p(tiles, "u8", dev),
                            _p(tile_row, "i32", dev), tiles.shape[0], _p(err, "i32", dev), _stream(stream)))


def mx_unpack(tiles, k, v, *, tile_row=None, frm=0, length=None, err=None, stream=None):
    """fka_mx_unpack: the values of positions [frm, length) -> k, v bf16 [Hkv][cap][d]."""
    Hkv, cap, d, length = _mx_sizes(k, v, tiles, tile_row, frm, length)
    dev = _on_current(tiles)
    _check(_lib.fka_mx_unpack(Hkv, d, int(frm), length, _p(tiles, "u8", dev), _p(tile_row, "i32", dev), tiles.shape[0],
                              _p(k, "bf16", dev), _p(v, "bf16", dev), cap, _p(err, "i32", dev), _stream(stream)))


def key_weights(q, lse, k, weights, *, length=None, decay=0.0, softmax_scale=0.0, stream=None):
    """fka_key_weights: q bf16 [R][Hq][d], lse fp32 [R][Hq], k bf16 [Hkv][cap][d] -> weights fp32 [Hkv][cap']."""
    R, Hq, d = q.shape
    Hkv, cap = k.shape[0], k.shape[1]
    if k.shape != (Hkv, cap, d) or lse.shape != (R, Hq) or weights.dim() != 2 or weights.shape[0] != Hkv:
        raise ValueError("lse must be [R][Hq], k [Hkv][cap][d] and weights [Hkv][cap']")
    h = Heads(Hq, Hkv, d, softmax_scale)
    dev = _on_current(weights)
    _check(_lib.fka_key_weights(C.byref(h), R, min(cap, weights.shape[1]) if length is None else int(length), _p(q, "bf16", dev),
                                _p(lse, "f32", dev), _p(k, "bf16", dev), cap, _p(weights, "f32", dev), weights.shape[1],
                                float(decay), _stream(stream)))


def evict_workspace(n_kv_heads, length, device="cuda"):
    """A workspace for evict over up to `length` positions."""
    return torch.empty(_lib.fka_evict_bytes(n_kv_heads, length), dtype=torch.uint8, device=device)


def evict(k, v, weights, index, k_out, v_out, weights_out=None, *, n_first=0, n_last=0, length=None, workspace, stream=None):
    """fka_evict: keeps index.shape[1] of each KV head's positions (k, v bf16 [Hkv][cap][d], weights fp32 [Hkv][cap'])."""
    if k.dim() != 3 or v.shape != k.shape or weights.dim() != 2 or weights.shape[0] != k.shape[0] or index.dim() != 2:
        raise ValueError("k and v must be [Hkv][cap][d], weights [Hkv][cap'], index [Hkv][keep]")
    Hkv, cap, d = k.shape
    keep = index.shape[1]
    if index.shape != (Hkv, keep) or k_out.shape != (Hkv, keep, d) or v_out.shape != k_out.shape:
        raise ValueError("k_out and v_out must be [Hkv][keep][d]")
    if weights_out is not None and weights_out.shape != (Hkv, keep):
        raise ValueError("weights_out must be [Hkv][keep]")
    dev = _on_current(k)
    _check(_lib.fka_evict(Hkv, d, min(cap, weights.shape[1]) if length is None else int(length), keep, int(n_first), int(n_last),
                          _p(k, "bf16", dev), _p(v, "bf16", dev), cap, _p(weights, "f32", dev), weights.shape[1],
                          _p(index, "i32", dev), _p(k_out, "bf16", dev), _p(v_out, "bf16", dev), _p(weights_out, "f32", dev),
                          _p(workspace, "u8", dev), workspace.numel(), _stream(stream)))


def raw_call(name: str, *args) -> int:
    """Call an exported function with raw ctypes arguments; returns its status (for ABI tests)."""
    return getattr(_lib, name)(*args)
