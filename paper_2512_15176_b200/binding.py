"""ctypes binding of ``libdeer.so``: the same entry points as ``include/deer.h``
with torch tensors in place of raw pointers.  Argument marshalling only --
every step of the path runs in the library's CUDA kernels; there is no CPU or
PyTorch fallback, and a missing library is a hard error.
"""
from __future__ import annotations

import ctypes
import os
from ctypes import POINTER, Structure, c_char_p, c_float, c_int, c_int32, c_size_t, c_void_p
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdeer.so")

DEER_OK = 0
DEER_ERR_INVALID_ARG, DEER_ERR_UNSUPPORTED, DEER_ERR_NO_PAGES, DEER_ERR_CUDA, DEER_ERR_WORKSPACE, DEER_ERR_BAD_PAGE = 1, 2, 3, 4, 5, 6
DEER_ERR_TIMEOUT = 7
DEER_MASK_CAUSAL, DEER_MASK_BIDIR = 0, 1
DEER_SEL_ARGMAX, DEER_SEL_ARGMAX_LOGPROB, DEER_SEL_SOFTMAX = 0, 1, 2
DEER_ACC_GREEDY, DEER_ACC_SAMPLE, DEER_ACC_SAMPLE_PRESTATS, DEER_ACC_BONUS = 0, 1, 2, 4
DEER_EMIT_PENDING = 1

EXPORTS = [
    "deer_last_error", "deer_kv_create", "deer_kv_destroy", "deer_kv_reserve", "deer_kv_commit", "deer_accept_commit", "deer_kv_status", "deer_selftest_bounded_wait",
    "deer_block_attn_workspace_bytes", "deer_block_attn", "deer_lmhead_workspace_bytes", "deer_lmhead_select",
    "deer_accept_workspace_bytes", "deer_accept", "deer_verify_step_host",
    "deer_lmhead_static_max_rows", "deer_lmhead_select_static", "deer_emit", "deer_draft_stats",
    "deer_linear_workspace_bytes", "deer_linear", "deer_rmsnorm", "deer_qk_norm_rope", "deer_qkv_split_norm_rope", "deer_swiglu",
    "deer_truncate", "deer_accept_truncated", "deer_block_attn_rows", "deer_refill", "deer_refresh_rows",
    "deer_moe_workspace_bytes", "deer_moe_route", "deer_moe_mlp",
    "deer_layer_workspace_bytes", "deer_linear_qkv_rope", "deer_linear_residual_norm", "deer_linear_swiglu",
    "deer_rmsnorm_quant", "deer_quantize", "deer_linear_quant", "deer_kv_create_quant", "deer_kv_store",
    "deer_kv_reserve_rows", "deer_kv_commit_rows", "deer_block_attn_quant_workspace_bytes", "deer_block_attn_quant",
]


class DeerError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__(f"libdeer status {code}: {text}")
        self.code = code


class deer_kv_desc(Structure):
    _fields_ = [("k_pool", c_void_p), ("v_pool", c_void_p), ("page_table", c_void_p), ("seq_len", c_void_p),
                ("n_pages", c_void_p), ("free_stack", c_void_p), ("free_top", c_void_p), ("status", c_void_p),
                ("num_pages", c_int32), ("n_kv_heads", c_int32), ("head_dim", c_int32), ("page_size", c_int32),
                ("max_seqs", c_int32), ("max_pages", c_int32)]


class deer_kv_quant_desc(Structure):
    _fields_ = [("k_scale", c_void_p), ("v_scale", c_void_p), ("k_tail", c_void_p), ("v_tail", c_void_p)]


class deer_step_dev(Structure):
    _fields_ = [("q", c_void_p), ("k_blk", c_void_p), ("v_blk", c_void_p), ("attn_out", c_void_p), ("h", c_void_p),
                ("seq_ids", c_void_p), ("draft_ids", c_void_p), ("target_ids", c_void_p), ("accept_len", c_void_p),
                ("out_ids", c_void_p), ("n_out", c_void_p), ("attn_ws", c_void_p), ("attn_ws_bytes", c_size_t),
                ("lm_ws", c_void_p), ("lm_ws_bytes", c_size_t)]


_lib = None


def lib() -> ctypes.CDLL:
    """Load the C-ABI library (once).  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2512_15176_b200.build` "
                           "(there is no fallback path)")
    L = ctypes.CDLL(LIB_PATH)
    L.deer_last_error.restype = c_char_p
    L.deer_last_error.argtypes = []
    L.deer_kv_create.argtypes = [POINTER(c_void_p), POINTER(deer_kv_desc)]
    L.deer_kv_destroy.argtypes = [c_void_p]
    L.deer_kv_reserve.argtypes = [c_void_p, c_void_p, c_int, c_int, c_void_p]
    L.deer_kv_commit.argtypes = [c_void_p, c_void_p, c_void_p, c_int, c_int, c_void_p]
    L.deer_accept_commit.argtypes = [c_void_p, c_void_p, c_int, c_int, c_int, c_void_p, c_void_p, c_int32, c_void_p, c_void_p,
                                     c_void_p, c_void_p]
    L.deer_kv_status.argtypes = [c_void_p, POINTER(c_int32), c_void_p]
    L.deer_selftest_bounded_wait.argtypes = [c_void_p, c_void_p]
    L.deer_block_attn_workspace_bytes.restype = c_size_t
    L.deer_block_attn_workspace_bytes.argtypes = [c_int] * 6
    L.deer_block_attn.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_int,
                                  c_int, c_float, c_int, c_void_p, c_size_t, c_void_p]
    L.deer_lmhead_workspace_bytes.restype = c_size_t
    L.deer_lmhead_workspace_bytes.argtypes = [c_int] * 3
    L.deer_lmhead_select.argtypes = [c_void_p, c_void_p, c_int, c_int, c_int, c_int, c_float, c_void_p, c_void_p, c_void_p,
                                     c_void_p, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    L.deer_lmhead_static_max_rows.restype = c_size_t
    L.deer_lmhead_static_max_rows.argtypes = []
    L.deer_lmhead_select_static.argtypes = [c_void_p, c_void_p, c_int, c_int, c_int, c_int, c_float, c_void_p, c_void_p,
                                            c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]
    L.deer_accept_workspace_bytes.restype = c_size_t
    L.deer_accept_workspace_bytes.argtypes = [c_int] * 4
    L.deer_accept.argtypes = [c_int, c_int, c_int, c_int, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_float,
                              c_void_p, c_void_p, c_void_p, c_int32, c_void_p, c_void_p, c_void_p, c_void_p, c_size_t,
                              c_void_p]
    L.deer_accept_truncated.argtypes = [c_int, c_int, c_int, c_int, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                        c_float, c_void_p, c_void_p, c_void_p, c_int32, c_void_p, c_void_p, c_void_p, c_void_p,
                                        c_size_t, c_void_p]
    L.deer_truncate.argtypes = [c_int, c_int, c_void_p, c_void_p, c_float, c_int, c_float, c_void_p, c_void_p, c_void_p]
    L.deer_linear_workspace_bytes.restype = c_size_t
    L.deer_linear_workspace_bytes.argtypes = [c_int] * 3
    L.deer_linear.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_void_p, c_size_t, c_void_p]
    L.deer_rmsnorm.argtypes = [c_void_p, c_void_p, c_void_p, c_int, c_int, c_float, c_void_p]
    L.deer_qk_norm_rope.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_float,
                                    c_float, c_void_p]
    L.deer_qkv_split_norm_rope.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int,
                                           c_int, c_int, c_float, c_float, c_void_p]
    L.deer_swiglu.argtypes = [c_void_p, c_void_p, c_int, c_int, c_void_p]
    L.deer_draft_stats.argtypes = [c_int, c_int, c_int, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    L.deer_emit.argtypes = [c_int, c_int, c_void_p, c_void_p, c_void_p, c_int32, c_int32, c_void_p, c_void_p, c_void_p, c_void_p,
                            c_void_p, c_int, c_void_p]
    L.deer_block_attn_rows.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_int, c_int,
                                       c_int, c_int, c_float, c_int, c_void_p, c_size_t, c_void_p]
    L.deer_refill.argtypes = [c_int, c_int, c_void_p, c_void_p, c_float, c_void_p, c_void_p, c_void_p, c_void_p]
    L.deer_refresh_rows.argtypes = [c_int, c_int, c_void_p, c_void_p, c_void_p]
    L.deer_layer_workspace_bytes.restype = c_size_t
    L.deer_layer_workspace_bytes.argtypes = [c_int] * 3
    L.deer_linear_qkv_rope.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                       c_int, c_int, c_int, c_int, c_float, c_float, c_void_p, c_size_t, c_void_p]
    L.deer_linear_residual_norm.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_int, c_int,
                                            c_float, c_void_p, c_size_t, c_void_p]
    L.deer_linear_swiglu.argtypes = [c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_void_p]
    L.deer_moe_workspace_bytes.restype = c_size_t
    L.deer_moe_workspace_bytes.argtypes = [c_int] * 5
    L.deer_moe_route.argtypes = [c_void_p, c_void_p, c_int, c_int, c_int, c_int, c_int, c_void_p, c_void_p, c_void_p, c_size_t,
                                 c_void_p]
    L.deer_moe_mlp.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_int, c_int,
                               c_void_p, c_size_t, c_void_p]
    L.deer_verify_step_host.argtypes = [c_void_p, POINTER(deer_step_dev), c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                        c_void_p, c_int, c_int, c_int, c_int, c_int, c_float, c_int, c_void_p, c_void_p,
                                        c_void_p, c_void_p]
    L.deer_rmsnorm_quant.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_int, c_float, c_void_p]
    L.deer_quantize.argtypes = [c_void_p, c_int, c_void_p, c_void_p, c_int, c_int, c_void_p]
    L.deer_linear_quant.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_void_p]
    L.deer_kv_create_quant.argtypes = [POINTER(c_void_p), POINTER(deer_kv_desc), POINTER(deer_kv_quant_desc)]
    L.deer_kv_store.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_int, c_void_p]
    L.deer_kv_reserve_rows.argtypes = [c_void_p, c_void_p, c_int, c_int, c_void_p]
    L.deer_kv_commit_rows.argtypes = [c_void_p, c_void_p, c_void_p, c_int, c_int, c_void_p]
    L.deer_block_attn_quant_workspace_bytes.restype = c_size_t
    L.deer_block_attn_quant_workspace_bytes.argtypes = [c_int] * 6
    L.deer_block_attn_quant.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_int, c_int,
                                        c_int, c_float, c_int, c_void_p, c_size_t, c_void_p]
    for name in EXPORTS:
        getattr(L, name)          # every declared entry point must be exported
    _lib = L
    return L


def _check(rc: int) -> None:
    if rc != DEER_OK:
        raise DeerError(rc, lib().deer_last_error().decode())


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    assert t.is_contiguous(), "tensors passed to libdeer must be contiguous"
    return t.data_ptr()


# The handle itself, where torch has it: torch.cuda.current_stream() builds a Stream object first, which takes longer than a
# launch.  (A call's tensors are on the device, so torch has initialised it by now.)
_raw_stream, _current_device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream) -> Optional[int]:
    if stream is None:
        if _raw_stream is None or _current_device is None:
            return torch.cuda.current_stream().cuda_stream or None
        return _raw_stream(_current_device()) or None
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream or None
    return stream or None


class KVCache:
    """Device tensors of one paged cache plus the library handle over them."""

    def __init__(self, k_pool, v_pool, page_table, seq_len, n_pages, free_stack, free_top):
        self._describe(k_pool, v_pool, page_table, seq_len, n_pages, free_stack, free_top)
        _check(lib().deer_kv_create(ctypes.byref(self.handle), ctypes.byref(self.desc)))

    def _describe(self, k_pool, v_pool, page_table, seq_len, n_pages, free_stack, free_top):
        self.k_pool, self.v_pool = k_pool, v_pool
        self.page_table, self.seq_len, self.n_pages = page_table, seq_len, n_pages
        self.free_stack, self.free_top = free_stack, free_top
        self.status = torch.zeros(1, dtype=torch.int32, device=k_pool.device)
        num_pages, Hkv, page, D = k_pool.shape
        self.desc = deer_kv_desc(_ptr(k_pool), _ptr(v_pool), _ptr(page_table), _ptr(seq_len), _ptr(n_pages),
                                 _ptr(free_stack), _ptr(free_top), _ptr(self.status),
                                 num_pages, Hkv, D, page, page_table.shape[0], page_table.shape[1])
        self.handle, self._heads = c_void_p(), (Hkv, D)

    @classmethod
    def from_layout(cls, layout, k_pool, v_pool, device="cuda"):
        """``layout`` is a ``workload.KVLayout`` (host arrays); pools are bf16 tensors."""
        i32 = lambda a: torch.from_numpy(a.copy()).to(device=device, dtype=torch.int32).contiguous()
        return cls(k_pool.to(device).contiguous(), v_pool.to(device).contiguous(), i32(layout.page_table),
                   i32(layout.seq_len), i32(layout.n_pages), i32(layout.free_stack), i32(layout.free_top))

    @property
    def n_kv_heads(self):
        return self.k_pool.shape[1]

    @property
    def head_dim(self):
        return self.k_pool.shape[3]

    def close(self):
        if self.handle:
            lib().deer_kv_destroy(self.handle)
            self.handle = c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


DEER_TAIL_ROWS = 48


class KVCacheQuant(KVCache):
    """A paged cache in 8 bits: pools of ``torch.float8_e4m3fn`` with one fp32 scale per page and head, and the bf16
    tail rows of the tokens behind each sequence's last full page."""

    def __init__(self, k_pool, v_pool, k_scale, v_scale, k_tail, v_tail, page_table, seq_len, n_pages, free_stack, free_top):
        num_pages, Hkv, _, D = k_pool.shape
        assert k_pool.dtype == v_pool.dtype == torch.float8_e4m3fn and v_pool.shape == k_pool.shape
        assert k_scale.shape == v_scale.shape == (num_pages, Hkv) and k_scale.dtype == v_scale.dtype == torch.float32
        assert k_tail.shape == v_tail.shape == (page_table.shape[0], Hkv, DEER_TAIL_ROWS, D)
        assert k_tail.dtype == v_tail.dtype == torch.bfloat16
        self._describe(k_pool, v_pool, page_table, seq_len, n_pages, free_stack, free_top)
        self.k_scale, self.v_scale, self.k_tail, self.v_tail = k_scale, v_scale, k_tail, v_tail
        quant = deer_kv_quant_desc(_ptr(k_scale), _ptr(v_scale), _ptr(k_tail), _ptr(v_tail))
        _check(lib().deer_kv_create_quant(ctypes.byref(self.handle), ctypes.byref(self.desc), ctypes.byref(quant)))

    @classmethod
    def empty(cls, num_pages, n_kv_heads, head_dim, max_seqs, max_pages, device="cuda"):
        """A cache without tokens, every page on the free stack."""
        z = lambda *shape, dtype=torch.int32: torch.zeros(*shape, dtype=dtype, device=device)
        pool = lambda: z(num_pages, n_kv_heads, 16, head_dim, dtype=torch.float8_e4m3fn)
        scale = lambda: z(num_pages, n_kv_heads, dtype=torch.float32)
        tail = lambda: z(max_seqs, n_kv_heads, DEER_TAIL_ROWS, head_dim, dtype=torch.bfloat16)
        return cls(pool(), pool(), scale(), scale(), tail(), tail(), torch.full((max_seqs, max_pages), -1, dtype=torch.int32, device=device),
                   z(max_seqs), z(max_seqs), torch.arange(num_pages - 1, -1, -1, dtype=torch.int32, device=device),
                   torch.full((1,), num_pages, dtype=torch.int32, device=device))

    @classmethod
    def from_layout(cls, layout, k_pool, v_pool, device="cuda"):
        """The tokens of a bf16 cache (``workload.KVLayout`` and its pools) as an 8-bit one: full pages quantised, the
        tokens behind each sequence's last full page as tail rows."""
        kv = cls.empty(k_pool.shape[0], k_pool.shape[1], k_pool.shape[3], *layout.page_table.shape, device=device)
        i32 = lambda a: torch.from_numpy(a.copy()).to(device=device, dtype=torch.int32)
        for dst, src in ((kv.page_table, layout.page_table), (kv.seq_len, layout.seq_len), (kv.n_pages, layout.n_pages),
                         (kv.free_stack, layout.free_stack), (kv.free_top, layout.free_top)):
            dst.copy_(i32(src))
        for pool, codes, scale, tail in ((k_pool, kv.k_pool, kv.k_scale, kv.k_tail), (v_pool, kv.v_pool, kv.v_scale, kv.v_tail)):
            pool = pool.to(device)
            amax = pool.abs().amax(dim=(2, 3)).float()
            scale.copy_((amax / torch.full_like(amax, 448.0)).clamp_min(2.0 ** -126))
            codes.copy_((pool.float() / scale[:, :, None, None]).to(torch.float8_e4m3fn))
            for s, n in enumerate(layout.seq_len):
                first, rest = int(n) // 16, int(n) % 16
                if rest:
                    tail[s, :, first % 3 * 16:first % 3 * 16 + rest] = pool[int(layout.page_table[s, first]), :, :rest]
        return kv

    def layer(self):
        """Another layer's cache over the same page table, lengths and free stack, with pools of its own."""
        same = lambda t: torch.zeros_like(t)
        return KVCacheQuant(same(self.k_pool), same(self.v_pool), same(self.k_scale), same(self.v_scale), same(self.k_tail),
                            same(self.v_tail), self.page_table, self.seq_len, self.n_pages, self.free_stack, self.free_top)


# The library sees pointers and sizes only: what a call would read or write past an operand's end is refused here.
_BF16, _F32, _I32 = torch.bfloat16, torch.float32, torch.int32
_CODES = (torch.float8_e4m3fn, torch.uint8)


def _refuse(call: str, what: str):
    raise DeerError(DEER_ERR_INVALID_ARG, f"{call}: {what}")


def deer_kv_store(kv: KVCacheQuant, seq_ids, k_rows, v_rows, keep=None, stream=None) -> None:
    B, k, *heads = k_rows.shape
    if not (k_rows.dtype is _BF16 and v_rows.dtype is _BF16 and v_rows.shape == k_rows.shape and tuple(heads) == kv._heads):
        _refuse("deer_kv_store", "k_rows and v_rows must be bf16 [B][k][Hkv][D] of the cache's Hkv and D")
    if not (seq_ids.dtype is _I32 and seq_ids.numel() == B and (keep is None or keep.dtype is _I32 and keep.numel() == B)):
        _refuse("deer_kv_store", "seq_ids and keep must be int32 [B]")
    _check(lib().deer_kv_store(kv.handle, _ptr(seq_ids), _ptr(k_rows), _ptr(v_rows), _ptr(keep), B, k, _stream(stream)))


def deer_kv_reserve_rows(kv: KVCache, seq_ids: torch.Tensor, k: int, stream=None) -> None:
    _check(lib().deer_kv_reserve_rows(kv.handle, _ptr(seq_ids), seq_ids.numel(), k, _stream(stream)))


def deer_kv_commit_rows(kv: KVCache, seq_ids: torch.Tensor, keep: torch.Tensor, k: int, stream=None) -> None:
    _check(lib().deer_kv_commit_rows(kv.handle, _ptr(seq_ids), _ptr(keep), seq_ids.numel(), k, _stream(stream)))


def deer_block_attn_quant_workspace_bytes(B, k, Hq, Hkv, D, max_seq_len) -> int:
    return lib().deer_block_attn_quant_workspace_bytes(B, k, Hq, Hkv, D, max_seq_len)


def deer_block_attn_quant(kv: KVCacheQuant, seq_ids, q, k_blk, v_blk, out, row_state, mask, scale, max_seq_len, workspace, stream=None):
    B, k, Hq, D = q.shape
    Hkv, D_kv = kv._heads
    if not (q.dtype is _BF16 and out.dtype is _BF16 and out.numel() == B * k * Hq * D and D == D_kv):
        _refuse("deer_block_attn_quant", "q and out must be bf16 [B][k][Hq][D] of the cache's D")
    if not (k_blk.dtype is _BF16 and v_blk.dtype is _BF16 and k_blk.numel() == v_blk.numel() == B * k * Hkv * D):
        _refuse("deer_block_attn_quant", "k_blk and v_blk must be bf16 [B][k][Hkv][D] of the cache's Hkv")
    if not (seq_ids.dtype is _I32 and seq_ids.numel() == B and (row_state is None or row_state.dtype is _I32 and row_state.numel() == B * k)):
        _refuse("deer_block_attn_quant", "seq_ids must be int32 [B], row_state int32 [B][k]")
    _check(lib().deer_block_attn_quant(kv.handle, _ptr(seq_ids), _ptr(q), _ptr(k_blk), _ptr(v_blk), _ptr(out), _ptr(row_state), B, k, Hq,
                                       int(mask), float(scale), int(max_seq_len), _ptr(workspace),
                                       workspace.numel() * workspace.element_size() if workspace is not None else 0,
                                       _stream(stream)))


def deer_rmsnorm_quant(x, gamma, codes, scales, eps, residual=None, total=None, stream=None):
    M, hid = x.shape
    if not (x.dtype is _BF16 and gamma.dtype is _BF16 and gamma.numel() == hid and (residual is None or residual.dtype is _BF16 and residual.numel() == M * hid)
            and (total is None or total.dtype is _BF16 and total.numel() == M * hid)):
        _refuse("deer_rmsnorm_quant", "x, residual and total must be bf16 [M][hid], gamma bf16 [hid]")
    if not (codes.dtype in _CODES and codes.numel() == M * hid and scales.dtype is _F32 and scales.numel() == M * ((hid + 127) // 128)):
        _refuse("deer_rmsnorm_quant", "codes must be e4m3 [M][hid], scales f32 [M][ceil(hid / 128)]")
    _check(lib().deer_rmsnorm_quant(_ptr(x), _ptr(residual), _ptr(gamma), _ptr(total), _ptr(codes), _ptr(scales), M, hid, float(eps),
                                    _stream(stream)))


def deer_quantize(x, codes, scales, gated=False, stream=None):
    M, K = codes.shape
    if not (x.dtype is _BF16 and x.numel() == M * K * (2 if gated else 1)):
        _refuse("deer_quantize", "x must be bf16 [M][K], or [M][2 K] gated, of the codes' M and K")
    if not (codes.dtype in _CODES and scales.dtype is _F32 and scales.numel() == M * ((K + 127) // 128)):
        _refuse("deer_quantize", "codes must be e4m3 [M][K], scales f32 [M][ceil(K / 128)]")
    _check(lib().deer_quantize(_ptr(x), 1 if gated else 0, _ptr(codes), _ptr(scales), M, K, _stream(stream)))


def deer_linear_quant(x, x_scale, w, w_scale, y, residual=None, stream=None):
    M, K = x.shape
    N, K_w = w.shape
    G = (K + 127) // 128
    if not (x.dtype in _CODES and w.dtype in _CODES and K_w == K):
        _refuse("deer_linear_quant", "x must be e4m3 [M][K], w e4m3 [N][K]")
    if not (x_scale.dtype is _F32 and w_scale.dtype is _F32 and x_scale.numel() == M * G and w_scale.numel() == (N + 127) // 128 * G):
        _refuse("deer_linear_quant", "x_scale must be f32 [M][ceil(K / 128)], w_scale f32 [ceil(N / 128)][ceil(K / 128)]")
    if not (y.dtype is _BF16 and y.numel() == M * N and (residual is None or residual.dtype is _BF16 and residual.numel() == M * N)):
        _refuse("deer_linear_quant", "y and residual must be bf16 [M][N]")
    _check(lib().deer_linear_quant(_ptr(x), _ptr(x_scale), _ptr(w), _ptr(w_scale), _ptr(residual), _ptr(y), M, K, N, _stream(stream)))


def deer_kv_reserve(kv: KVCache, seq_ids: torch.Tensor, k: int, stream=None) -> None:
    _check(lib().deer_kv_reserve(kv.handle, _ptr(seq_ids), seq_ids.numel(), k, _stream(stream)))


def deer_selftest_bounded_wait(kv: KVCache, stream=None) -> None:
    _check(lib().deer_selftest_bounded_wait(kv.handle, _stream(stream)))


def deer_kv_commit(kv: KVCache, seq_ids: torch.Tensor, keep: torch.Tensor, k: int, stream=None) -> None:
    _check(lib().deer_kv_commit(kv.handle, _ptr(seq_ids), _ptr(keep), seq_ids.numel(), k, _stream(stream)))


def deer_kv_status(kv: KVCache, stream=None) -> int:
    code = c_int32(0)
    _check(lib().deer_kv_status(kv.handle, ctypes.byref(code), _stream(stream)))
    return code.value


def deer_block_attn_workspace_bytes(B, k, Hq, Hkv, D, max_seq_len) -> int:
    return lib().deer_block_attn_workspace_bytes(B, k, Hq, Hkv, D, max_seq_len)


def deer_block_attn(kv: KVCache, seq_ids, q, k_blk, v_blk, out, mask, append, scale, max_seq_len, workspace, stream=None):
    B, k, Hq, D = q.shape
    _check(lib().deer_block_attn(kv.handle, _ptr(seq_ids), _ptr(q), _ptr(k_blk), _ptr(v_blk), _ptr(out), B, k, Hq,
                                 int(mask), int(append), float(scale), int(max_seq_len), _ptr(workspace),
                                 workspace.numel() * workspace.element_size() if workspace is not None else 0,
                                 _stream(stream)))


def deer_lmhead_workspace_bytes(M, hid, V) -> int:
    return lib().deer_lmhead_workspace_bytes(M, hid, V)


def deer_lmhead_select(h, w, mode, temperature, draft_ids, out_ids, out_max_logprob, out_lse, out_draft_logit, out_logits,
                       workspace, stream=None):
    M, hid = h.shape
    V = w.shape[0]
    _check(lib().deer_lmhead_select(_ptr(h), _ptr(w), M, hid, V, int(mode), float(temperature), _ptr(draft_ids),
                                    _ptr(out_ids), _ptr(out_max_logprob), _ptr(out_lse), _ptr(out_draft_logit),
                                    _ptr(out_logits), _ptr(workspace),
                                    workspace.numel() * workspace.element_size() if workspace is not None else 0,
                                    _stream(stream)))


def deer_lmhead_static_max_rows() -> int:
    return lib().deer_lmhead_static_max_rows()


def deer_lmhead_select_static(h, w, mode, temperature, draft_ids, out_ids, out_max_logprob, out_lse, out_draft_logit,
                              out_logits, stream=None):
    """deer_lmhead_select for callers that cannot supply (or allocate) a workspace:
    the scratch is a fixed array inside the library, so M is limited to
    deer_lmhead_static_max_rows() and calls on one GPU must not overlap."""
    M, hid = h.shape
    V = w.shape[0]
    _check(lib().deer_lmhead_select_static(_ptr(h), _ptr(w), M, hid, V, int(mode), float(temperature), _ptr(draft_ids),
                                           _ptr(out_ids), _ptr(out_max_logprob), _ptr(out_lse), _ptr(out_draft_logit),
                                           _ptr(out_logits), _stream(stream)))


def deer_accept_workspace_bytes(mode, B, k, V) -> int:
    return lib().deer_accept_workspace_bytes(mode, B, k, V)


def deer_accept(mode, B, k, V, draft_ids, target_ids, target_logits, target_lse, target_draft_logit, temperature,
                draft_logits, u, r, eos_id, accept_len, out_ids, n_out, workspace, stream=None):
    _check(lib().deer_accept(int(mode), B, k, V, _ptr(draft_ids), _ptr(target_ids), _ptr(target_logits), _ptr(target_lse),
                             _ptr(target_draft_logit), float(temperature), _ptr(draft_logits), _ptr(u), _ptr(r), int(eos_id),
                             _ptr(accept_len), _ptr(out_ids), _ptr(n_out), _ptr(workspace),
                             workspace.numel() * workspace.element_size() if workspace is not None else 0,
                             _stream(stream)))


def deer_accept_commit(kv: KVCache, seq_ids, mode, k, draft_ids, target_ids, eos_id, accept_len, out_ids, n_out, stream=None):
    _check(lib().deer_accept_commit(kv.handle, _ptr(seq_ids), int(mode), seq_ids.numel(), k, _ptr(draft_ids), _ptr(target_ids),
                                    int(eos_id), _ptr(accept_len), _ptr(out_ids), _ptr(n_out), _stream(stream)))


def deer_truncate(target_logits, target_lse, temperature, top_k, top_p, tau, lse_trunc, stream=None):
    V = target_logits.shape[-1]
    M = target_logits.numel() // V
    _check(lib().deer_truncate(M, V, _ptr(target_logits), _ptr(target_lse), float(temperature), int(top_k), float(top_p),
                               _ptr(tau), _ptr(lse_trunc), _stream(stream)))


def deer_accept_truncated(mode, B, k, V, draft_ids, target_ids, target_logits, target_lse, target_draft_logit, target_tau,
                          temperature, draft_logits, u, r, eos_id, accept_len, out_ids, n_out, workspace, stream=None):
    _check(lib().deer_accept_truncated(int(mode), B, k, V, _ptr(draft_ids), _ptr(target_ids), _ptr(target_logits),
                                       _ptr(target_lse), _ptr(target_draft_logit), _ptr(target_tau), float(temperature),
                                       _ptr(draft_logits), _ptr(u), _ptr(r), int(eos_id), _ptr(accept_len), _ptr(out_ids),
                                       _ptr(n_out), _ptr(workspace),
                                       workspace.numel() * workspace.element_size() if workspace is not None else 0,
                                       _stream(stream)))


def deer_linear_workspace_bytes(M, K, N) -> int:
    return lib().deer_linear_workspace_bytes(M, K, N)


def deer_linear(x, w, y, residual=None, workspace=None, stream=None):
    M, K = x.shape
    N = w.shape[0]
    _check(lib().deer_linear(_ptr(x), _ptr(w), _ptr(residual), _ptr(y), M, K, N, _ptr(workspace),
                             workspace.numel() * workspace.element_size() if workspace is not None else 0, _stream(stream)))


def deer_rmsnorm(x, gamma, y, eps, stream=None):
    M, hid = x.shape
    _check(lib().deer_rmsnorm(_ptr(x), _ptr(gamma), _ptr(y), M, hid, float(eps), _stream(stream)))


def deer_qk_norm_rope(kv: "KVCache", seq_ids, q, k_blk, q_gamma, k_gamma, eps, theta, stream=None):
    B, k, Hq, _ = q.shape
    _check(lib().deer_qk_norm_rope(kv.handle, _ptr(seq_ids), _ptr(q), _ptr(k_blk), _ptr(q_gamma), _ptr(k_gamma), B, k, Hq,
                                   float(eps), float(theta), _stream(stream)))


def deer_qkv_split_norm_rope(kv: "KVCache", seq_ids, qkv, q, k_blk, v_blk, q_gamma, k_gamma, eps, theta, stream=None):
    B, k, Hq, _ = q.shape
    _check(lib().deer_qkv_split_norm_rope(kv.handle, _ptr(seq_ids), _ptr(qkv), _ptr(q), _ptr(k_blk), _ptr(v_blk), _ptr(q_gamma),
                                          _ptr(k_gamma), B, k, Hq, float(eps), float(theta), _stream(stream)))


def deer_swiglu(gate_up, y, stream=None):
    M, I = y.shape
    _check(lib().deer_swiglu(_ptr(gate_up), _ptr(y), M, I, _stream(stream)))


def deer_layer_workspace_bytes(M, K, N) -> int:
    return lib().deer_layer_workspace_bytes(M, K, N)


def deer_linear_qkv_rope(kv: "KVCache", seq_ids, x, w_qkv, q, k_blk, v_blk, q_gamma, k_gamma, eps, theta, workspace, stream=None):
    B, k, Hq, _ = q.shape
    _check(lib().deer_linear_qkv_rope(kv.handle, _ptr(seq_ids), _ptr(x), _ptr(w_qkv), _ptr(q), _ptr(k_blk), _ptr(v_blk), _ptr(q_gamma),
                                      _ptr(k_gamma), B, k, Hq, x.shape[1], float(eps), float(theta), _ptr(workspace),
                                      workspace.numel() * workspace.element_size(), _stream(stream)))


def deer_linear_residual_norm(x, w, y, residual=None, gamma=None, y_norm=None, eps=1e-6, workspace=None, stream=None):
    M, K = x.shape
    _check(lib().deer_linear_residual_norm(_ptr(x), _ptr(w), _ptr(residual), _ptr(gamma), _ptr(y), _ptr(y_norm), M, K, w.shape[0],
                                           float(eps), _ptr(workspace),
                                           workspace.numel() * workspace.element_size() if workspace is not None else 0,
                                           _stream(stream)))


def deer_linear_swiglu(x, w_pairs, y, stream=None):
    M, K = x.shape
    _check(lib().deer_linear_swiglu(_ptr(x), _ptr(w_pairs), _ptr(y), M, K, y.shape[1], _stream(stream)))


def deer_moe_workspace_bytes(M, hid, E, I, top_k) -> int:
    return lib().deer_moe_workspace_bytes(M, hid, E, I, top_k)


def deer_moe_route(x, w_router, top_k, experts, weights, renormalise=True, workspace=None, stream=None):
    M, hid = x.shape
    E = w_router.shape[0]
    if workspace is None:                      # plumbing: room for the M x E fp32 logits
        workspace = torch.empty(max(16, M * E * 4), dtype=torch.uint8, device=x.device)
    _check(lib().deer_moe_route(_ptr(x), _ptr(w_router), M, hid, E, int(top_k), 1 if renormalise else 0,
                                _ptr(experts), _ptr(weights), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                _stream(stream)))


def deer_moe_mlp(x, w_router, w_gate_up, w_down, y, top_k, workspace, residual=None, stream=None):
    M, hid = x.shape
    E, two_i, _ = w_gate_up.shape
    _check(lib().deer_moe_mlp(_ptr(x), _ptr(w_router), _ptr(w_gate_up), _ptr(w_down), _ptr(residual), _ptr(y), M, hid, E, two_i // 2,
                              int(top_k), _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)))


def deer_draft_stats(B, k, V, draft_ids, draft_logits, workspace, stream=None):
    _check(lib().deer_draft_stats(B, k, V, _ptr(draft_ids), _ptr(draft_logits), _ptr(workspace),
                                  workspace.numel() * workspace.element_size(), _stream(stream)))


def deer_emit(accept_len, out_ids, n_out, eos_id, tokens, n_tokens, finished, keep, flags=0, stream=None, appended=None):
    B, k = out_ids.shape
    _check(lib().deer_emit(B, k, _ptr(accept_len), _ptr(out_ids), _ptr(n_out), int(eos_id), tokens.shape[1], _ptr(tokens),
                           _ptr(n_tokens), _ptr(finished), _ptr(keep), _ptr(appended), int(flags), _stream(stream)))


def deer_block_attn_rows(kv: KVCache, seq_ids, q, k_blk, v_blk, out, row_state, mask, append, scale, max_seq_len, workspace,
                         stream=None):
    B, k, Hq, D = q.shape
    _check(lib().deer_block_attn_rows(kv.handle, _ptr(seq_ids), _ptr(q), _ptr(k_blk), _ptr(v_blk), _ptr(out), _ptr(row_state),
                                      B, k, Hq, int(mask), int(append), float(scale), int(max_seq_len), _ptr(workspace),
                                      workspace.numel() * workspace.element_size() if workspace is not None else 0,
                                      _stream(stream)))


def deer_refill(ids, logprob, log_threshold, row_state, tokens, left=None, stream=None):
    B, k = row_state.shape
    _check(lib().deer_refill(B, k, _ptr(ids), _ptr(logprob), float(log_threshold), _ptr(row_state), _ptr(tokens), _ptr(left),
                             _stream(stream)))


def deer_refresh_rows(appended, row_state, stream=None):
    B, k = row_state.shape
    _check(lib().deer_refresh_rows(B, k, _ptr(appended), _ptr(row_state), _stream(stream)))


def deer_verify_step_host(kv: KVCache, dev: deer_step_dev, w, q_host, k_blk_host, v_blk_host, h_host, draft_ids_host,
                          B, k, Hq, hid, V, scale, max_seq_len, accept_len_host, out_ids_host, n_out_host, stream=None):
    _check(lib().deer_verify_step_host(kv.handle, ctypes.byref(dev), _ptr(w), _ptr(q_host), _ptr(k_blk_host),
                                       _ptr(v_blk_host), _ptr(h_host), _ptr(draft_ids_host), B, k, Hq, hid, V, float(scale),
                                       int(max_seq_len), _ptr(accept_len_host), _ptr(out_ids_host), _ptr(n_out_host),
                                       _stream(stream)))
