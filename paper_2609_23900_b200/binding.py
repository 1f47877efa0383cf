"""Thin ctypes binding of liblumo_gdn.so: argument marshalling only.

Every step of the path (tree conv, tree scan, commit) runs in the CUDA kernels behind the
C ABI declared in include/lumo_gdn.h; this module turns torch tensors into pointers and
error codes into exceptions.  It raises at import if the shared library is missing: there
is no CPU fallback.
"""
from __future__ import annotations

import ctypes
import os
from typing import List, Optional, Sequence

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblumo_gdn.so")
if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it with `python -m paper_2609_23900_b200.build` "
        "(the GDN tree verifier has no CPU fallback)")
_lib = ctypes.CDLL(LIB_PATH)

LUMO_F32, LUMO_BF16 = 0, 1
_DTYPE = {torch.float32: LUMO_F32, torch.bfloat16: LUMO_BF16}

(SEQ_OK, SEQ_BAD_LEN, SEQ_BAD_NODE, SEQ_BAD_ROOT, SEQ_BAD_LINK, SEQ_BAD_ROW, SEQ_TIMEOUT, SEQ_BAD_CTX, SEQ_BAD_PAGE,
 SEQ_NO_PAGES) = range(10)

TABLES = ["depth", "n_child", "child_off", "child_list", "is_leaf", "leaves", "path_off", "path_nodes",
          "anc_win", "slot_inv", "chain_head", "chain_off", "chain_nodes", "chain_level", "cut_nodes",
          "schedule", "schedule_full", "gram_groups", "attn_vis"]

KERNEL_KINDS = ["conv", "scan", "commit", "path", "attn", "attn_merge", "kv_write", "kv_publish",
                "rope", "kv4_write", "kv4_read", "kv4_publish", "kv4_attn", "kv4_merge", "pages", "rows_copy"]

EXPORTS = ["lumo_ctx_create", "lumo_ctx_destroy", "lumo_last_error", "lumo_ctx_scratch_bytes",
           "lumo_ctx_timing_enable", "lumo_ctx_timing_read", "lumo_ctx_set_scan_algo", "lumo_ctx_set_overlap", "lumo_ctx_set_timeout_drill",
           "lumo_tree_desc_create", "lumo_tree_desc_destroy", "lumo_tree_desc_get",
           "lumo_tree_path_from_node", "lumo_gdn_tree_verify", "lumo_gdn_commit",
           "lumo_gdn_tree_scan_static", "lumo_static_stack_bytes", "lumo_conv_rows_per_cta", "lumo_tree_accept", "lumo_select_spine_top3", "lumo_gdn_commit_verify",
           "lumo_kv_write_tree", "lumo_tree_attention", "lumo_kv_publish",
           "lumo_qk_norm_rope", "lumo_kv4_write_tree", "lumo_kv4_append", "lumo_kv4_read", "lumo_kv4_work_bytes", "lumo_kv4_attention",
           "lumo_kv4_publish", "lumo_pages_work_ints", "lumo_pages_init", "lumo_pages_fork", "lumo_pages_reserve", "lumo_pages_free",
           "lumo_pages_compact", "lumo_rows_copy"]


class LumoError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"lumo status {code}: {msg}")
        self.code = code


class _Args(ctypes.Structure):
    """Mirror of lumo_gdn_args."""
    _fields_ = [
        ("Hk", ctypes.c_int32), ("Hv", ctypes.c_int32), ("d", ctypes.c_int32),
        ("in_dtype", ctypes.c_int32), ("gate_dtype", ctypes.c_int32), ("out_dtype", ctypes.c_int32),
        ("scale", ctypes.c_float), ("qk_l2norm", ctypes.c_int32), ("l2_eps", ctypes.c_float),
        ("n_state_rows", ctypes.c_int32),
        ("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
        ("alpha", ctypes.c_void_p), ("beta", ctypes.c_void_p),
        ("x", ctypes.c_void_p), ("conv_w", ctypes.c_void_p), ("conv_b", ctypes.c_void_p),
        ("conv_hist", ctypes.c_void_p),
        ("state", ctypes.c_void_p), ("state_row", ctypes.c_void_p),
        ("out", ctypes.c_void_p),
        ("snapshot_mode", ctypes.c_int32), ("n_snap", ctypes.c_int32),
        ("snap_nodes", ctypes.c_void_p), ("snap_out", ctypes.c_void_p),
        ("status", ctypes.c_void_p),
        ("gate_mode", ctypes.c_int32), ("a_log", ctypes.c_void_p), ("dt_bias", ctypes.c_void_p),
    ]


class _AcceptArgs(ctypes.Structure):
    """Mirror of lumo_accept_args."""
    _fields_ = [("V", ctypes.c_int32), ("mode", ctypes.c_int32), ("token", ctypes.c_void_p),
                ("p_target", ctypes.c_void_p), ("q_draft", ctypes.c_void_p), ("uniforms", ctypes.c_void_p),
                ("noise", ctypes.c_void_p), ("work", ctypes.c_void_p)]


class _SelectArgs(ctypes.Structure):
    """Mirror of lumo_select_args."""
    _fields_ = [("rows", ctypes.c_int32), ("V", ctypes.c_int32), ("dtype", ctypes.c_int32), ("split", ctypes.c_int32),
                ("logits", ctypes.c_void_p)]


class _AttnArgs(ctypes.Structure):
    """Mirror of lumo_attn_args."""
    _fields_ = [("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("dh", ctypes.c_int32), ("scale", ctypes.c_float),
                ("n_cache_rows", ctypes.c_int32), ("max_positions", ctypes.c_int32),
                ("k_cache", ctypes.c_void_p), ("v_cache", ctypes.c_void_p),
                ("ctx_len", ctypes.c_void_p), ("cache_row", ctypes.c_void_p),
                ("q", ctypes.c_void_p), ("k_new", ctypes.c_void_p), ("v_new", ctypes.c_void_p),
                ("out", ctypes.c_void_p), ("lse", ctypes.c_void_p),
                ("kv_layout", ctypes.c_int32), ("n_splits", ctypes.c_int32), ("status", ctypes.c_void_p)]


class _QkArgs(ctypes.Structure):
    """Mirror of lumo_qk_args."""
    _fields_ = [("T", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("dh", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("rot", ctypes.c_int32), ("style", ctypes.c_int32), ("axes", ctypes.c_int32), ("turns", ctypes.c_int32),
                ("section", ctypes.c_int32 * 3), ("normalise", ctypes.c_int32), ("eps", ctypes.c_float), ("weight_offset", ctypes.c_float),
                ("mscale", ctypes.c_float), ("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("q_out", ctypes.c_void_p), ("k_out", ctypes.c_void_p),
                ("q_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64), ("q_out_stride", ctypes.c_int64), ("k_out_stride", ctypes.c_int64),
                ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("inv_freq", ctypes.c_void_p), ("pos", ctypes.c_void_p),
                ("ctx_len", ctypes.c_void_p)]


class _Kv4Args(ctypes.Structure):
    """Mirror of lumo_kv4_args."""
    _fields_ = [("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("dh", ctypes.c_int32), ("scale", ctypes.c_float),
                ("n_rows", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("k_exp", ctypes.c_int32), ("v_exp", ctypes.c_int32), ("pages", ctypes.c_void_p), ("table", ctypes.c_void_p),
                ("refs", ctypes.c_void_p), ("ctx_len", ctypes.c_void_p), ("cache_row", ctypes.c_void_p), ("q", ctypes.c_void_p),
                ("k_new", ctypes.c_void_p), ("v_new", ctypes.c_void_p), ("q_stride", ctypes.c_int64), ("kv_stride", ctypes.c_int64),
                ("out", ctypes.c_void_p), ("out_dtype", ctypes.c_int32), ("lse", ctypes.c_void_p), ("n_splits", ctypes.c_int32),
                ("status", ctypes.c_void_p), ("work", ctypes.c_void_p), ("work_bytes", ctypes.c_int64)]


class _PageTableArgs(ctypes.Structure):
    """Mirror of lumo_page_table."""
    _fields_ = [("n_rows", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("table", ctypes.c_void_p), ("row_pages", ctypes.c_void_p), ("refs", ctypes.c_void_p), ("free_list", ctypes.c_void_p),
                ("free_count", ctypes.c_void_p), ("work", ctypes.c_void_p), ("n_pools", ctypes.c_int32), ("pools", ctypes.c_void_p),
                ("page_bytes", ctypes.c_int64)]


_lib.lumo_ctx_create.argtypes = [ctypes.c_int, ctypes.POINTER(ctypes.c_void_p)]
_lib.lumo_ctx_destroy.argtypes = [ctypes.c_void_p]
_lib.lumo_ctx_destroy.restype = None
_lib.lumo_last_error.argtypes = [ctypes.c_void_p]
_lib.lumo_last_error.restype = ctypes.c_char_p
_lib.lumo_ctx_scratch_bytes.argtypes = [ctypes.c_void_p]
_lib.lumo_ctx_scratch_bytes.restype = ctypes.c_int64
_lib.lumo_ctx_set_scan_algo.argtypes = [ctypes.c_void_p, ctypes.c_int]
_lib.lumo_ctx_set_overlap.argtypes = [ctypes.c_void_p, ctypes.c_int]
_lib.lumo_ctx_set_timeout_drill.argtypes = [ctypes.c_void_p, ctypes.c_int]
_lib.lumo_ctx_timing_enable.argtypes = [ctypes.c_void_p, ctypes.c_int]
_lib.lumo_ctx_timing_read.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int,
                                      ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_double)]
_lib.lumo_tree_desc_create.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                       ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                       ctypes.POINTER(ctypes.c_void_p)]
_lib.lumo_tree_desc_destroy.argtypes = [ctypes.c_void_p]
_lib.lumo_tree_desc_destroy.restype = None
_lib.lumo_tree_desc_get.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int,
                                    ctypes.POINTER(ctypes.POINTER(ctypes.c_int32)),
                                    ctypes.POINTER(ctypes.c_int64)]
_lib.lumo_tree_path_from_node.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int,
                                          ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
_lib.lumo_gdn_tree_verify.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(_Args), ctypes.c_int,
                                      ctypes.c_void_p]
_lib.lumo_gdn_tree_scan_static.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(_Args), ctypes.c_int,
                                           ctypes.c_void_p]
_lib.lumo_static_stack_bytes.restype = ctypes.c_int64
_lib.lumo_conv_rows_per_cta.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int]
_lib.lumo_gdn_commit_verify.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                        ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p]
_lib.lumo_select_spine_top3.argtypes = [ctypes.c_void_p, ctypes.POINTER(_SelectArgs), ctypes.c_void_p, ctypes.c_void_p,
                                        ctypes.c_void_p]
_lib.lumo_tree_accept.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(_AcceptArgs), ctypes.c_int,
                                  ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
_lib.lumo_gdn_commit.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(_Args), ctypes.c_int,
                                 ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p]


_lib.lumo_kv_write_tree.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(_AttnArgs), ctypes.c_int, ctypes.c_void_p]
_lib.lumo_tree_attention.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(_AttnArgs), ctypes.c_int, ctypes.c_void_p]
_lib.lumo_kv_publish.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(_AttnArgs), ctypes.c_int,
                                 ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p]


_lib.lumo_qk_norm_rope.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(_QkArgs), ctypes.c_void_p]
for _f in (_lib.lumo_kv4_write_tree, _lib.lumo_kv4_attention):
    _f.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(_Kv4Args), ctypes.c_int, ctypes.c_void_p]
_lib.lumo_kv4_append.argtypes = [ctypes.c_void_p, ctypes.POINTER(_Kv4Args), ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p,
                                 ctypes.c_void_p, ctypes.c_void_p]
_lib.lumo_kv4_read.argtypes = [ctypes.c_void_p, ctypes.POINTER(_Kv4Args), ctypes.c_int] + [ctypes.c_void_p] * 6
_lib.lumo_kv4_work_bytes.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_int]
_lib.lumo_kv4_work_bytes.restype = ctypes.c_int64
_lib.lumo_kv4_publish.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(_Kv4Args), ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p,
                                  ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p]
_lib.lumo_pages_work_ints.argtypes = [ctypes.c_int, ctypes.c_int]
_lib.lumo_pages_work_ints.restype = ctypes.c_int64
_lib.lumo_pages_init.argtypes = [ctypes.c_void_p, ctypes.POINTER(_PageTableArgs), ctypes.c_void_p]
_lib.lumo_pages_compact.argtypes = [ctypes.c_void_p, ctypes.POINTER(_PageTableArgs), ctypes.c_void_p]
for _f in (_lib.lumo_pages_fork, _lib.lumo_pages_free):
    _f.argtypes = [ctypes.c_void_p, ctypes.POINTER(_PageTableArgs), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p]
_lib.lumo_pages_reserve.argtypes = [ctypes.c_void_p, ctypes.POINTER(_PageTableArgs), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int,
                                    ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p]
_lib.lumo_rows_copy.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p,
                                ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p]

_ACCEPT_MODES = {"greedy": 0, "rejection": 1}
_SELECT_DTYPES = {torch.float32: 0, torch.bfloat16: 1}


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("tensors passed to the library must be contiguous CUDA tensors")
    return t.data_ptr()


def _rows_ptr(t: Optional[torch.Tensor], heads: int, dh: int, name: str):
    """Pointer and token stride of a tensor [..., heads, dh] whose heads are adjacent and whose tokens may be parts of longer rows."""
    if t is None:
        return None, 0
    if not t.is_cuda or t.shape[-2:] != (heads, dh) or t.stride(-1) != 1 or (heads > 1 and t.stride(-2) != dh):
        raise ValueError(f"{name} must be a CUDA tensor [..., {heads}, {dh}] with adjacent heads")
    if t.is_contiguous():
        return t.data_ptr(), 0
    axes = [(n, st) for n, st in zip(t.shape[:-2], t.stride()[:-2]) if n != 1]      # (an axis of one entry has no say in the spacing)
    stride, tokens = axes[-1][1], 1
    for n, st in reversed(axes):
        if st != stride * tokens:
            raise ValueError(f"{name}: the tokens must be evenly spaced")
        tokens *= n
    if stride < heads * dh:                                  # 0 of an expanded tensor among them, which the library takes for heads * dh
        raise ValueError(f"{name}: the tokens must not share elements")
    return t.data_ptr(), stride


def _int32(**tensors):
    for name, t in tensors.items():
        if t is not None and t.dtype != torch.int32:
            raise ValueError(f"{name} must be int32")


def _listed(first: torch.Tensor, **tensors) -> int:
    """Length of a call's list: every int32 tensor of it has that many entries, ``status`` at least."""
    n = first.numel()
    for name, t in tensors.items():
        if t is not None and (t.dtype != torch.int32 or (t.numel() < n if name == "status" else t.numel() != n)):
            raise ValueError(f"{name} must be int32 with one entry per listed row or token")
    return n


_ANY = 1 << 62           # room of a tensor that is not given: the library says which ones a call needs
_KV4_ROOM = ("ctx_len, cache_row or status", "q, out or lse", "k_new and v_new")       # a Kv4Layer's tensors by what a call counts in them


def pages_work_ints(n_rows: int, n_pages: int) -> int:
    """Ints of scratch a page table's calls need."""
    return int(_lib.lumo_pages_work_ints(int(n_rows), int(n_pages)))


_cuda_ready = torch.cuda.is_initialized
_cuda_device = getattr(torch._C, "_cuda_getDevice", None)              # private: another build of torch may lack either
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    # the current stream's handle without building a Stream object (0.1 against 3.2 us per call, measured)
    if _raw_stream and _cuda_device and _cuda_ready():
        return _raw_stream(_cuda_device())
    return torch.cuda.current_stream().cuda_stream


class Context:
    """lumo_ctx: one per device."""

    def __init__(self, device: int = 0):
        h = ctypes.c_void_p()
        rc = _lib.lumo_ctx_create(int(device), ctypes.byref(h))
        if rc != 0:
            raise LumoError(rc, _lib.lumo_last_error(None).decode())
        self._h = h
        self.device = int(device)

    def _check(self, rc: int):
        if rc:
            raise LumoError(rc, _lib.lumo_last_error(self._h).decode())

    @property
    def scratch_bytes(self) -> int:
        return _lib.lumo_ctx_scratch_bytes(self._h)

    def set_scan_algo(self, algo: str = "auto"):
        """"auto" | "rank1" | "gram" | "solve" | "direct" (Gram form with the closed-form tail) | "tensor" (the same with
        the output sum on the tensor core): which scan kernel verify uses."""
        self._check(_lib.lumo_ctx_set_scan_algo(self._h, {"auto": 0, "rank1": 1, "gram": 2, "solve": 3, "direct": 4, "tensor": 5}[algo]))

    def set_timeout_drill(self, on: bool):
        """Test aid: the tensor-core scans and the 4-bit attention issue nothing asynchronous, so their bounded waits run out."""
        self._check(_lib.lumo_ctx_set_timeout_drill(self._h, int(on)))

    def set_overlap(self, on: bool = True):
        """Programmatic dependent launch of the library's kernels (default on); off: plain stream order."""
        self._check(_lib.lumo_ctx_set_overlap(self._h, int(on)))

    def timing_enable(self, on: bool = True):
        self._check(_lib.lumo_ctx_timing_enable(self._h, int(on)))

    def timing_read(self, reset: bool = True) -> dict:
        """{kernel kind: (launches, total device ms)} of the launches recorded since the last reset."""
        out = {}
        for i, name in enumerate(KERNEL_KINDS):
            n, ms = ctypes.c_int64(), ctypes.c_double()
            last = reset and i == len(KERNEL_KINDS) - 1
            self._check(_lib.lumo_ctx_timing_read(self._h, i, int(last), ctypes.byref(n), ctypes.byref(ms)))
            out[name] = (n.value, ms.value)
        return out

    def close(self):
        if self._h:
            _lib.lumo_ctx_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- entry points -------------------------------------------------------------------
    def tree_desc(self, parent, slot=None, n_slots: Optional[int] = None, depth=None) -> "TreeDesc":
        return TreeDesc(self, parent, slot, n_slots, depth)

    def path_from_node(self, desc: "TreeDesc", node: torch.Tensor, lmax: int, accepted: torch.Tensor,
                       length: torch.Tensor, status: Optional[torch.Tensor] = None, stream=None):
        self._check(_lib.lumo_tree_path_from_node(self._h, desc._h, _ptr(node), int(lmax), _ptr(accepted),
                                                  _ptr(length), _ptr(status), _stream(stream)))

    @staticmethod
    def pack(layers: Sequence["GdnLayer"]):
        """ctypes array of the layers' argument blocks (reusable across calls)."""
        return (_Args * len(layers))(*[l.args for l in layers])

    def verify(self, desc: "TreeDesc", layers, stream=None):
        arr = layers if isinstance(layers, ctypes.Array) else self.pack(layers)
        self._check(_lib.lumo_gdn_tree_verify(self._h, desc._h, arr, len(layers), _stream(stream)))

    def scan_static(self, desc: "TreeDesc", layers, stream=None):
        """The tree scan with the library's built-in, fixed-size stack: for callers that must not
        allocate device memory.  Scan only (no convolution); refuses shapes that need more stack than
        ``static_stack_bytes()``.  Calls that overlap on the GPU race on the shared stack."""
        arr = layers if isinstance(layers, ctypes.Array) else self.pack(layers)
        self._check(_lib.lumo_gdn_tree_scan_static(self._h, desc._h, arr, len(arr), _stream(stream)))

    def conv_rows_per_cta(self, desc: "TreeDesc", Hk: int, Hv: int, d: int, n_layers: int = 1) -> int:
        """Which instantiation of the tree convolution (16, 8 or 4 entries per warp) this shape launches."""
        return int(_lib.lumo_conv_rows_per_cta(self._h, desc._h, int(Hk), int(Hv), int(d), int(n_layers)))

    @staticmethod
    def static_stack_bytes() -> int:
        return int(_lib.lumo_static_stack_bytes())

    def accept(self, desc: "TreeDesc", *, token, p_target, accepted, length, next_token, final_node,
               mode: str = "greedy", q_draft=None, uniforms=None, noise=None, work=None, stream=None):
        """Acceptance walk on the device: fills accepted [B, lmax], length, next_token, final_node."""
        # filled by position and passed as it is: 1.6 us of host time for block and call, by name and by reference 2.3
        a = _AcceptArgs(p_target.shape[-1], _ACCEPT_MODES[mode], _ptr(token), _ptr(p_target), _ptr(q_draft), _ptr(uniforms),
                        _ptr(noise), _ptr(work))
        self._check(_lib.lumo_tree_accept(self._h, desc._h, a, accepted.shape[1], _ptr(accepted),
                                          _ptr(length), _ptr(next_token), _ptr(final_node), _stream(stream)))

    def commit_verify(self, prev_desc: "TreeDesc", prev_layers, accepted: torch.Tensor, length: torch.Tensor,
                      desc: "TreeDesc", layers, stream=None):
        """commit(prev_desc, prev_layers, accepted, length) then verify(desc, layers), the state read once."""
        parr = prev_layers if isinstance(prev_layers, ctypes.Array) else self.pack(prev_layers)
        arr = layers if isinstance(layers, ctypes.Array) else self.pack(layers)
        self._check(_lib.lumo_gdn_commit_verify(self._h, prev_desc._h, parr, _ptr(accepted), _ptr(length),
                                                int(accepted.shape[1]), desc._h, arr, len(layers), _stream(stream)))

    def select_spine_top3(self, logits: torch.Tensor, spine: torch.Tensor, cand: torch.Tensor, split: int = 0,
                          stream=None):
        """Fused draft selection: spine [R] and cand [R, 3] (int32, device) from logits [R, V] (f32 or bf16)."""
        shape = logits.shape
        a = _SelectArgs(shape[0], shape[1], _SELECT_DTYPES[logits.dtype], int(split), _ptr(logits))
        self._check(_lib.lumo_select_spine_top3(self._h, a, _ptr(spine), _ptr(cand), _stream(stream)))

    def commit(self, desc: "TreeDesc", layers, accepted: torch.Tensor, length: torch.Tensor, stream=None):
        arr = layers if isinstance(layers, ctypes.Array) else self.pack(layers)
        self._check(_lib.lumo_gdn_commit(self._h, desc._h, arr, len(layers), _ptr(accepted), _ptr(length),
                                         int(accepted.shape[1]), _stream(stream)))


    # ---- attention half ----
    @staticmethod
    def pack_attn(layers: Sequence["AttnLayer"]):
        return (_AttnArgs * len(layers))(*[l.args for l in layers])

    def kv_write_tree(self, desc: "TreeDesc", layers, stream=None):
        arr = layers if isinstance(layers, ctypes.Array) else self.pack_attn(layers)
        self._check(_lib.lumo_kv_write_tree(self._h, desc._h, arr, len(arr), _stream(stream)))

    def tree_attention(self, desc: "TreeDesc", layers, stream=None):
        arr = layers if isinstance(layers, ctypes.Array) else self.pack_attn(layers)
        self._check(_lib.lumo_tree_attention(self._h, desc._h, arr, len(arr), _stream(stream)))

    def kv_publish(self, desc: "TreeDesc", layers, accepted: torch.Tensor, length: torch.Tensor,
                   ctx_len_out: Optional[torch.Tensor] = None, stream=None):
        arr = layers if isinstance(layers, ctypes.Array) else self.pack_attn(layers)
        self._check(_lib.lumo_kv_publish(self._h, desc._h, arr, len(arr), _ptr(accepted), _ptr(length),
                                         int(accepted.shape[1]), _ptr(ctx_len_out), _stream(stream)))

    # ---- norm and rotation, the paged 4-bit cache ----
    def qk_norm_rope(self, layer: "QkNormRope", desc: Optional["TreeDesc"] = None, stream=None):
        """Norm of every query and key head and the position rotation, in one pass; with ``desc`` the tokens are its trees' nodes."""
        if desc is not None and desc.B > layer.sequences:
            raise ValueError("ctx_len must be [B], a length for each of the trees")
        self._check(_lib.lumo_qk_norm_rope(self._h, desc._h if desc is not None else None, layer.args, _stream(stream)))

    @staticmethod
    def pack_kv4(layers: Sequence["Kv4Layer"]):
        """ctypes array of the layers' argument blocks (reusable across calls); keeps the layers, and knows how much their tensors hold."""
        arr = (_Kv4Args * len(layers))(*[l.args for l in layers])
        arr.layers = list(layers)
        arr.room = tuple(min((l.room[i] for l in layers), default=_ANY) for i in range(len(_KV4_ROOM)))
        return arr

    @staticmethod
    def _kv4(layers, sequences: int = 0, kind: int = 0, tokens: int = 0):
        """Packed layers whose tensors hold a word for each of ``sequences`` and, of one kind of tensors, ``tokens`` tokens."""
        room = getattr(layers, "room", None)
        if room is None:
            if isinstance(layers, ctypes.Array):
                raise ValueError("an array of layers has to come from pack_kv4")
            layers = Context.pack_kv4(layers)
            room = layers.room
        if sequences > room[0] or tokens > room[kind]:
            i = 0 if sequences > room[0] else kind
            raise ValueError(f"{_KV4_ROOM[i]} too small: room for {room[i]}, {sequences if i == 0 else tokens} needed")
        return layers

    def kv4_work_bytes(self, desc: "TreeDesc", Hq: int, Hkv: int, n_splits: int = 0) -> int:
        """Bytes of workspace ``kv4_attention`` needs (Kv4Layer's ``work``)."""
        return int(_lib.lumo_kv4_work_bytes(self._h, desc._h, int(Hq), int(Hkv), int(n_splits)))

    def kv4_write_tree(self, desc: "TreeDesc", layers, stream=None):
        arr = self._kv4(layers, desc.B, 2, desc.nodes)
        self._check(_lib.lumo_kv4_write_tree(self._h, desc._h, arr, len(arr), _stream(stream)))

    def kv4_append(self, layers, tok_row: torch.Tensor, tok_pos: torch.Tensor, status: Optional[torch.Tensor] = None, stream=None):
        """Entries of listed tokens (int32 rows and positions, [T]); ``status``, if given, gets a word per token."""
        T = _listed(tok_row, tok_row=tok_row, tok_pos=tok_pos, status=status)
        arr = self._kv4(layers, 0, 2, T)
        self._check(_lib.lumo_kv4_append(self._h, arr, len(arr), T, _ptr(tok_row), _ptr(tok_pos), _ptr(status), _stream(stream)))

    def kv4_read(self, layer: "Kv4Layer", tok_row: torch.Tensor, tok_pos: torch.Tensor, k_out: torch.Tensor, v_out: torch.Tensor,
                 status: Optional[torch.Tensor] = None, stream=None):
        """The listed tokens' entries as bf16 [T, Hkv, dh]."""
        T = _listed(tok_row, tok_row=tok_row, tok_pos=tok_pos, status=status)
        for name, o in (("k_out", k_out), ("v_out", v_out)):
            if o.dtype != torch.bfloat16 or not o.is_contiguous() or o.numel() < T * layer.args.Hkv * layer.args.dh:
                raise ValueError(f"{name} must be contiguous bf16 [T, Hkv, dh]")
        self._check(_lib.lumo_kv4_read(self._h, layer.args, T, _ptr(tok_row), _ptr(tok_pos), _ptr(k_out), _ptr(v_out), _ptr(status),
                                       _stream(stream)))

    def kv4_attention(self, desc: "TreeDesc", layers, stream=None):
        arr = self._kv4(layers, desc.B, 1, desc.nodes)
        self._check(_lib.lumo_kv4_attention(self._h, desc._h, arr, len(arr), _stream(stream)))

    def kv4_publish(self, desc: "TreeDesc", layers, accepted: torch.Tensor, length: torch.Tensor,
                    ctx_len_out: Optional[torch.Tensor] = None, stream=None):
        arr = self._kv4(layers, desc.B)
        shape, B = accepted.shape, desc.B
        if (len(shape) != 2 or shape[0] < B or length.numel() < B or accepted.dtype != torch.int32 or length.dtype != torch.int32 or
                ctx_len_out is not None and (ctx_len_out.numel() < B or ctx_len_out.dtype != torch.int32)):
            raise ValueError("accepted must be int32 [B, lmax], length and ctx_len_out int32 [B]")
        self._check(_lib.lumo_kv4_publish(self._h, desc._h, arr, len(arr), _ptr(accepted), _ptr(length), shape[1],
                                          _ptr(ctx_len_out), _stream(stream)))

    # ---- pages ----
    def pages_init(self, table: "PageTable", stream=None):
        self._check(_lib.lumo_pages_init(self._h, table.args, _stream(stream)))

    def pages_fork(self, table: "PageTable", src: torch.Tensor, dst: torch.Tensor, status: Optional[torch.Tensor] = None, stream=None):
        """Row dst[i], empty so far, shares the pages of row src[i]."""
        n = _listed(src, src=src, dst=dst, status=status)
        self._check(_lib.lumo_pages_fork(self._h, table.args, _ptr(src), _ptr(dst), n, _ptr(status), _stream(stream)))

    def pages_reserve(self, table: "PageTable", rows: torch.Tensor, start: torch.Tensor, end: Optional[torch.Tensor] = None, add: int = 0,
                      status: Optional[torch.Tensor] = None, stream=None):
        """Positions [start, end) (or [start, start + add)) of the rows made writable: shared pages copied, missing ones added."""
        n = _listed(rows, rows=rows, start=start, end=end, status=status)
        self._check(_lib.lumo_pages_reserve(self._h, table.args, _ptr(rows), _ptr(start), _ptr(end), int(add), n, _ptr(status),
                                            _stream(stream)))

    def pages_free(self, table: "PageTable", rows: torch.Tensor, keep: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                   stream=None):
        """Pages behind the rows' first ``keep`` positions (all pages without it) given back."""
        n = _listed(rows, rows=rows, keep=keep, status=status)
        self._check(_lib.lumo_pages_free(self._h, table.args, _ptr(rows), _ptr(keep), n, _ptr(status), _stream(stream)))

    def pages_compact(self, table: "PageTable", stream=None):
        """The pages in use moved to the lowest numbers, in all pools and tables."""
        self._check(_lib.lumo_pages_compact(self._h, table.args, _stream(stream)))

    def rows_copy(self, blocks: "RowBlocks", src: torch.Tensor, dst: torch.Tensor, status: Optional[torch.Tensor] = None, stream=None):
        """Row src[i] of every block copied to its row dst[i]."""
        n = _listed(src, src=src, dst=dst, status=status)
        self._check(_lib.lumo_rows_copy(self._h, blocks.ptrs, blocks.row_bytes, len(blocks.tensors), blocks.n_rows, _ptr(src), _ptr(dst),
                                        n, _ptr(status), _stream(stream)))


class TreeDesc:
    """lumo_tree_desc built from host arrays parent [B, N] (and optional slot, depth)."""

    def __init__(self, ctx: Context, parent, slot=None, n_slots: Optional[int] = None, depth=None):
        parent = np.ascontiguousarray(parent, dtype=np.int32)
        if parent.ndim != 2:
            raise ValueError("parent must be [B, N]")
        self.B, self.N = parent.shape
        slot_a = None if slot is None else np.ascontiguousarray(slot, dtype=np.int32)
        depth_a = None if depth is None else np.ascontiguousarray(depth, dtype=np.int32)
        self.nodes = self.B * self.N
        self.Ns = int(n_slots) if n_slots is not None else self.N
        h = ctypes.c_void_p()
        rc = _lib.lumo_tree_desc_create(
            ctx._h, self.B, self.N, self.Ns, parent.ctypes.data,
            None if depth_a is None else depth_a.ctypes.data,
            None if slot_a is None else slot_a.ctypes.data, ctypes.byref(h))
        ctx._check(rc)
        self._h = h
        self._ctx = ctx

    def table(self, name: str, b: int = 0) -> np.ndarray:
        data = ctypes.POINTER(ctypes.c_int32)()
        count = ctypes.c_int64()
        rc = _lib.lumo_tree_desc_get(self._h, TABLES.index(name), int(b), ctypes.byref(data), ctypes.byref(count))
        if rc != 0:
            raise LumoError(rc, "bad table request")
        return np.ctypeslib.as_array(data, shape=(count.value,)).copy() if count.value else np.zeros(0, np.int32)

    def close(self):
        if self._h:
            _lib.lumo_tree_desc_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class GdnLayer:
    """lumo_gdn_args for one layer; keeps the tensors alive."""

    def __init__(self, *, Hk: int, Hv: int, d: int, q, k, v, alpha, beta, state, state_row, out=None,
                 x=None, conv_w=None, conv_b=None, conv_hist=None, scale: float = 1.0,
                 qk_l2norm: bool = False, l2_eps: float = 1e-6, snapshot_mode: int = 0, snap_nodes=None,
                 snap_out=None, status=None, a_log=None, dt_bias=None):
        """a_log and dt_bias ([Hv] float32) switch to raw gate inputs: alpha and beta are then activated in
        the kernels."""
        self.tensors = dict(q=q, k=k, v=v, alpha=alpha, beta=beta, state=state, state_row=state_row, out=out,
                            x=x, conv_w=conv_w, conv_b=conv_b, conv_hist=conv_hist, snap_nodes=snap_nodes,
                            snap_out=snap_out, status=status, a_log=a_log, dt_bias=dt_bias)
        if (a_log is None) != (dt_bias is None):
            raise ValueError("a_log and dt_bias go together")
        for t in (a_log, dt_bias):
            if t is not None and t.dtype != torch.float32:
                raise ValueError("a_log and dt_bias must be float32")
        if state.dtype != torch.float32:
            raise ValueError("state must be float32")
        for name in ("state_row", "snap_nodes", "status"):
            t = self.tensors[name]
            if t is not None and t.dtype != torch.int32:
                raise ValueError(f"{name} must be int32")
        if alpha.dtype != beta.dtype or q.dtype != k.dtype or q.dtype != v.dtype:
            raise ValueError("q/k/v (and alpha/beta) must share a dtype")
        for name in ("x", "conv_w", "conv_b", "conv_hist"):
            t = self.tensors[name]
            if t is not None and t.dtype != q.dtype:
                raise ValueError(f"{name} must have the dtype of q/k/v")
        a = _Args()
        a.Hk, a.Hv, a.d = Hk, Hv, d
        a.in_dtype = _DTYPE[q.dtype]
        a.gate_dtype = _DTYPE[alpha.dtype]
        a.out_dtype = _DTYPE[out.dtype] if out is not None else LUMO_F32
        a.scale, a.qk_l2norm, a.l2_eps = float(scale), int(qk_l2norm), float(l2_eps)
        a.n_state_rows = int(state.shape[0])
        a.snapshot_mode = int(snapshot_mode)
        a.n_snap = int(snap_nodes.shape[1]) if snap_nodes is not None else 0
        a.gate_mode = 0 if a_log is None else 1
        for name in ("q", "k", "v", "alpha", "beta", "x", "conv_w", "conv_b", "conv_hist", "state",
                     "state_row", "out", "snap_nodes", "snap_out", "status", "a_log", "dt_bias"):
            setattr(a, name, _ptr(self.tensors[name]))
        self.args = a


class AttnLayer:
    """lumo_attn_args for one full-attention layer; keeps the tensors alive."""

    def __init__(self, *, Hq: int, Hkv: int, k_cache, v_cache, ctx_len, cache_row, scale: float, q=None, k_new=None,
                 v_new=None, out=None, lse=None, n_splits: int = 0, status=None, kv_layout: int = 0):
        """kv_layout 0: caches are [rows, positions, Hkv, dh]; 1: [rows, Hkv, positions, dh]."""
        self.tensors = dict(k_cache=k_cache, v_cache=v_cache, ctx_len=ctx_len, cache_row=cache_row, q=q, k_new=k_new,
                            v_new=v_new, out=out, lse=lse, status=status)
        if k_cache.dtype != torch.bfloat16 or v_cache.dtype != torch.bfloat16 or k_cache.shape != v_cache.shape:
            raise ValueError("k_cache and v_cache must be bfloat16 tensors of one shape [rows, positions, Hkv, dh]")
        if k_cache.dim() != 4 or k_cache.shape[1 if kv_layout else 2] != Hkv:
            raise ValueError("cache shape must be [rows, positions, Hkv, dh] (layout 0) or [rows, Hkv, positions, dh] (layout 1)")
        for name in ("q", "k_new", "v_new"):
            t = self.tensors[name]
            if t is not None and t.dtype != torch.bfloat16:
                raise ValueError(f"{name} must be bfloat16")
        for name in ("out", "lse"):
            t = self.tensors[name]
            if t is not None and t.dtype != torch.float32:
                raise ValueError(f"{name} must be float32")
        for name in ("ctx_len", "cache_row", "status"):
            t = self.tensors[name]
            if t is not None and t.dtype != torch.int32:
                raise ValueError(f"{name} must be int32")
        a = _AttnArgs()
        a.Hq, a.Hkv, a.dh, a.scale = int(Hq), int(Hkv), int(k_cache.shape[3]), float(scale)
        a.n_cache_rows, a.max_positions = int(k_cache.shape[0]), int(k_cache.shape[2 if kv_layout else 1])
        a.n_splits = int(n_splits)
        a.kv_layout = int(kv_layout)
        for name in self.tensors:
            setattr(a, name, _ptr(self.tensors[name]))
        self.args = a


class QkNormRope:
    """lumo_qk_args: the norm and rotation in front of one full-attention layer; keeps the tensors alive."""

    def __init__(self, *, q, q_out, k=None, k_out=None, inv_freq=None, q_weight=None, k_weight=None, normalise: bool = True, eps: float = 1e-6,
                 weight_offset: float = 0.0, mscale: float = 1.0, style: str = "half", pos=None, ctx_len=None, sections=None, turns: bool = False):
        """q [..., Hq, dh], k [..., Hkv, dh] (tokens may be parts of longer rows), outputs alike; inv_freq [rot / 2] fp32.  pos: int32 [T], or
        [3, T] with ``sections``, the pairs of each axis, in blocks or (``turns``) taking turns; without pos the call's trees give the
        positions, behind ctx_len [B].  style: "half" or "pairs"."""
        self.tensors = dict(q=q, k=k, q_out=q_out, k_out=k_out, inv_freq=inv_freq, q_weight=q_weight, k_weight=k_weight, pos=pos, ctx_len=ctx_len)
        for name in ("k", "q_out", "k_out", "q_weight", "k_weight"):
            t = self.tensors[name]
            if t is not None and t.dtype != q.dtype:
                raise ValueError(f"{name} must have the dtype of q")
        if inv_freq is not None and inv_freq.dtype != torch.float32:
            raise ValueError("inv_freq must be float32")
        _int32(pos=pos, ctx_len=ctx_len)
        Hq, dh = int(q.shape[-2]), int(q.shape[-1])
        Hkv = int(k.shape[-2]) if k is not None else 0
        a = _QkArgs()
        a.T, a.Hq, a.Hkv, a.dh, a.dtype = q.numel() // (Hq * dh), Hq, Hkv, dh, _DTYPE[q.dtype]
        if (k is None) != (k_out is None) or q_out.shape != q.shape or (k is not None and (k_out.shape != k.shape or k.numel() != a.T * Hkv * dh)):
            raise ValueError("outputs must have their inputs' shapes, and q and k the same tokens")
        a.rot = 2 * int(inv_freq.numel()) if inv_freq is not None else 0
        a.style, a.turns = {"half": 0, "pairs": 1}[style], int(turns)
        a.axes = 3 if sections is not None else 1
        if sections is not None:
            a.section[:] = [int(v) for v in sections]
        if pos is not None and pos.numel() != a.axes * a.T:
            raise ValueError("pos must have a number per axis and token")
        for name, t in (("q_weight", q_weight), ("k_weight", k_weight)):
            if t is not None and t.numel() != dh:
                raise ValueError(f"{name} must have dh elements")
        a.normalise, a.eps, a.weight_offset, a.mscale = int(normalise), float(eps), float(weight_offset), float(mscale)
        for name, heads in (("q", Hq), ("k", Hkv), ("q_out", Hq), ("k_out", Hkv)):
            ptr, stride = _rows_ptr(self.tensors[name], heads, dh, name)
            setattr(a, name, ptr)
            setattr(a, name + "_stride", stride)
        for name in ("q_weight", "k_weight", "inv_freq", "pos", "ctx_len"):
            setattr(a, name, _ptr(self.tensors[name]))
        self.args = a
        self.sequences = ctx_len.numel() if ctx_len is not None and pos is None and a.rot else _ANY      # whose lengths are read


class Kv4Layer:
    """lumo_kv4_args for one full-attention layer over a paged 4-bit cache; keeps the tensors alive."""

    def __init__(self, *, Hq: int, Hkv: int, pages, table, page_size: int, scale: float = 1.0, ctx_len=None, cache_row=None, refs=None, q=None,
                 k_new=None, v_new=None, out=None, lse=None, k_exp: int = 0, v_exp: int = 0, n_splits: int = 0, status=None, work=None):
        """pages: uint8 [n_pages, Hkv, 2, page_size * 72]; table: int32 [rows, max_pages]."""
        self.tensors = dict(pages=pages, table=table, refs=refs, ctx_len=ctx_len, cache_row=cache_row, q=q, k_new=k_new, v_new=v_new, out=out,
                            lse=lse, status=status, work=work)
        if pages.dtype != torch.uint8 or pages.dim() != 4 or tuple(pages.shape[1:]) != (Hkv, 2, page_size * 72):
            raise ValueError("pages must be a uint8 tensor [n_pages, Hkv, 2, page_size * 72]")
        if table.dim() != 2:
            raise ValueError("table must be [rows, max_pages]")
        if refs is not None and refs.numel() != pages.shape[0]:
            raise ValueError("refs must be [n_pages]")
        _int32(table=table, refs=refs, ctx_len=ctx_len, cache_row=cache_row, status=status)
        for name in ("q", "k_new", "v_new"):
            t = self.tensors[name]
            if t is not None and t.dtype != torch.bfloat16:
                raise ValueError(f"{name} must be bfloat16")
        if lse is not None and lse.dtype != torch.float32:
            raise ValueError("lse must be float32")
        a = _Kv4Args()
        a.Hq, a.Hkv, a.dh, a.scale = int(Hq), int(Hkv), 128, float(scale)
        a.n_rows, a.max_pages = int(table.shape[0]), int(table.shape[1])
        a.n_pages, a.page_size = int(pages.shape[0]), int(page_size)
        a.k_exp, a.v_exp, a.n_splits = int(k_exp), int(v_exp), int(n_splits)
        a.out_dtype = _DTYPE[out.dtype] if out is not None else LUMO_F32
        a.q, a.q_stride = _rows_ptr(q, int(Hq), 128, "q")
        a.k_new, a.kv_stride = _rows_ptr(k_new, int(Hkv), 128, "k_new")
        a.v_new, v_stride = _rows_ptr(v_new, int(Hkv), 128, "v_new")
        if k_new is not None and v_new is not None and v_stride != a.kv_stride:
            raise ValueError("k_new and v_new must have the same token stride")
        for name in ("pages", "table", "refs", "ctx_len", "cache_row", "out", "lse", "status", "work"):
            setattr(a, name, _ptr(self.tensors[name]))
        a.work_bytes = work.numel() * work.element_size() if work is not None else 0
        self.args = a
        # what the tensors hold, by _KV4_ROOM
        room = lambda per, *tensors: min((t.numel() // max(per, 1) for t in tensors if t is not None), default=_ANY)       # noqa: E731
        self.room = (room(1, ctx_len, cache_row, status), min(room(int(Hq) * 128, q, out), room(int(Hq), lse)), room(int(Hkv) * 128, k_new, v_new))


class PageTable:
    """lumo_page_table: pages of a cache (any kind), the rows that hold them and the free ones; keeps the tensors alive."""

    def __init__(self, *, page_size: int, table, row_pages, refs, free_list, free_count, work, pools=()):
        """table int32 [rows, max_pages], row_pages int32 [rows], refs and free_list int32 [n_pages], free_count int32 [1], work int32
        [pages_work_ints(rows, n_pages)]; pools: tensors [n_pages, ...] of equal page sizes."""
        self.tensors = dict(table=table, row_pages=row_pages, refs=refs, free_list=free_list, free_count=free_count, work=work)
        self.pools = list(pools)
        _int32(**self.tensors)
        n_rows, max_pages, n_pages = int(table.shape[0]), int(table.shape[1]), int(refs.numel())
        if row_pages.numel() != n_rows or free_list.numel() != n_pages or free_count.numel() != 1 or work.numel() < pages_work_ints(n_rows, n_pages):
            raise ValueError("row_pages, free_list, free_count or work does not fit table and refs")
        sizes = {t.numel() // n_pages * t.element_size() for t in self.pools}
        if any(t.shape[0] != n_pages for t in self.pools) or len(sizes) > 1:
            raise ValueError("pools must be [n_pages, ...] with pages of one size")
        self._ptrs = (ctypes.c_void_p * max(1, len(self.pools)))(*[_ptr(t) for t in self.pools])
        a = _PageTableArgs()
        a.n_rows, a.max_pages, a.n_pages, a.page_size = n_rows, max_pages, n_pages, int(page_size)
        for name, t in self.tensors.items():
            setattr(a, name, _ptr(t))
        a.n_pools, a.pools = len(self.pools), ctypes.addressof(self._ptrs)
        a.page_bytes = sizes.pop() if sizes else 16
        self.args = a


class RowBlocks:
    """Tensors [n_rows, ...] whose rows ``Context.rows_copy`` copies (recurrent states, convolution histories); keeps them alive."""

    def __init__(self, tensors):
        self.tensors = list(tensors)
        self.n_rows = int(self.tensors[0].shape[0])
        if any(t.shape[0] != self.n_rows for t in self.tensors):
            raise ValueError("the blocks must have the same number of rows")
        self.ptrs = (ctypes.c_void_p * len(self.tensors))(*[_ptr(t) for t in self.tensors])
        self.row_bytes = (ctypes.c_int64 * len(self.tensors))(*[t.numel() // self.n_rows * t.element_size() for t in self.tensors])
