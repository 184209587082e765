"""Thin binding over ``libtra_b200.so`` (the C ABI of ``include/tra.h``).

Argument marshalling only: every step of the path runs in the library's CUDA kernels.
PyTorch supplies device memory and streams.  There is no CPU fallback: if the shared
library is missing or cannot be loaded, importing this module raises.
"""
from __future__ import annotations

import ctypes
import math
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# TRA_B200_LIB selects another build of the same library (the bounds-checking debug build)
LIB_PATH = os.environ.get("TRA_B200_LIB") or os.path.join(_HERE, "libtra_b200.so")

TRA_OK = 0
TRA_ERR_INVALID_ARG, TRA_ERR_UNSUPPORTED, TRA_ERR_CAPACITY, TRA_ERR_CUDA, TRA_ERR_TIMEOUT, TRA_ERR_BOUNDS = -1, -2, -3, -4, -5, -6
TRA_KEEP_DIAGONAL = 1
TRA_ORDER_RASTER = 2
TRA_ORDER_RASTER_QO = 4
TRA_RADII_EXTENDED = 0
TRA_RADII_LITERAL = 1
TRA_BUDGET_UNIFORM = 0
TRA_BUDGET_LOGNORMAL = 1
TRA_BF16, TRA_FP16, TRA_FP32 = 0, 1, 2
TRA_NORM_NONE, TRA_NORM_RMS, TRA_NORM_LAYER = 0, 1, 2
TRA_ROTARY_ROTATE, TRA_ROTARY_TILE_MAJOR = 1, 2

EXPORTS = [
    "tra_plan_create", "tra_plan_destroy", "tra_plan_num_tokens", "tra_plan_num_video_tokens", "tra_plan_num_blocks",
    "tra_plan_num_radii", "tra_plan_num_tile_pairs", "tra_plan_tables", "tra_plan_count_table", "tra_plan_status",
    "tra_status_string", "tra_selftest_wait_timeout", "tra_tile_major_gather", "tra_tile_major_scatter",
    "tra_entropy_attn", "tra_budget_radius", "tra_build_block_mask", "tra_sparse_attn",
    "tra_build_block_list_static",
    "tra_hot_path_host_workspace_bytes", "tra_hot_path_host",
    "tra_rotary_create", "tra_rotary_destroy", "tra_rotary_forward", "tra_rotary_backward_workspace_bytes",
    "tra_rotary_backward",
    "tra_packed_create", "tra_packed_destroy", "tra_packed_status", "tra_packed_attn_workspace_bytes",
    "tra_packed_attn", "tra_packed_attn_backward_workspace_bytes", "tra_packed_attn_backward",
]


class tra_config_t(ctypes.Structure):
    _fields_ = [
        ("T", ctypes.c_int), ("H", ctypes.c_int), ("W", ctypes.c_int),
        ("head_dim", ctypes.c_int), ("block", ctypes.c_int),
        ("tile_h", ctypes.c_int), ("tile_w", ctypes.c_int),
        ("tau", ctypes.c_double), ("gamma", ctypes.c_double),
        ("radii", ctypes.POINTER(ctypes.c_double)), ("n_radii", ctypes.c_int),
        ("radius_policy", ctypes.c_int), ("flags", ctypes.c_uint), ("budget_map", ctypes.c_int),
        ("n_text", ctypes.c_int),
    ]


class tra_rotary_config_t(ctypes.Structure):
    _fields_ = [
        ("head_dim", ctypes.c_int), ("n_axes", ctypes.c_int), ("axis", ctypes.POINTER(ctypes.c_int)),
        ("inv_freq", ctypes.POINTER(ctypes.c_double)), ("halves", ctypes.c_int), ("norm", ctypes.c_int),
        ("eps", ctypes.c_double),
    ]


class tra_rotary_tensor_t(ctypes.Structure):
    _fields_ = [
        ("src", ctypes.c_void_p), ("dst", ctypes.c_void_p), ("x", ctypes.c_void_p), ("weight", ctypes.c_void_p),
        ("bias", ctypes.c_void_p), ("weight_grad", ctypes.c_void_p), ("bias_grad", ctypes.c_void_p),
        ("src_stride", ctypes.c_int64 * 3), ("dst_stride", ctypes.c_int64 * 3), ("x_stride", ctypes.c_int64 * 3),
        ("heads", ctypes.c_int), ("flags", ctypes.c_uint),
    ]


class tra_packed_config_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("heads", "kv_heads", "head_dim", "dtype", "causal")]


class tra_packed_args_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("q", "k", "v", "o", "lse")] + \
        [(n, ctypes.c_int64 * 2) for n in ("q_stride", "k_stride", "v_stride", "o_stride")] + \
        [(n, ctypes.c_void_p) for n in ("cu_q", "k_begin", "k_end")] + \
        [(n, ctypes.c_int) for n in ("n_seq", "total_q", "total_k", "max_q", "max_k")] + [("sm_scale", ctypes.c_float)] + \
        [("o_rest", ctypes.c_void_p)]


class tra_packed_grads_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("d_o", "dq", "dk", "dv")] + \
        [(n, ctypes.c_int64 * 2) for n in ("do_stride", "dq_stride", "dk_stride", "dv_stride")]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2608_02504_b200.build` "
            "(there is no CPU fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, f32 = ctypes.c_void_p, ctypes.c_int, ctypes.c_float
    lib.tra_plan_create.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(tra_config_t), vp]
    lib.tra_plan_destroy.argtypes = [vp]
    for name in ("tra_plan_num_tokens", "tra_plan_num_video_tokens", "tra_plan_num_blocks", "tra_plan_num_radii",
                 "tra_plan_num_tile_pairs"):
        getattr(lib, name).argtypes = [vp]
    lib.tra_plan_tables.argtypes = [vp, vp, vp, vp]
    lib.tra_plan_count_table.argtypes = [vp, vp]
    lib.tra_plan_status.argtypes = [vp, vp]
    lib.tra_status_string.argtypes = [i32]
    lib.tra_selftest_wait_timeout.argtypes = [vp, i32, vp]
    lib.tra_hot_path_host_workspace_bytes.argtypes = [vp, i32]
    lib.tra_hot_path_host_workspace_bytes.restype = ctypes.c_size_t
    lib.tra_hot_path_host.argtypes = [vp, vp, vp, vp, vp, vp, ctypes.c_size_t, i32, i32, i32, f32, vp]
    lib.tra_status_string.restype = ctypes.c_char_p
    lib.tra_tile_major_gather.argtypes = [vp, vp, vp, i32, i32, vp]
    lib.tra_tile_major_scatter.argtypes = [vp, vp, vp, i32, i32, vp]
    lib.tra_entropy_attn.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, i32, f32, vp]
    lib.tra_budget_radius.argtypes = [vp, vp, vp, vp, vp, i32, i32, vp]
    lib.tra_build_block_mask.argtypes = [vp, vp, vp, vp, vp, ctypes.c_int64, vp, vp, i32, i32, vp]
    lib.tra_sparse_attn.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, f32, vp]
    lib.tra_build_block_list_static.argtypes = [vp, vp, vp, vp, ctypes.c_int64, vp, vp, i32, i32, vp]
    lib.tra_rotary_create.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(tra_rotary_config_t)]
    lib.tra_rotary_destroy.argtypes = [vp]
    lib.tra_rotary_forward.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, vp]
    lib.tra_rotary_backward_workspace_bytes.argtypes = [vp]
    lib.tra_rotary_backward_workspace_bytes.restype = ctypes.c_size_t
    lib.tra_rotary_backward.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, vp, ctypes.c_size_t, vp]
    lib.tra_packed_create.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(tra_packed_config_t)]
    lib.tra_packed_destroy.argtypes = [vp]
    lib.tra_packed_status.argtypes = [vp, vp]
    lib.tra_packed_attn_workspace_bytes.argtypes = [vp, i32, i32, i32, i32]
    lib.tra_packed_attn_workspace_bytes.restype = ctypes.c_size_t
    lib.tra_packed_attn.argtypes = [vp, vp, vp, ctypes.c_size_t, vp]
    lib.tra_packed_attn_backward_workspace_bytes.argtypes = [vp, i32]
    lib.tra_packed_attn_backward_workspace_bytes.restype = ctypes.c_size_t
    lib.tra_packed_attn_backward.argtypes = [vp, vp, vp, vp, ctypes.c_size_t, vp]
    return lib


_lib = _load()


class TraError(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        super().__init__(f"{where}: {_lib.tra_status_string(code).decode()} ({code})")


def _check(code, where):
    if code != TRA_OK:
        raise TraError(code, where)


def _stream(stream=None):
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def _dev(t, dtype, name):
    if t is None:
        return None
    if not (t.is_cuda and t.is_contiguous() and t.dtype == dtype):
        raise ValueError(f"{name}: expected a contiguous CUDA tensor of dtype {dtype}")
    return ctypes.c_void_p(t.data_ptr())


class Plan:
    """Owns a ``tra_plan_t`` (geometry, thresholds, count table, block boxes)."""

    def __init__(self, T, H, W, head_dim, block, tile_h, tile_w, tau=0.9, gamma=0.6, radii=None,
                 radius_policy=TRA_RADII_EXTENDED, flags=0, budget_map=TRA_BUDGET_UNIFORM, n_text=0,
                 stream=None):
        cfg = tra_config_t()
        cfg.T, cfg.H, cfg.W = T, H, W
        cfg.head_dim, cfg.block, cfg.tile_h, cfg.tile_w = head_dim, block, tile_h, tile_w
        cfg.tau, cfg.gamma = tau, gamma
        self._radii_keepalive = None
        if radii is not None:
            arr = (ctypes.c_double * len(radii))(*[float(r) for r in radii])
            self._radii_keepalive = arr
            cfg.radii = ctypes.cast(arr, ctypes.POINTER(ctypes.c_double))
            cfg.n_radii = len(radii)
        cfg.radius_policy, cfg.flags, cfg.budget_map = radius_policy, flags, budget_map
        cfg.n_text = n_text
        self.cfg = cfg
        self._h = ctypes.c_void_p()
        _check(_lib.tra_plan_create(ctypes.byref(self._h), ctypes.byref(cfg), _stream(stream)), "tra_plan_create")
        self.N = _lib.tra_plan_num_tokens(self._h)              # tokens per sequence (video + text)
        self.N_video = _lib.tra_plan_num_video_tokens(self._h)
        self.NB = _lib.tra_plan_num_blocks(self._h)
        self.n_radii = _lib.tra_plan_num_radii(self._h)
        self.T, self.H, self.W = T, H, W
        self.head_dim, self.block, self.flags = head_dim, block, flags

    @classmethod
    def from_config(cls, cfg: dict, **overrides):
        kw = dict(T=cfg["T"], H=cfg["H"], W=cfg["W"], head_dim=cfg["head_dim"], block=cfg["block"],
                  tile_h=cfg["tile_h"], tile_w=cfg["tile_w"], tau=cfg["tau"], gamma=cfg["gamma"])
        kw.update(overrides)
        return cls(**kw)

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            _lib.tra_plan_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- host copies of the plan tables -------------------------------------------------
    def tables(self):
        import numpy as np
        radii = np.empty(self.n_radii, np.float64)
        theta = np.empty((self.n_radii, self.T), np.int32)
        coord = np.empty((self.N_video, 3), np.int32)
        _check(_lib.tra_plan_tables(self._h, radii.ctypes.data, theta.ctypes.data, coord.ctypes.data),
               "tra_plan_tables")
        return radii, theta, coord

    def count_table(self):
        import numpy as np
        counts = np.empty((self.T, self.H, self.W, self.n_radii), np.uint32)
        _check(_lib.tra_plan_count_table(self._h, counts.ctypes.data), "tra_plan_count_table")
        return counts

    def status(self, stream=None):
        return _lib.tra_plan_status(self._h, _stream(stream))

    def selftest_wait_timeout(self, limit_ms=20):
        """Runs the bounded-wait self-test kernel; the plan status then reads TRA_ERR_TIMEOUT."""
        _check(_lib.tra_selftest_wait_timeout(self._h, limit_ms, _stream()), "tra_selftest_wait_timeout")

    def check_status(self, stream=None):
        _check(self.status(stream), "tra_plan_status")

    # -- layout ---------------------------------------------------------------------------
    def _permute(self, fn, src, name, out=None):
        if not (src.is_cuda and src.is_contiguous()):
            raise ValueError(f"{name}: expected a contiguous CUDA tensor")
        if src.dim() < 2 or src.shape[-2] != self.N:
            raise ValueError(f"{name}: expected [..., N, row]")
        row_bytes = src.shape[-1] * src.element_size()
        n_bh = src.numel() // (self.N * src.shape[-1])
        dst = torch.empty_like(src) if out is None else out
        if not (dst.is_cuda and dst.is_contiguous() and dst.shape == src.shape and dst.dtype == src.dtype):
            raise ValueError(f"{name}: `out` must be a contiguous CUDA tensor like the input")
        _check(fn(self._h, ctypes.c_void_p(src.data_ptr()), ctypes.c_void_p(dst.data_ptr()), n_bh,
                  row_bytes, _stream()), name)
        return dst

    def tile_major_gather(self, x_raster, out=None):
        """raster-order [..., N, row] -> tile-major order (a new tensor, or ``out``)."""
        return self._permute(_lib.tra_tile_major_gather, x_raster, "tra_tile_major_gather", out)

    def tile_major_scatter(self, x_tile_major, out=None):
        """tile-major order [..., N, row] -> raster order (a new tensor, or ``out``)."""
        return self._permute(_lib.tra_tile_major_scatter, x_tile_major, "tra_tile_major_scatter", out)

    # -- the four hot calls -------------------------------------------------------------
    def _bh(self, Q):
        if Q.dim() != 4 or Q.shape[2] != self.N or Q.shape[3] != self.head_dim:
            raise ValueError("expected Q/K/V of shape [B, heads, N, head_dim]")
        return Q.shape[0], Q.shape[1]

    def entropy_attn(self, Q, K, V, O=None, entropy=None, lse=None, want_entropy=True, want_lse=False,
                     sm_scale=None):
        """Dense attention + per-query entropy (tile-major inputs).  Returns (O, entropy, lse)."""
        B, heads = self._bh(Q)
        if O is None:
            O = torch.empty_like(Q)
        if entropy is None and want_entropy:
            entropy = torch.empty(B, heads, self.N, dtype=torch.float32, device=Q.device)
        if lse is None and want_lse:
            lse = torch.empty(B, heads, self.N, dtype=torch.float32, device=Q.device)
        scale = 1.0 / math.sqrt(self.head_dim) if sm_scale is None else sm_scale
        bf = torch.bfloat16
        _check(_lib.tra_entropy_attn(self._h, _dev(Q, bf, "Q"), _dev(K, bf, "K"), _dev(V, bf, "V"),
                                     _dev(O, bf, "O"), _dev(entropy, torch.float32, "entropy"),
                                     _dev(lse, torch.float32, "lse"), B, heads, scale, _stream()),
               "tra_entropy_attn")
        return O, entropy, lse

    def budget_radius(self, entropy, budget=None, radius=None, ridx=None, want_budget=True,
                      want_radius=True):
        """entropy [B, heads, N] fp32 -> (budget int32, radius fp32, ridx as int16 storage of uint16)."""
        B, heads = entropy.shape[0], entropy.shape[1]
        dev = entropy.device
        if budget is None and want_budget:
            budget = torch.empty(B, heads, self.N, dtype=torch.int32, device=dev)
        if radius is None and want_radius:
            radius = torch.empty(B, heads, self.N, dtype=torch.float32, device=dev)
        if ridx is None:
            ridx = torch.empty(B, heads, self.N, dtype=torch.int16, device=dev)
        _check(_lib.tra_budget_radius(self._h, _dev(entropy, torch.float32, "entropy"),
                                      _dev(budget, torch.int32, "budget"),
                                      _dev(radius, torch.float32, "radius"),
                                      _dev(ridx, torch.int16, "ridx"), B, heads, _stream()),
               "tra_budget_radius")
        return budget, radius, ridx

    @property
    def n_tile_pairs(self):
        """Thread blocks per (batch, head) of a block-sparse launch: pairs of query tiles (a tile holds two
        blocks of up to 64 tokens, or one larger block)."""
        return _lib.tra_plan_num_tile_pairs(self._h)

    def build_block_mask(self, ridx, block_mask=None, row_ptr=None, col_idx=None, nnz=None, tile_pairs=None,
                         want_tile_pairs=False):
        """ridx [B, heads, N] -> (block_mask uint8 [B, heads, NB, NB], row_ptr, col_idx, nnz); with
        ``want_tile_pairs`` (or a ``tile_pairs`` buffer) a fifth result: the int32 [B*heads, pairs, 2]
        table of query tiles that share a thread block in ``sparse_attn``."""
        B, heads = ridx.shape[0], ridx.shape[1]
        dev = ridx.device
        rows = B * heads * self.NB
        if block_mask is None:
            block_mask = torch.empty(B, heads, self.NB, self.NB, dtype=torch.uint8, device=dev)
        if row_ptr is None:
            row_ptr = torch.empty(rows + 1, dtype=torch.int32, device=dev)
        if col_idx is None:
            col_idx = torch.empty(rows * self.NB, dtype=torch.int32, device=dev)
        if nnz is None:
            nnz = torch.zeros(1, dtype=torch.int64, device=dev)
        if tile_pairs is None and want_tile_pairs:
            # (blocks of 32 tokens or fewer have no tile pairs: one entry, so that the library's refusal is seen)
            tile_pairs = torch.empty(B * heads, max(self.n_tile_pairs, 1), 2, dtype=torch.int32, device=dev)
        _check(_lib.tra_build_block_mask(self._h, _dev(ridx, torch.int16, "ridx"),
                                         _dev(block_mask, torch.uint8, "block_mask"),
                                         _dev(row_ptr, torch.int32, "row_ptr"),
                                         _dev(col_idx, torch.int32, "col_idx"), col_idx.numel(),
                                         _dev(nnz, torch.int64, "nnz"), _dev(tile_pairs, torch.int32, "tile_pairs"),
                                         B, heads, _stream()),
               "tra_build_block_mask")
        if tile_pairs is not None:
            return block_mask, row_ptr, col_idx, nnz, tile_pairs
        return block_mask, row_ptr, col_idx, nnz

    def build_block_list_static(self, ridx, row_ptr, col_idx, nnz=None, tile_pairs=None):
        """ridx [B, heads, N] -> the active-block list, written into the caller's ``row_ptr`` / ``col_idx``
        (and ``nnz`` / ``tile_pairs`` when given), through ``tra_build_block_list_static``: the variant of
        ``build_block_mask`` for callers that must not allocate.  The Boolean mask stays in a fixed
        16 MiB array inside the library, so every output must be passed in and nothing is created here;
        shapes whose mask is larger raise ``TraError`` (TRA_ERR_CAPACITY)."""
        B, heads = ridx.shape[0], ridx.shape[1]
        _check(_lib.tra_build_block_list_static(self._h, _dev(ridx, torch.int16, "ridx"),
                                                _dev(row_ptr, torch.int32, "row_ptr"),
                                                _dev(col_idx, torch.int32, "col_idx"), col_idx.numel(),
                                                _dev(nnz, torch.int64, "nnz"),
                                                _dev(tile_pairs, torch.int32, "tile_pairs"), B, heads, _stream()),
               "tra_build_block_list_static")

    def sparse_attn(self, Q, K, V, row_ptr, col_idx, O=None, lse=None, want_lse=False, sm_scale=None,
                    ridx=None, tile_pairs=None):
        """Block-sparse attention over the retained key blocks (tile-major inputs).  With ``ridx`` the
        token mask of Eq. 15 is applied inside the retained blocks as well; with ``ridx`` and
        ``row_ptr = col_idx = None`` the call evaluates Eq. 16 itself (token mask alone, no block list)."""
        B, heads = self._bh(Q)
        if O is None:
            O = torch.empty_like(Q)
        if lse is None and want_lse:
            lse = torch.empty(B, heads, self.N, dtype=torch.float32, device=Q.device)
        scale = 1.0 / math.sqrt(self.head_dim) if sm_scale is None else sm_scale
        bf = torch.bfloat16
        _check(_lib.tra_sparse_attn(self._h, _dev(Q, bf, "Q"), _dev(K, bf, "K"), _dev(V, bf, "V"),
                                    _dev(row_ptr, torch.int32, "row_ptr"),
                                    _dev(col_idx, torch.int32, "col_idx"), _dev(ridx, torch.int16, "ridx"),
                                    _dev(tile_pairs, torch.int32, "tile_pairs"), _dev(O, bf, "O"),
                                    _dev(lse, torch.float32, "lse"), B, heads, scale, _stream()),
               "tra_sparse_attn")
        return O, lse


class HostPipeline:
    """One pass of the hot path over tensors that live in pinned host memory (``tra_hot_path_host``).

    The library runs the pass in groups of heads (heads are independent problems): while the kernels
    of group g run, the inputs of group g + 1 travel to the device on a copy stream and the output of
    group g - 1 travels back on another, so the PCIe time hides behind the kernels.  This class only
    owns the device workspace the call needs.

    Inputs and outputs are bf16, raster token order, shape [1, heads, N, head_dim], pinned.
    """

    def __init__(self, plan: "Plan", heads: int, group: int = 8, device=None, sm_scale=None, first_group=None):
        """``first_group`` (default ``group``): heads in the first group; a small first group lets the
        kernels start while most of the input is still on its way."""
        if heads < 1 or group < 1 or (first_group is not None and first_group < 1):
            raise ValueError("heads, group and first_group must be positive")
        self.plan, self.heads, self.group = plan, heads, min(group, heads)
        self.first_group = self.group if first_group is None else min(first_group, self.group)
        self.dev = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
        self.scale = 1.0 / math.sqrt(plan.head_dim) if sm_scale is None else sm_scale
        self.workspace_bytes = int(_lib.tra_hot_path_host_workspace_bytes(plan._h, self.group))
        self.workspace = torch.empty(self.workspace_bytes + 256, dtype=torch.uint8, device=self.dev)
        self._ws_ptr = (self.workspace.data_ptr() + 255) & ~255
        # 3 gathers, dense, budget, vote + scan + fill + pairing, sparse, scatter; a raster-order plan has no
        # gathers and no scatter, one with only Q and O in raster order gathers K and V
        self.launches_per_group = 7 if plan.flags & TRA_ORDER_RASTER else (9 if plan.flags & TRA_ORDER_RASTER_QO else 11)
        self.n_groups = len(self.group_sizes(heads, self.group, self.first_group))

    @staticmethod
    def group_sizes(heads, group, first_group):
        """The head groups of one pass (mirrors the library): a small first group, doubling up to
        ``group``, and a small last group."""
        sizes, left, ramp = [], heads, first_group
        while left > 0:
            n = min(ramp, left)
            if left - n == 0 and n > first_group and sizes:
                n -= first_group
            sizes.append(n)
            left -= n
            ramp = min(2 * ramp, group)
        return sizes

    @staticmethod
    def _check_host(t, shape, name):
        if t.is_cuda or not t.is_pinned() or t.dtype != torch.bfloat16 or tuple(t.shape) != shape or \
                not t.is_contiguous():
            raise ValueError(f"{name}: expected a contiguous pinned bf16 host tensor of shape {shape}")

    def run(self, Qh, Kh, Vh, Oh):
        """Q, K, V (pinned host) -> O (pinned host).  Returns the number of kernels launched once every
        copy and kernel has been enqueued; synchronise the current stream before reading ``Oh``."""
        shape = (1, self.heads, self.plan.N, self.plan.head_dim)
        for t, name in ((Qh, "Q"), (Kh, "K"), (Vh, "V"), (Oh, "O")):
            self._check_host(t, shape, name)
        vp = ctypes.c_void_p
        _check(_lib.tra_hot_path_host(self.plan._h, vp(Qh.data_ptr()), vp(Kh.data_ptr()), vp(Vh.data_ptr()),
                                      vp(Oh.data_ptr()), vp(self._ws_ptr), self.workspace_bytes, self.heads,
                                      self.group, self.first_group, self.scale,
                                      _stream(torch.cuda.current_stream(self.dev))), "tra_hot_path_host")
        return self.n_groups * self.launches_per_group


_DTYPES = {torch.bfloat16: TRA_BF16, torch.float16: TRA_FP16, torch.float32: TRA_FP32}

# The calls below are made for every layer and token, on a few microseconds of kernel: descriptors are packed by one
# struct call each (the layouts of tra_rotary_tensor_t, tra_packed_args_t and tra_packed_grads_t), devices are compared by index.
_ROTARY_TENSOR = struct.Struct("7Q9qiI")
_PACKED_ARGS = struct.Struct("5Q8q3Q5ifQ")
_PACKED_GRADS = struct.Struct("4Q8q")
assert (_ROTARY_TENSOR.size, _PACKED_ARGS.size, _PACKED_GRADS.size) == tuple(
    ctypes.sizeof(t) for t in (tra_rotary_tensor_t, tra_packed_args_t, tra_packed_grads_t))


# (torch.cuda.current_stream builds a Stream object for it: 1.3 us against 0.1)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _empty_like(t):
    return torch.empty_like(t, memory_format=torch.contiguous_format)


class Rotary:
    """Head norm, rotary positions with several axes, and token order: what Q, K and V go through between a
    layer's projections and its attention, in one pass, and its gradients (``tra_rotary_forward`` / ``_backward``).

    ``axis_dims``: channels of each axis, e.g. (44, 42, 42) for (time, height, width) of 128 channels; pair k of
    an axis with c channels turns by ``scale[axis] * theta ** (-2 k / c)`` radians per position.  Any other
    layout of frequencies: pass ``axis`` and ``inv_freq``, one entry per channel pair, instead.
    ``halves``: channels p and p + d/2 form a pair (default: 2p and 2p + 1).
    ``norm``: None, "rms" or "layer", over the channels of each head by itself.  A model that norms over the channels of all heads
    together does that before the split into heads and calls with None.
    """

    def __init__(self, head_dim, axis_dims=None, theta=10000.0, scale=None, axis=None, inv_freq=None, halves=False,
                 norm=None, eps=1e-6):
        if norm not in (None, "rms", "layer"):
            raise ValueError("norm: expected None, 'rms' or 'layer'")
        if (axis_dims is None) == (axis is None or inv_freq is None) or (axis is None) != (inv_freq is None):
            raise ValueError("expected either axis_dims, or axis and inv_freq")
        if axis_dims is not None:
            if any(c < 0 or c % 2 for c in axis_dims) or sum(axis_dims) != head_dim:
                raise ValueError("axis_dims: expected even numbers of channels that add up to head_dim")
            scale = [1.0] * len(axis_dims) if scale is None else list(scale)
            if len(scale) != len(axis_dims):
                raise ValueError("scale: expected one factor per axis")
            axis = [a for a, c in enumerate(axis_dims) for _ in range(c // 2)]
            inv_freq = [scale[a] * theta ** (-2.0 * k / c) for a, c in enumerate(axis_dims) for k in range(c // 2)]
            n_axes = len(axis_dims)
        else:
            if scale is not None:
                raise ValueError("scale: goes with axis_dims")
            axis, inv_freq = [int(a) for a in axis], [float(f) for f in inv_freq]
            if len(axis) != len(inv_freq) or 2 * len(axis) != head_dim:
                raise ValueError("axis, inv_freq: expected head_dim / 2 entries")
            n_axes = max(axis) + 1 if axis else 0
        cfg = tra_rotary_config_t()
        cfg.head_dim, cfg.n_axes, cfg.halves, cfg.eps = head_dim, n_axes, int(halves), eps
        cfg.axis = (ctypes.c_int * len(axis))(*axis)
        cfg.inv_freq = (ctypes.c_double * len(inv_freq))(*inv_freq)
        cfg.norm = {None: TRA_NORM_NONE, "rms": TRA_NORM_RMS, "layer": TRA_NORM_LAYER}[norm]
        self._h = ctypes.c_void_p()
        _check(_lib.tra_rotary_create(ctypes.byref(self._h), ctypes.byref(cfg)), "tra_rotary_create")
        self.head_dim, self.n_axes, self.norm = head_dim, n_axes, norm
        self.workspace_bytes = int(_lib.tra_rotary_backward_workspace_bytes(self._h))

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            _lib.tra_rotary_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- argument marshalling -----------------------------------------------------------------
    @staticmethod
    def _tile_major(plan, name):
        """Which tensors the plan's attention calls take in tile-major order."""
        if plan is None or plan.flags & TRA_ORDER_RASTER:
            return 0
        return TRA_ROTARY_TILE_MAJOR if name != "q" or not plan.flags & TRA_ORDER_RASTER_QO else 0

    def _param(self, t, name, dtype, index):
        if t is None:
            return 0
        if t.dtype != dtype or t.get_device() != index or t.shape != (self.head_dim,) or not t.is_contiguous():
            raise ValueError(f"{name}: expected a contiguous [head_dim] tensor of the tensors' type and device")
        return t.data_ptr()

    @staticmethod
    def _strides(t, name, shape, dtype, index, heads_first=False):
        """Strides (batch, token, head) of a tensor [B, tokens, heads, d] or, heads first, [B, heads, tokens, d]."""
        s = t.stride()
        if t.get_device() != index or t.dtype != dtype or t.shape != shape or s[3] != 1:
            raise ValueError(f"{name}: expected a CUDA tensor of shape {shape}, type {dtype}, on device {index}, "
                             "with contiguous channels")
        return (s[0], s[2], s[1]) if heads_first else s[:3]

    def _begin(self, first, plan, pos, heads_first):
        shape = first.shape
        if len(shape) != 4 or shape[3] != self.head_dim or first.dtype not in _DTYPES or not first.is_cuda:
            raise ValueError("expected CUDA tensors [B, tokens, heads, head_dim] "
                             "([B, heads, tokens, head_dim] on the attention side of a plan), bf16, fp16 or fp32")
        index = first.get_device()
        if index != torch.cuda.current_device():
            raise ValueError("the tensors' device must be the current one")
        B, tokens = shape[0], shape[2 if heads_first else 1]
        if plan is not None and tokens != plan.N:
            raise ValueError(f"expected {plan.N} tokens, the plan's")
        if plan is None and pos is None:
            raise ValueError("expected a plan or pos")
        pos_ptr = None
        if pos is not None:
            if pos.get_device() != index or pos.dtype != torch.int32 or pos.shape != (tokens, self.n_axes) or \
                    not pos.is_contiguous():
                raise ValueError("pos: expected a contiguous int32 CUDA tensor [tokens, n_axes]")
            pos_ptr = pos.data_ptr()
        return B, tokens, index, pos_ptr

    def forward(self, q, k=None, v=None, *, plan=None, pos=None, q_weight=None, k_weight=None, q_bias=None, k_bias=None,
                out=None):
        """Projections q, k, v [B, tokens, heads, d] (any strides with contiguous channels, e.g. slices of a fused
        projection; k and v may be None) -> (q', k', v').

        With ``plan`` the tokens are its raster-order sequence, positions come from its grid (unless ``pos`` is
        given) and the outputs are [B, heads, tokens, d] in the order its attention calls take; without it,
        ``pos`` int32 [tokens, n_axes] names every token's position and outputs keep the inputs' layout.
        V is only moved: without a plan it comes back as a copy.  ``out``: output tensors instead of new ones (new ones of
        one shape are slices of one allocation)."""
        if k is None and (k_weight is not None or k_bias is not None):
            raise ValueError("k_weight, k_bias: given without k")
        B, tokens, index, pos_ptr = self._begin(q, plan, pos, False)
        on_plan, dtype, d = plan is not None, q.dtype, self.head_dim
        desc, outs, n = bytearray(3 * _ROTARY_TENSOR.size), [], 0
        if out is None and on_plan and k is not None and v is not None and k.shape == q.shape and v.shape == q.shape:
            out = q.new_empty((3, B, q.shape[2], tokens, d)).unbind(0)      # one allocation (and 4 us less per call)
        for i, (name, x, w, b) in enumerate((("q", q, q_weight, q_bias), ("k", k, k_weight, k_bias), ("v", v, None, None))):
            if x is None:
                outs.append(None)
                continue
            if x.dim() != 4:
                raise ValueError(f"{name}: expected [B, tokens, heads, head_dim]")
            heads = x.shape[2]
            src = self._strides(x, name, (B, tokens, heads, d), dtype, index)
            shape = (B, heads, tokens, d) if on_plan else (B, tokens, heads, d)
            y = (x.new_empty(shape) if on_plan else _empty_like(x)) if out is None or out[i] is None else out[i]
            dst = self._strides(y, "out " + name, shape, dtype, index, on_plan)
            flags = self._tile_major(plan, name)
            if name != "v":
                flags |= TRA_ROTARY_ROTATE
                w, b = self._param(w, name + "_weight", dtype, index), self._param(b, name + "_bias", dtype, index)
            else:
                w = b = 0
            _ROTARY_TENSOR.pack_into(desc, n * _ROTARY_TENSOR.size, x.data_ptr(), y.data_ptr(), 0, w, b, 0, 0, *src, *dst,
                                     0, 0, 0, heads, flags)
            outs.append(y)
            n += 1
        _check(_lib.tra_rotary_forward(self._h, plan._h if on_plan else None, pos_ptr, bytes(desc), n, B, tokens,
                                       _DTYPES[dtype], _raw_stream(index)), "tra_rotary_forward")
        return tuple(outs)

    def backward(self, dq, dk=None, dv=None, *, q=None, k=None, plan=None, pos=None, q_weight=None, k_weight=None,
                 want_weight_grads=True, out=None):
        """Gradients of ``forward``'s outputs (in their layout) -> ((dq, dk, dv) in the inputs' layout, grads).

        ``q``, ``k``: the forward's inputs, needed (and only taken) with a norm.  ``grads``: fp32 [d] tensors
        "q_weight", "k_weight" (and "q_bias", "k_bias" of a layer norm), summed over all rows, whether or not a
        weight was passed; empty without a norm or with ``want_weight_grads=False``."""
        on_plan, d = plan is not None, self.head_dim
        if k is not None and dk is None:
            raise ValueError("k: given without dk")
        B, tokens, index, pos_ptr = self._begin(dq, plan, pos, on_plan)
        dtype, device = dq.dtype, dq.device
        desc, outs, grads, n = bytearray(3 * _ROTARY_TENSOR.size), [], {}, 0
        for i, (name, dy, x, w) in enumerate((("q", dq, q, q_weight), ("k", dk, k, k_weight), ("v", dv, None, None))):
            if dy is None:
                outs.append(None)
                continue
            if dy.dim() != 4:
                raise ValueError(f"d{name}: expected four dimensions")
            heads = dy.shape[1 if on_plan else 2]
            x_shape = (B, tokens, heads, d)
            src = self._strides(dy, "d" + name, (B, heads, tokens, d) if on_plan else x_shape, dtype, index, on_plan)
            dx = dy.new_empty(x_shape) if out is None or out[i] is None else out[i]
            dst = self._strides(dx, "out d" + name, x_shape, dtype, index)
            flags = self._tile_major(plan, name)
            xp, x_strides, w_grad, b_grad = 0, (0, 0, 0), 0, 0
            if name != "v":
                flags |= TRA_ROTARY_ROTATE
                if (x is not None) != (self.norm is not None):
                    raise ValueError(f"{name}: the forward's input is needed with a norm and only with one")
                if x is not None:
                    xp, x_strides = x.data_ptr(), self._strides(x, name, x_shape, dtype, index)
                    if want_weight_grads:
                        g = grads[name + "_weight"] = torch.empty(d, dtype=torch.float32, device=device)
                        w_grad = g.data_ptr()
                        if self.norm == "layer":
                            g = grads[name + "_bias"] = torch.empty(d, dtype=torch.float32, device=device)
                            b_grad = g.data_ptr()
                w = self._param(w, name + "_weight", dtype, index)
            else:
                w = 0
            _ROTARY_TENSOR.pack_into(desc, n * _ROTARY_TENSOR.size, dy.data_ptr(), dx.data_ptr(), xp, w, 0, w_grad, b_grad,
                                     *src, *dst, *x_strides, heads, flags)
            outs.append(dx)
            n += 1
        ws = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=device) if grads else None
        _check(_lib.tra_rotary_backward(self._h, plan._h if on_plan else None, pos_ptr, bytes(desc), n, B, tokens,
                                        _DTYPES[dtype], ws.data_ptr() if grads else None,
                                        self.workspace_bytes if grads else 0, _raw_stream(index)), "tra_rotary_backward")
        return tuple(outs), grads


class PackedAttn:
    """Attention over packed sequences: prompts and clips of different lengths in one batch, grouped heads, causal
    or not, chunks and single new tokens behind a cache (``tra_packed_attn``), and its gradients.

    Tensors: q, o [total_q, heads, head_dim], k, v [total_k, kv_heads, head_dim], any strides (multiples of 8
    elements) with contiguous channels.  ``cu_q`` int32 [n_seq + 1]: sequence s has the queries cu_q[s] .. cu_q[s+1] - 1.
    """

    def __init__(self, heads, kv_heads, head_dim, dtype=torch.bfloat16, causal=True):
        if dtype not in (torch.bfloat16, torch.float16):
            raise ValueError("dtype: expected bf16 or fp16")
        cfg = tra_packed_config_t(heads, kv_heads, head_dim, _DTYPES[dtype], int(causal))
        self._h = ctypes.c_void_p()
        _check(_lib.tra_packed_create(ctypes.byref(self._h), ctypes.byref(cfg)), "tra_packed_create")
        self.heads, self.kv_heads, self.head_dim, self.dtype, self.causal = heads, kv_heads, head_dim, dtype, bool(causal)
        self._index = torch.cuda.current_device()
        self.device = torch.device("cuda", self._index)

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            _lib.tra_packed_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def status(self, stream=None):
        return _lib.tra_packed_status(self._h, _stream(stream))

    def check_status(self, stream=None):
        _check(self.status(stream), "tra_packed_status")

    def _tensor(self, t, name, total, heads):
        s = t.stride()
        if t.get_device() != self._index or t.dtype != self.dtype or t.shape != (total, heads, self.head_dim) or s[2] != 1:
            raise ValueError(f"{name}: expected {self.dtype} [{total}, {heads}, {self.head_dim}] on {self.device} with "
                             "contiguous channels")
        return t.data_ptr(), s[0], s[1]

    def _ints(self, t, name, n):
        if t.get_device() != self._index or t.dtype != torch.int32 or t.shape != (n,) or not t.is_contiguous():
            raise ValueError(f"{name}: expected a contiguous int32 tensor of {n} entries on {self.device}")
        return t.data_ptr()

    def _args(self, q, k, v, o, lse, rest, cu_q, cu_k, k_range, max_q, max_k, sm_scale):
        if q.dim() != 3 or k.dim() != 3 or cu_q.dim() != 1 or cu_q.shape[0] < 2:
            raise ValueError("expected q, k, v [tokens, heads, head_dim] and cu_q [n_seq + 1]")
        if torch.cuda.current_device() != self._index:
            raise ValueError(f"the current device must be {self.device}")
        tq, tk, n = q.shape[0], k.shape[0], cu_q.shape[0] - 1
        qp, q0, q1 = self._tensor(q, "q", tq, self.heads)
        kp, k0, k1 = self._tensor(k, "k", tk, self.kv_heads)
        vp, v0, v1 = self._tensor(v, "v", tk, self.kv_heads)
        op, o0, o1 = self._tensor(o, "o", tq, self.heads)
        lp = 0
        if lse is not None:
            if lse.get_device() != self._index or lse.dtype != torch.float32 or lse.shape != (tq, self.heads) or \
                    not lse.is_contiguous():
                raise ValueError("lse: expected a contiguous fp32 tensor [total_q, heads]")
            lp = lse.data_ptr()
        cq = self._ints(cu_q, "cu_q", n + 1)
        if k_range is not None:
            if cu_k is not None:
                raise ValueError("expected cu_k or k_range, not both")
            begin, end = self._ints(k_range[0], "k_range", n), self._ints(k_range[1], "k_range", n)
        else:
            begin = cq if cu_k is None else self._ints(cu_k, "cu_k", n + 1)
            end = begin + 4
        return _PACKED_ARGS.pack(qp, kp, vp, op, lp, q0, q1, k0, k1, v0, v1, o0, o1, cq, begin, end, n, tq, tk, max_q, max_k,
                                 self.head_dim ** -0.5 if sm_scale is None else sm_scale, 0 if rest is None else rest.data_ptr())

    @staticmethod
    def _writes(lse, rest):
        """How often torch has written into lse more than into its remainder (the kernels' own writes are not counted): the
        same as when a call made them as long as both are as they were, or were written or copied together."""
        return None if rest is None or lse.is_inference() or rest.is_inference() else lse._version - rest._version

    @staticmethod
    def _rest_fits(rest, q):
        return isinstance(rest, torch.Tensor) and rest.shape == q.shape and rest.dtype == q.dtype and rest.device == q.device and rest.is_contiguous()

    def forward(self, q, k, v, cu_q, cu_k=None, *, k_range=None, max_q, max_k, o=None, lse=None, want_lse=False,
                sm_scale=None, o_rest=None):
        """-> (o, lse).  Keys: packed like the queries (``cu_k``, default ``cu_q``), or ``k_range`` = (begin, end), two
        int32 [n_seq] tensors, e.g. the filled parts of a cache's slots.  ``max_q``, ``max_k``: upper bounds of the
        sequences' queries and keys, at most the tensors' tokens (a longer sequence is cut and reported by ``check_status``).  Rows of o and lse that
        belong to no sequence are not written.

        ``o_rest``: what rounding took from o, for ``backward``: a contiguous tensor like q to write it to, or False for
        none.  By default an lse made here (``want_lse``) gets one, and one that an lse passed in carries is written again.
        The one that was written is also kept as ``lse.o_rest``; a copy or a slice of lse does not carry it along."""
        if o is None:
            o = _empty_like(q)
        if o_rest is None:
            if lse is not None:
                o_rest = getattr(lse, "o_rest", None)
                if o_rest is not None and not self._rest_fits(o_rest, q):
                    o_rest = None                        # of a call on other tensors
            elif want_lse:
                o_rest = _empty_like(q)
        elif o_rest is False:
            o_rest = None
        elif not self._rest_fits(o_rest, q) or (lse is None and not want_lse):
            raise ValueError("o_rest: expected a contiguous tensor like q, beside an lse")
        if lse is None and want_lse:
            lse = q.new_empty((q.shape[0], self.heads), dtype=torch.float32)
        a = self._args(q, k, v, o, lse, o_rest, cu_q, cu_k, k_range, max_q, max_k, sm_scale)
        n = _lib.tra_packed_attn_workspace_bytes(self._h, cu_q.shape[0] - 1, q.shape[0], max_q, max_k)
        ws = q.new_empty((n,), dtype=torch.uint8) if n else None
        _check(_lib.tra_packed_attn(self._h, a, ws.data_ptr() if n else None, n, _raw_stream(self._index)), "tra_packed_attn")
        if lse is not None:
            lse.o_rest, lse.o_rest_writes = o_rest, self._writes(lse, o_rest)
        return o, lse

    def backward(self, do, q, k, v, o, lse, cu_q, cu_k=None, *, max_q, max_k, dq=None, dk=None, dv=None, sm_scale=None,
                 o_rest=None):
        """Gradients (dq, dk, dv) of ``forward`` over packed keys, from its o and lse.  Rows that belong to no sequence
        are not written.

        ``o_rest``: what rounding took from o, as ``forward`` wrote it; without it the gradients of rows that see few keys,
        or one above all, are mostly the rounding of o.  Default: the one kept beside the lse, if it carries one, and an error when
        torch has written into one of the two since and not into the other; False: none."""
        dq = _empty_like(q) if dq is None else dq
        dk = _empty_like(k) if dk is None else dk
        dv = _empty_like(v) if dv is None else dv
        if lse is None:
            raise ValueError("lse: the forward call's, made with want_lse")
        if o_rest is None:
            o_rest = getattr(lse, "o_rest", None)
            if o_rest is not None:
                writes = self._writes(lse, o_rest)
                if getattr(lse, "o_rest_writes", writes) != writes:
                    raise ValueError("lse.o_rest: the lse was written since; pass o_rest (False: none)")
        elif o_rest is False:
            o_rest = None
        if o_rest is not None and not self._rest_fits(o_rest, q):
            raise ValueError("o_rest: expected a contiguous tensor like q")
        a = self._args(q, k, v, o, lse, o_rest, cu_q, cu_k, None, max_q, max_k, sm_scale)
        tq, tk = q.shape[0], k.shape[0]
        ptrs, strides = zip(*((p, s) for p, *s in (self._tensor(do, "do", tq, self.heads), self._tensor(dq, "dq", tq, self.heads),
                                                   self._tensor(dk, "dk", tk, self.kv_heads), self._tensor(dv, "dv", tk, self.kv_heads))))
        g = _PACKED_GRADS.pack(*ptrs, *(x for s in strides for x in s))
        n = _lib.tra_packed_attn_backward_workspace_bytes(self._h, tq)
        ws = q.new_empty((n,), dtype=torch.uint8) if n else None
        _check(_lib.tra_packed_attn_backward(self._h, a, g, ws.data_ptr() if n else None, n, _raw_stream(self._index)),
               "tra_packed_attn_backward")
        return dq, dk, dv
