"""Thin Python binding of libswam.so (argument marshalling only).

Every step of the path runs in the library's CUDA kernels; torch is used here
for device memory and streams.  There is no CPU fallback: if the shared
library is missing or cannot be loaded, importing a symbol raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Tuple

import torch

from . import workloads as W

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libswam.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_STATE, ERR_CUDA, ERR_DEVICE_CHECK, ERR_TIMEOUT = range(8)
F32, BF16 = 0, 1
REUSE, REFRESH_FULL, REFRESH_LIGHT = 0, 1, 2
OPT_ATTN_VARIANT, OPT_SPARSE_PATH, OPT_VISIBILITY, OPT_HOST_ROWS = 1, 2, 3, 4
HOST_ROWS_RETAINED, HOST_ROWS_ALL = 0, 1
SEES_OBSERVED, SEES_FUTURE, SEES_ALL = 0, 1, 2
ATTN_AUTO, ATTN_WARP_MMA = 0, 1
SPARSE_FUSED, SPARSE_STAGED, SPARSE_FUSED_KV = 0, 1, 2

EXPORTS = [
    "swam_create", "swam_destroy", "swam_workspace_bytes", "swam_bind_workspace", "swam_score", "swam_score_noalloc",
    "swam_select", "swam_aggregate", "swam_select_maps",
    "swam_pack", "swam_sparse_attn", "swam_scatter", "swam_cross_attn", "swam_cross_attn_scratch_bytes",
    "swam_prefix_attn", "swam_prefix_attn_scratch_bytes", "swam_step", "swam_host_io_bytes", "swam_bind_host_io",
    "swam_step_host", "swam_host_join", "swam_get_selection", "swam_get_scores", "swam_set_selection", "swam_state_bytes",
    "swam_state_export", "swam_state_import", "swam_check", "swam_selftest_timeout", "swam_launch_floor", "swam_set_option", "swam_launch_count",
    "swam_last_error", "swam_version",
]


class SwamShape(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("n_obs", ctypes.c_int32), ("n_frames", ctypes.c_int32),
        ("n_spatial", ctypes.c_int32), ("n_action", ctypes.c_int32), ("n_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("k_core", ctypes.c_int32), ("k_anchor", ctypes.c_int32),
        ("dtype", ctypes.c_int32), ("softmax_scale", ctypes.c_float), ("cv_beta", ctypes.c_float),
        ("query_weights", ctypes.POINTER(ctypes.c_float)), ("n_kv_heads", ctypes.c_int32),
    ]


class SwamCrossArgs(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in ("q", "k", "v", "kv_len", "out", "lse", "scratch")]
                + [("scratch_bytes", ctypes.c_size_t)]
                + [(n, ctypes.c_int32) for n in ("n_q", "n_kv", "n_kv_heads", "reserved")]
                + [(n, ctypes.c_int64) for n in ("q_token", "q_sample", "k_token", "k_sample", "v_token", "v_sample",
                                                 "out_token", "out_sample")])


class SwamPrefixArgs(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in ("q", "k_prefix", "v_prefix", "k", "v", "prefix_len", "own_len", "out", "lse",
                                                "scratch")]
                + [("scratch_bytes", ctypes.c_size_t)]
                + [(n, ctypes.c_int32) for n in ("n_q", "n_prefix", "n_own", "n_groups", "causal", "n_kv_heads")]
                + [(n, ctypes.c_int64) for n in ("q_token", "q_sample", "k_prefix_token", "k_prefix_group", "v_prefix_token",
                                                 "v_prefix_group", "k_token", "k_sample", "v_token", "v_sample",
                                                 "out_token", "out_sample")])


class SwamError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"swam error {code}: {msg}")
        self.code = code


_lib = None


def load_library() -> ctypes.CDLL:
    """Load libswam.so; raises if it has not been built (python -m paper_2609_38984_b200.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2609_38984_b200.build`; "
                               "there is no CPU fallback")
        lib = ctypes.CDLL(LIB_PATH)
        vp, i32 = ctypes.c_void_p, ctypes.c_int32
        lib.swam_create.argtypes = [ctypes.POINTER(SwamShape), ctypes.POINTER(vp)]
        lib.swam_destroy.argtypes = [vp]
        lib.swam_workspace_bytes.argtypes = [vp, ctypes.POINTER(ctypes.c_size_t)]
        lib.swam_bind_workspace.argtypes = [vp, vp, ctypes.c_size_t]
        lib.swam_host_io_bytes.argtypes = [vp, ctypes.POINTER(ctypes.c_size_t)]
        lib.swam_bind_host_io.argtypes = [vp, vp, ctypes.c_size_t]
        lib.swam_score.argtypes = [vp, vp, vp, vp, vp, vp, vp]
        lib.swam_score_noalloc.argtypes = [vp, vp, vp, vp, vp]
        lib.swam_select.argtypes = [vp, vp, vp, vp, vp, vp]
        lib.swam_aggregate.argtypes = [vp, vp, vp, i32, i32, vp, vp, vp, vp]
        lib.swam_select_maps.argtypes = [vp, vp, vp, vp, vp, vp, vp]
        lib.swam_pack.argtypes = [vp] * 9
        lib.swam_sparse_attn.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp]
        lib.swam_scatter.argtypes = [vp] * 7
        for name, args in (("cross", SwamCrossArgs), ("prefix", SwamPrefixArgs)):
            getattr(lib, f"swam_{name}_attn").argtypes = [vp, ctypes.POINTER(args), vp]
            getattr(lib, f"swam_{name}_attn_scratch_bytes").argtypes = [vp, ctypes.POINTER(args), ctypes.POINTER(ctypes.c_size_t)]
        lib.swam_step.argtypes = [vp, vp, vp, vp, i32, vp, vp]
        lib.swam_step_host.argtypes = [vp, vp, vp, vp, i32, vp, vp]
        lib.swam_host_join.argtypes = [vp, vp]
        lib.swam_get_selection.argtypes = [vp, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp)]
        lib.swam_get_scores.argtypes = [vp, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp)]
        lib.swam_set_selection.argtypes = [vp, vp, vp, vp, vp]
        lib.swam_state_bytes.argtypes = [vp, ctypes.POINTER(ctypes.c_size_t)]
        lib.swam_state_export.argtypes = [vp, vp, vp]
        lib.swam_state_import.argtypes = [vp, vp, vp]
        lib.swam_check.argtypes = [vp, vp]
        lib.swam_selftest_timeout.argtypes = [vp, ctypes.c_uint64, vp]
        lib.swam_launch_floor.argtypes = [vp, vp]
        lib.swam_set_option.argtypes = [vp, i32, i32]
        lib.swam_launch_count.argtypes = [vp, ctypes.POINTER(ctypes.c_int64)]
        lib.swam_last_error.argtypes = [vp]
        lib.swam_last_error.restype = ctypes.c_char_p
        lib.swam_version.restype = ctypes.c_char_p
        _lib = lib
    return _lib


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    assert t.is_contiguous(), "tensors must be contiguous"
    return ctypes.c_void_p(t.data_ptr())


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _raw_stream() -> int:
    # the handle without the Stream object around it, which costs several microseconds a call
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def torch_dtype(dtype: int) -> torch.dtype:
    return torch.float32 if dtype == F32 else torch.bfloat16


class Swam:
    """One context = one shape.  Methods mirror the C entry points and take CUDA tensors laid out
    [B, L, N_h, D] (or [B, L', N_h, D] for packed tensors); K and V have n_kv_heads heads instead of N_h."""

    def __init__(self, batch, n_obs, n_frames, n_spatial, n_action, n_heads, head_dim, k_core, k_anchor,
                 dtype=BF16, softmax_scale: float = 0.0, cv_beta: float = 1.0, query_weights=None,
                 device: Optional[torch.device] = None, bind: bool = True, n_kv_heads: int = 0):
        self.lib = load_library()
        self._weights = None
        if query_weights is not None:
            self._weights = (ctypes.c_float * len(query_weights))(*[float(x) for x in query_weights])
        self.shape = SwamShape(batch, n_obs, n_frames, n_spatial, n_action, n_heads, head_dim, k_core, k_anchor,
                               dtype, softmax_scale, cv_beta,
                               ctypes.cast(self._weights, ctypes.POINTER(ctypes.c_float)) if self._weights else None,
                               n_kv_heads)
        self.ctx = ctypes.c_void_p()
        if device is None:
            if not torch.cuda.is_available():
                raise RuntimeError("swam needs a CUDA device; there is no CPU fallback")
            device = torch.device("cuda", torch.cuda.current_device())
        self.device = device
        rc = self.lib.swam_create(ctypes.byref(self.shape), ctypes.byref(self.ctx))
        if rc != OK:
            self.ctx = ctypes.c_void_p()
            raise SwamError(rc, "swam_create rejected the shape")
        self.B, self.F, self.N_s, self.H = batch, n_frames, n_spatial, n_action
        self.n_obs, self.N_h, self.D = n_obs, n_heads, head_dim
        self.N_kv = n_kv_heads if n_kv_heads > 0 else n_heads
        self.K = k_core + k_anchor
        self.L = n_obs + n_frames * n_spatial + n_action
        self.Lp = n_obs + n_frames * self.K + n_action
        self.dtype = dtype
        self._torch_dtype = torch_dtype(dtype)
        self._device_index = device.index if device.index is not None else torch.cuda.current_device()
        self._scratch_need = {}
        self._lse_like = {}
        self.workspace = None
        self.staging = None
        if bind:
            self.bind_workspace()

    @classmethod
    def from_workload(cls, wl: W.Workload, **kw) -> "Swam":
        kc, ks = wl.budgets
        return cls(wl.batch, wl.n_obs, wl.n_frames, wl.n_spatial, wl.n_action, wl.n_heads, wl.head_dim, kc, ks,
                   dtype=wl.dtype, n_kv_heads=wl.kv_heads, **kw)

    def __del__(self):
        try:
            if getattr(self, "ctx", None) and self.ctx.value:
                self.lib.swam_destroy(self.ctx)
                self.ctx = ctypes.c_void_p()
        except Exception:
            pass

    # -- helpers -----------------------------------------------------------
    def _chk(self, rc: int):
        if rc != OK:
            raise SwamError(rc, self.lib.swam_last_error(self.ctx).decode())

    def workspace_bytes(self) -> int:
        n = ctypes.c_size_t()
        self._chk(self.lib.swam_workspace_bytes(self.ctx, ctypes.byref(n)))
        return n.value

    def bind_workspace(self):
        self.workspace = torch.empty(self.workspace_bytes() + 256, dtype=torch.uint8, device=self.device)
        off = (-self.workspace.data_ptr()) % 256
        self._chk(self.lib.swam_bind_workspace(self.ctx, ctypes.c_void_p(self.workspace.data_ptr() + off),
                                               self.workspace.numel() - off))

    def host_io_bytes(self) -> int:
        n = ctypes.c_size_t()
        self._chk(self.lib.swam_host_io_bytes(self.ctx, ctypes.byref(n)))
        return n.value

    def bind_host_io(self):
        self.staging = torch.empty(self.host_io_bytes() + 256, dtype=torch.uint8, device=self.device)
        off = (-self.staging.data_ptr()) % 256
        self._chk(self.lib.swam_bind_host_io(self.ctx, ctypes.c_void_p(self.staging.data_ptr() + off),
                                             self.staging.numel() - off))

    def empty_full(self) -> torch.Tensor:
        return torch.empty((self.B, self.L, self.N_h, self.D), dtype=torch_dtype(self.dtype), device=self.device)

    def empty_packed(self, kv: bool = False) -> torch.Tensor:
        return torch.empty((self.B, self.Lp, self.N_kv if kv else self.N_h, self.D), dtype=torch_dtype(self.dtype),
                           device=self.device)

    # -- the calls ---------------------------------------------------------
    def score(self, q, k, lse_action=None, quality: bool = False):
        scores = torch.empty((self.B, self.F, self.N_s), dtype=torch.float32, device=self.device)
        qual = torch.empty((self.B, 3), dtype=torch.float32, device=self.device) if quality else None
        self._chk(self.lib.swam_score(self.ctx, _ptr(q), _ptr(k), _ptr(lse_action), _ptr(scores), _ptr(qual), _stream()))
        return (scores, qual) if quality else scores

    def score_noalloc(self, q, k, scores):
        """Scores into the caller's `scores` tensor using the library's built-in scratch: no workspace, nothing
        allocated (for callers that cannot obtain device memory at call time)."""
        self._chk(self.lib.swam_score_noalloc(self.ctx, _ptr(q), _ptr(k), _ptr(scores), _stream()))
        return scores

    def select(self, scores) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
        sel = torch.empty((self.B, self.F, self.K), dtype=torch.int32, device=self.device)
        pack = torch.empty((self.B, self.Lp), dtype=torch.int32, device=self.device)
        inv = torch.empty((self.B, self.L), dtype=torch.int32, device=self.device)
        self._chk(self.lib.swam_select(self.ctx, _ptr(scores), _ptr(sel), _ptr(pack), _ptr(inv), _stream()))
        return sel, pack, inv

    def aggregate(self, layer_scores, layer_quality, k_layer: int):
        """V, V_all and the chosen core layers from per-layer scores [n_layers, B, F, N_s] and qualities [n_layers, B, 3]."""
        n_layers = layer_scores.shape[0]
        v_core = torch.empty((self.B, self.F, self.N_s), dtype=torch.float32, device=self.device)
        v_all = torch.empty_like(v_core)
        layers = torch.empty((self.B, k_layer), dtype=torch.int32, device=self.device)
        self._chk(self.lib.swam_aggregate(self.ctx, _ptr(layer_scores), _ptr(layer_quality), n_layers, k_layer,
                                          _ptr(v_core), _ptr(v_all), _ptr(layers), _stream()))
        return v_core, v_all, layers

    def select_maps(self, core_scores, anchor_scores):
        sel = torch.empty((self.B, self.F, self.K), dtype=torch.int32, device=self.device)
        pack = torch.empty((self.B, self.Lp), dtype=torch.int32, device=self.device)
        inv = torch.empty((self.B, self.L), dtype=torch.int32, device=self.device)
        self._chk(self.lib.swam_select_maps(self.ctx, _ptr(core_scores), _ptr(anchor_scores), _ptr(sel), _ptr(pack),
                                            _ptr(inv), _stream()))
        return sel, pack, inv

    def pack(self, q, k, v, pack_map):
        outs = [self.empty_packed(kv=i > 0) if x is not None else None for i, x in enumerate((q, k, v))]
        self._chk(self.lib.swam_pack(self.ctx, _ptr(q), _ptr(k), _ptr(v), _ptr(pack_map), _ptr(outs[0]),
                                     _ptr(outs[1]), _ptr(outs[2]), _stream()))
        return outs

    def sparse_attn(self, qp, kp, vp, want_lse: bool = False):
        n = qp.shape[1]
        out = torch.empty_like(qp)
        lse = torch.empty((self.B, self.N_h, n), dtype=torch.float32, device=self.device) if want_lse else None
        self._chk(self.lib.swam_sparse_attn(self.ctx, _ptr(qp), _ptr(kp), _ptr(vp), n, _ptr(out), _ptr(lse), _stream()))
        return (out, lse) if want_lse else out

    def _tokens(self, name: str, t: torch.Tensor, lead: Optional[int], heads: int):
        """Token and sample strides of a [samples, tokens, heads, D] tensor whose heads are contiguous (0, 0: contiguous)."""
        if t.dtype is not self._torch_dtype or t.get_device() != self._device_index or t.dim() != 4:
            raise ValueError(f"{name}: expected a 4-dimensional {self._torch_dtype} tensor on {self.device}")
        n, tokens, h, d = t.shape
        if (lead is not None and n != lead) or h != heads or h == 0 or d != self.D:
            raise ValueError(f"{name}: expected shape [{'groups' if lead is None else lead}, tokens, {heads}, {self.D}], got {list(t.shape)}")
        if n == 0 or tokens == 0 or t.is_contiguous():
            return 0, 0
        s0, s1, s2, s3 = t.stride()
        if s3 != 1 or (h > 1 and s2 != d):
            raise ValueError(f"{name}: the heads of a token must be contiguous")
        if (tokens > 1 and s1 == 0) or (n > 1 and s0 == 0):
            raise ValueError(f"{name}: expanded (stride 0) tokens or samples are not accepted")
        tok = s1 if tokens > 1 else h * d
        return tok, (s0 if n > 1 else tokens * tok)

    def _lengths(self, name: str, t: Optional[torch.Tensor], n: int):
        if t is None:
            return None
        if t.dtype is not torch.int32 or t.get_device() != self._device_index or t.shape != (n,) or not t.is_contiguous():
            raise ValueError(f"{name}: expected a contiguous int32 tensor of shape [{n}] on {self.device}")
        return t.data_ptr()

    def _out_lse(self, q, out, want_lse: bool):
        # (empty_like costs half of what empty does on the host; the pattern is one element expanded to the shape)
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
        elif out.shape != q.shape:
            raise ValueError(f"out: expected shape {list(q.shape)}")
        if not want_lse:
            return out, None
        n_q = q.shape[1]
        like = self._lse_like.get(n_q)
        if like is None:
            like = torch.empty(1, dtype=torch.float32, device=self.device).expand(self.B, self.N_h, n_q)
            if len(self._lse_like) < 64:
                self._lse_like[n_q] = like
        return out, torch.empty_like(like, memory_format=torch.contiguous_format)

    def _scratch(self, query, a, key):
        """Scratch of a call: the tensor that holds it (it stays alive until the call has been enqueued) and its aligned
        address.  The size depends on the sizes of the call alone (and the attention variant), so it is asked for once."""
        need = self._scratch_need.get(key)
        if need is None:
            n = ctypes.c_size_t()
            self._chk(query(self.ctx, ctypes.byref(a), ctypes.byref(n)))
            if len(self._scratch_need) >= 64:       # a decoding loop brings another length with every call
                self._scratch_need.clear()
            need = self._scratch_need[key] = n.value
        if need == 0:
            return None
        buf = torch.empty(need + 256, dtype=torch.uint8, device=self.device)
        a.scratch, a.scratch_bytes = (buf.data_ptr() + 255) & ~255, need
        return buf

    def cross_attn(self, q, k, v, kv_len=None, out=None, want_lse: bool = False):
        """Queries [B, n_q, N_h, D] attend an encoder's states k, v [B, n_kv, heads, D] (any divisor of N_h heads), of which
        the first kv_len[b] (int32 CUDA tensor [B], default all) are real.  Tensors may be strided views with
        contiguous heads.  A row without keys gives zeros (lse -inf).  Returns out, or (out, lse [B, N_h, n_q])."""
        heads = k.shape[2] if k.dim() == 4 else 0
        if v.shape != k.shape:
            raise ValueError("k and v differ in shape")
        k_tok, k_smp = self._tokens("k", k, self.B, heads)
        v_tok, v_smp = self._tokens("v", v, self.B, heads)
        q_tok, q_smp = self._tokens("q", q, self.B, self.N_h)
        out, lse = self._out_lse(q, out, want_lse)
        o_tok, o_smp = self._tokens("out", out, self.B, self.N_h)
        n_q, n_kv = q.shape[1], k.shape[1]
        a = SwamCrossArgs(q.data_ptr(), k.data_ptr(), v.data_ptr(), self._lengths("kv_len", kv_len, self.B), out.data_ptr(),
                          lse.data_ptr() if want_lse else None, None, 0, n_q, n_kv, heads, 0, q_tok, q_smp, k_tok, k_smp,
                          v_tok, v_smp, o_tok, o_smp)
        scratch = self._scratch(self.lib.swam_cross_attn_scratch_bytes, a, (n_q, n_kv, heads))  # noqa: F841
        rc = self.lib.swam_cross_attn(self.ctx, ctypes.byref(a), _raw_stream())
        if rc != OK:
            self._chk(rc)
        return (out, lse) if want_lse else out

    def prefix_attn(self, q, k_prefix, v_prefix, k, v, prefix_len=None, own_len=None, causal: bool = False, out=None,
                    want_lse: bool = False):
        """Queries [B, n_q, N_h, D] attend a prefix k_prefix, v_prefix [groups, n_prefix, heads, D] that the B / groups
        consecutive samples of a group share, followed by their own k, v [B, n_own, heads, D].  prefix_len [groups] and
        own_len [B] (int32 CUDA tensors, default all) give the real lengths; `causal`: query t sees the own keys up to
        own_len[b] - n_q + t.  A row without keys gives zeros (lse -inf).  Returns out, or (out, lse [B, N_h, n_q])."""
        heads = k.shape[2] if k.dim() == 4 else 0
        if v.shape != k.shape or v_prefix.shape != k_prefix.shape:
            raise ValueError("k and v differ in shape")
        kp_tok, kp_grp = self._tokens("k_prefix", k_prefix, None, heads)
        vp_tok, vp_grp = self._tokens("v_prefix", v_prefix, None, heads)
        k_tok, k_smp = self._tokens("k", k, self.B, heads)
        v_tok, v_smp = self._tokens("v", v, self.B, heads)
        q_tok, q_smp = self._tokens("q", q, self.B, self.N_h)
        out, lse = self._out_lse(q, out, want_lse)
        o_tok, o_smp = self._tokens("out", out, self.B, self.N_h)
        n_q, n_prefix, n_own, groups = q.shape[1], k_prefix.shape[1], k.shape[1], k_prefix.shape[0]
        a = SwamPrefixArgs(q.data_ptr(), k_prefix.data_ptr(), v_prefix.data_ptr(), k.data_ptr(), v.data_ptr(),
                           self._lengths("prefix_len", prefix_len, groups), self._lengths("own_len", own_len, self.B),
                           out.data_ptr(), lse.data_ptr() if want_lse else None, None, 0, n_q, n_prefix, n_own, groups,
                           1 if causal else 0, heads, q_tok, q_smp, kp_tok, kp_grp, vp_tok, vp_grp, k_tok, k_smp, v_tok, v_smp,
                           o_tok, o_smp)
        key = (n_q, n_prefix, n_own, groups, heads, a.causal)
        scratch = self._scratch(self.lib.swam_prefix_attn_scratch_bytes, a, key)  # noqa: F841
        rc = self.lib.swam_prefix_attn(self.ctx, ctypes.byref(a), _raw_stream())
        if rc != OK:
            self._chk(rc)
        return (out, lse) if want_lse else out

    def scatter(self, out_p, pack_map, inv_map, cached, out=None):
        out = cached if out is None else out
        self._chk(self.lib.swam_scatter(self.ctx, _ptr(out_p), _ptr(pack_map), _ptr(inv_map), _ptr(cached), _ptr(out),
                                        _stream()))
        return out

    def step(self, q, k, v, mode: int, out):
        self._chk(self.lib.swam_step(self.ctx, _ptr(q), _ptr(k), _ptr(v), mode, _ptr(out), _stream()))
        return out

    def step_host(self, q_host, k_host, v_host, mode: int, out_host):
        """Host (pinned) tensors in and out; copies and kernels are enqueued on the current stream."""
        if self.staging is None:
            self.bind_host_io()
        self._chk(self.lib.swam_step_host(self.ctx, _ptr(q_host), _ptr(k_host), _ptr(v_host), mode, _ptr(out_host),
                                          _stream()))
        return out_host

    def host_join(self):
        """The current stream waits for the last step_host result to arrive in its host buffer."""
        self._chk(self.lib.swam_host_join(self.ctx, _stream()))

    def _view(self, ptr: ctypes.c_void_p, shape, dtype) -> torch.Tensor:
        off = ptr.value - self.workspace.data_ptr()
        n = 1
        for s in shape:
            n *= s
        nbytes = n * torch.empty((), dtype=dtype).element_size()
        return self.workspace[off:off + nbytes].view(dtype).view(*shape)

    def selection(self):
        """Views of the cached sel_idx, pack_map, inv_map inside the workspace."""
        a, b, c = ctypes.c_void_p(), ctypes.c_void_p(), ctypes.c_void_p()
        self._chk(self.lib.swam_get_selection(self.ctx, ctypes.byref(a), ctypes.byref(b), ctypes.byref(c)))
        return (self._view(a, (self.B, self.F, self.K), torch.int32), self._view(b, (self.B, self.Lp), torch.int32),
                self._view(c, (self.B, self.L), torch.int32))

    def set_selection(self, sel_idx: torch.Tensor, pack_map: torch.Tensor, inv_map: torch.Tensor):
        """Install a selection made elsewhere (another context's, or swam_select on other scores) for REUSE steps."""
        for t, shape in ((sel_idx, (self.B, self.F, self.K)), (pack_map, (self.B, self.Lp)), (inv_map, (self.B, self.L))):
            if t.dtype != torch.int32 or tuple(t.shape) != shape or not t.is_contiguous() or not t.is_cuda:
                raise ValueError(f"expected a contiguous int32 CUDA tensor of shape {shape}")
        self._chk(self.lib.swam_set_selection(self.ctx, _ptr(sel_idx), _ptr(pack_map), _ptr(inv_map), _stream()))

    def export_state(self) -> torch.Tensor:
        """The cross-step state (scores, diagnostics, normalisers, selection, maps) as one opaque byte tensor."""
        n = ctypes.c_size_t()
        self._chk(self.lib.swam_state_bytes(self.ctx, ctypes.byref(n)))
        buf = torch.empty(n.value, dtype=torch.uint8, device=self.device)
        self._chk(self.lib.swam_state_export(self.ctx, _ptr(buf), _stream()))
        return buf

    def import_state(self, buf: torch.Tensor):
        n = ctypes.c_size_t()
        self._chk(self.lib.swam_state_bytes(self.ctx, ctypes.byref(n)))
        if buf.dtype != torch.uint8 or buf.numel() != n.value or not buf.is_cuda or not buf.is_contiguous():
            raise ValueError(f"expected a contiguous uint8 CUDA tensor of {n.value} bytes")
        self._chk(self.lib.swam_state_import(self.ctx, _ptr(buf), _stream()))

    def cached_scores(self):
        a, b, c = ctypes.c_void_p(), ctypes.c_void_p(), ctypes.c_void_p()
        self._chk(self.lib.swam_get_scores(self.ctx, ctypes.byref(a), ctypes.byref(b), ctypes.byref(c)))
        return (self._view(a, (self.B, self.F, self.N_s), torch.float32),
                self._view(b, (self.B, self.N_h, self.H), torch.float32), self._view(c, (self.B, 3), torch.float32))

    def check(self):
        self._chk(self.lib.swam_check(self.ctx, _stream()))

    def selftest_timeout(self, limit_cycles: int = 100_000):
        """Enqueue the wait self-test: the next check() raises SwamError(ERR_TIMEOUT)."""
        self._chk(self.lib.swam_selftest_timeout(self.ctx, limit_cycles, _stream()))

    def set_option(self, option: int, value: int):
        self._scratch_need.clear()
        self._chk(self.lib.swam_set_option(self.ctx, option, value))

    def set_visibility(self, observed_rows_see: int, future_rows_see: int, action_rows_see: int):
        """Segment-prefix visibility: what the rows of each segment see (SEES_OBSERVED / SEES_FUTURE / SEES_ALL)."""
        self.set_option(OPT_VISIBILITY, observed_rows_see | (future_rows_see << 2) | (action_rows_see << 4))

    def launch_count(self) -> int:
        n = ctypes.c_int64()
        self._chk(self.lib.swam_launch_count(self.ctx, ctypes.byref(n)))
        return n.value


def to_device(x, dtype: int, device=None) -> torch.Tensor:
    """numpy float32 [B, L, N_h, D] (already storage-exact) -> CUDA tensor of the workload dtype."""
    t = torch.from_numpy(x)
    return t.to(device or "cuda", dtype=torch_dtype(dtype)).contiguous()
