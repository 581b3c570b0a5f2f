"""ctypes binding of libforgestep.so: argument marshalling only.

Every step of the training path runs inside the CUDA library; PyTorch is used here for
device memory and the stream.  Loading fails loudly when the library has not been built:
there is no CPU or PyTorch fallback.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, List, Optional, Tuple

import numpy as np

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libforgestep.so")
_lib = None

FT_OK, FT_EINVAL, FT_ENOMEM, FT_ECUDA, FT_ENONFINITE, FT_ETIMEOUT, FT_ENOTFOUND = range(7)
STATUS_NAMES = ["FT_OK", "FT_EINVAL", "FT_ENOMEM", "FT_ECUDA", "FT_ENONFINITE", "FT_ETIMEOUT", "FT_ENOTFOUND"]
KIND_MASTER, KIND_BF16, KIND_ADAM_M, KIND_ADAM_V, KIND_GRAD = range(5)
MAX_IN_FLIGHT = 2  # FT_MAX_IN_FLIGHT of the header
PROF_CLASSES = ["gemm", "attn_fwd", "attn_bwd", "norm", "elementwise", "ce", "optimizer"]


class FtConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "d_model", "n_heads", "n_kv_heads", "head_dim", "d_ffn", "vocab",
                                          "max_batch", "max_seq")] + \
               [(n, C.c_float) for n in ("rms_eps", "rope_theta", "lr", "beta1", "beta2", "adam_eps", "weight_decay",
                                         "max_grad_norm")] + \
               [("recompute", C.c_int32), ("debug_taps", C.c_int32)] + \
               [(n, C.c_float) for n in ("emb_scale", "resid_scale", "logit_scale")] + [("tie_embeddings", C.c_int32),
                                                                                         ("qk_norm", C.c_int32)] + \
               [("mtp", C.c_int32), ("mtp_weight", C.c_float), ("dp_world", C.c_int32), ("dp_rank", C.c_int32)]


class FtAdamWTensor(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("param", "grad", "m", "v", "m_scale", "v_scale", "copy")] + \
               [("numel", C.c_int64), ("weight_decay", C.c_float)]


class ForgeStepError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS_NAMES[status] if 0 <= status < 7 else status}: {msg}")
        self.status = status


def lib():
    """The loaded C-ABI library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise ImportError(f"{_LIB_PATH} is missing: build it with `python -m paper_2609_13645_b200.build`")
        L = C.CDLL(_LIB_PATH)
        vp, i32, i64, f32p, i32p = C.c_void_p, C.c_int32, C.c_int64, C.POINTER(C.c_float), C.POINTER(C.c_int32)
        cfgp = C.POINTER(FtConfig)
        L.ft_workspace_bytes.restype = C.c_size_t
        L.ft_workspace_bytes.argtypes = [cfgp]
        L.ft_init_model.argtypes = [cfgp, C.c_uint64, vp, C.c_size_t, vp, C.POINTER(vp)]
        L.ft_train_step.argtypes = [vp, vp, vp, i32, i32, f32p, f32p]
        L.ft_train_step_host.argtypes = [vp, vp, vp, i32, i32, f32p, f32p]
        L.ft_forward_loss.argtypes = [vp, vp, vp, i32, i32, f32p]
        L.ft_forward_backward.argtypes = [vp, vp, vp, i32, i32, f32p]
        L.ft_apply_update.argtypes = [vp, f32p]
        L.ft_num_params.restype = i32
        L.ft_num_params.argtypes = [vp]
        L.ft_param_info.argtypes = [vp, i32, C.POINTER(C.c_char_p), i32p, C.POINTER(i64)]
        L.ft_get_param.argtypes = [vp, i32, i32, vp, C.c_size_t]
        L.ft_set_param.argtypes = [vp, i32, i32, vp, C.c_size_t]
        L.ft_get_step.argtypes = [vp, C.POINTER(i64)]
        L.ft_set_step.argtypes = [vp, i64]
        L.ft_get_tap.argtypes = [vp, C.c_char_p, i32, vp, C.c_size_t, C.POINTER(C.c_size_t), i32p]
        L.ft_last_error.restype = C.c_char_p
        L.ft_last_error.argtypes = [vp]
        L.ft_launch_count.restype = i64
        L.ft_launch_count.argtypes = [vp]
        L.ft_set_profiling.argtypes = [vp, i32]
        L.ft_set_profiling.restype = C.c_int
        L.ft_get_profile.argtypes = [vp, i32, C.POINTER(C.c_double), C.POINTER(C.c_double), C.POINTER(i64)]
        L.ft_get_profile.restype = C.c_int
        L.ft_debug_gemm_tile.argtypes = [i32]
        L.ft_debug_gemm_tile.restype = None
        L.ft_debug_gemm_pairs.argtypes = [i32]
        L.ft_debug_gemm_pairs.restype = None
        L.ft_debug_gemm_swiglu_tma.argtypes = [i32]
        L.ft_debug_gemm_swiglu_tma.restype = None
        L.ft_debug_gemm_group.argtypes = [i32]
        L.ft_debug_gemm_group.restype = None
        L.ft_debug_gemm_tma_out.argtypes = [i32]
        L.ft_debug_gemm_tma_out.restype = None
        L.ft_get_gemm_profile.argtypes = [vp, i32, C.POINTER(i32), C.POINTER(C.c_double), C.POINTER(i64)]
        L.ft_get_gemm_profile.restype = C.c_int
        L.ft_set_fused_update.argtypes = [vp, i32]
        L.ft_set_fused_update.restype = C.c_int
        L.ft_set_rope_scaling.argtypes = [vp, vp, C.c_float]
        L.ft_set_rope_scaling.restype = C.c_int
        L.ft_set_overlap.argtypes = [vp, i32]
        L.ft_set_overlap.restype = C.c_int
        L.ft_submit_step_host.argtypes = [vp, vp, vp, i32, i32]
        L.ft_submit_step_host.restype = C.c_int
        L.ft_collect_step.argtypes = [vp, vp, vp]
        L.ft_collect_step.restype = C.c_int
        L.ft_set_streaming_ce.argtypes = [vp, i32]
        L.ft_set_streaming_ce.restype = C.c_int
        L.ft_set_attention_stored_ds.argtypes = [vp, i32]
        L.ft_set_attention_stored_ds.restype = C.c_int
        L.ft_attention_window_bytes.argtypes = [vp, i32, i32]
        L.ft_attention_window_bytes.restype = C.c_size_t
        L.ft_set_attention_window.argtypes = [vp, i32, i32, vp, C.c_uint64]
        L.ft_set_attention_window.restype = C.c_int
        L.ft_set_fused_swiglu_bwd.argtypes = [vp, i32]
        L.ft_set_fused_swiglu_bwd.restype = C.c_int
        L.ft_set_graph.argtypes = [vp, i32]
        L.ft_set_graph.restype = C.c_int
        L.ft_graph_replays.argtypes = [vp]
        L.ft_graph_replays.restype = i64
        L.ft_destroy.restype = None
        L.ft_destroy.argtypes = [vp]
        L.ft_k_gemm.argtypes = [vp, i32, i64, vp, i32, i64, vp, i64, vp, i32, i32, i32, i32, vp, vp]
        L.ft_k_gemm_ws.argtypes = [vp, i32, i64, vp, i32, i64, vp, i64, vp, i32, i32, i32, i32, vp, C.c_uint64, vp, vp]
        L.ft_k_gemm_ws.restype = C.c_int
        L.ft_k_attention_fwd.argtypes = [vp, vp, vp, i32, i32, i32, i32, i32, vp]
        L.ft_k_attention_bwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, vp]
        L.ft_k_attention_bwd_ws.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, C.c_uint64, i32, i32, i32, i32, i32, vp]
        L.ft_k_attention_bwd_ws.restype = C.c_int
        L.ft_k_attention_bwd_noalloc.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, vp]
        L.ft_k_attention_bwd_noalloc.restype = C.c_int
        L.ft_k_attention_window_fwd.argtypes = [vp, vp, vp] + [i32] * 7 + [vp]
        L.ft_k_attention_window_bwd.argtypes = [vp] * 8 + [C.c_uint64] + [i32] * 7 + [vp]
        L.ft_k_attention_window_scratch_bytes.restype = C.c_size_t
        L.ft_k_attention_window_scratch_bytes.argtypes = [i32] * 7
        L.ft_k_layernorm_fwd.argtypes = [vp, i64, vp, vp, vp, i64, vp, vp, i32, i32, C.c_float, i32, vp]
        L.ft_k_layernorm_bwd.argtypes = [vp, i64, vp, i64, vp, vp, vp, vp, i64, vp, i64, vp, vp, vp, C.c_uint64, i32, i32, i32, vp]
        L.ft_k_layernorm_scratch_bytes.restype = C.c_size_t
        L.ft_k_layernorm_scratch_bytes.argtypes = [i32, i32]
        L.ft_k_dropout_add.argtypes = [vp, i64, vp, i64, vp, i64, i32, i32, C.c_float, C.c_float, C.c_uint64, i32, vp, i32, vp]
        L.ft_k_packed_bounds.argtypes = [vp, i32, i32, i32, vp, vp]
        L.ft_k_attention_packed_fwd.argtypes = [vp] * 4 + [i32] * 4 + [vp]
        L.ft_k_attention_packed_scratch_bytes.restype = C.c_size_t
        L.ft_k_attention_packed_scratch_bytes.argtypes = [i32] * 5
        L.ft_k_attention_packed_bwd.argtypes = [vp] * 9 + [C.c_uint64] + [i32] * 5 + [vp]
        L.ft_k_rotary.argtypes = [vp, i64, vp, i64, vp, vp, vp] + [i32] * 8 + [vp]
        L.ft_k_rotary_tables.argtypes = [vp, vp, vp, i32, i32, C.c_float, C.c_float, vp]
        L.ft_k_adamw_plan_bytes.restype = C.c_size_t
        L.ft_k_adamw_plan_bytes.argtypes = [vp, i32, i32, i32, i32]
        L.ft_k_adamw_plan.argtypes = [vp, i32, i32, i32, i32, vp, C.c_uint64]
        L.ft_k_adamw.argtypes = [vp, vp, C.c_uint64] + [C.c_double] * 4 + [vp, vp, vp, C.c_uint64, vp]
        for name in ("ft_k_attention_window_fwd", "ft_k_attention_window_bwd", "ft_k_layernorm_fwd", "ft_k_layernorm_bwd",
                     "ft_k_dropout_add", "ft_k_packed_bounds", "ft_k_attention_packed_fwd", "ft_k_attention_packed_bwd", "ft_k_rotary",
                     "ft_k_rotary_tables", "ft_k_adamw_plan", "ft_k_adamw"):
            getattr(L, name).restype = C.c_int
        for name in ("ft_init_model", "ft_train_step", "ft_train_step_host", "ft_forward_loss", "ft_forward_backward",
                     "ft_apply_update", "ft_param_info", "ft_get_param", "ft_set_param", "ft_get_step", "ft_set_step",
                     "ft_get_tap", "ft_k_gemm", "ft_k_attention_fwd", "ft_k_attention_bwd"):
            getattr(L, name).restype = C.c_int
        _lib = L
    return _lib


def make_config(n_layers, d_model, n_heads, n_kv_heads, head_dim, d_ffn, vocab, max_batch, max_seq, rms_eps=1e-5,
                rope_theta=1e4, lr=1e-3, beta1=0.9, beta2=0.95, adam_eps=1e-8, weight_decay=0.1, max_grad_norm=0.0,
                recompute=0, debug_taps=0, emb_scale=1.0, resid_scale=1.0, logit_scale=1.0, tie_embeddings=0, qk_norm=0,
                mtp=0, mtp_weight=1.0, dp_world=0, dp_rank=0) -> FtConfig:
    return FtConfig(n_layers, d_model, n_heads, n_kv_heads, head_dim, d_ffn, vocab, max_batch, max_seq, rms_eps,
                    rope_theta, lr, beta1, beta2, adam_eps, weight_decay, max_grad_norm, recompute, debug_taps,
                    emb_scale, resid_scale, logit_scale, int(tie_embeddings), int(qk_norm), int(mtp), mtp_weight, int(dp_world),
                    int(dp_rank))


def workspace_bytes(cfg: FtConfig) -> int:
    return int(lib().ft_workspace_bytes(C.byref(cfg)))


def _stream_ptr():
    import torch
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _stream_of(index: int) -> int:
    """The current stream of device `index` as a plain address (the raw query takes 0.1 us where torch.cuda.current_stream()
    takes 3.3, which a launch-bound operator would notice)."""
    torch = _torch or _import_torch()
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(index) if raw is not None else torch.cuda.current_stream(index).cuda_stream


_torch = None


def _import_torch():
    global _torch
    import torch
    _torch = torch
    return torch


def bf16_bits_to_f32(a: np.ndarray) -> np.ndarray:
    """uint16 bf16 bit patterns -> float32 values (exact)."""
    return (a.astype(np.uint32) << 16).view(np.float32)


class Model:
    """A decoder + optimizer state living in one torch-allocated workspace on the current CUDA device."""

    def __init__(self, cfg: FtConfig, seed: int = 1234):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("forgestep needs a CUDA device (sm_100a); there is no CPU path")
        self.cfg = cfg
        nbytes = workspace_bytes(cfg)
        if nbytes == 0:
            raise ForgeStepError(FT_EINVAL, "invalid config")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        self._h = C.c_void_p()
        self._pending = []
        st = lib().ft_init_model(C.byref(cfg), C.c_uint64(seed), C.c_void_p(self.workspace.data_ptr()), nbytes,
                                 _stream_ptr(), C.byref(self._h))
        self._check(st)
        self.params: List[Tuple[str, Tuple[int, ...]]] = []
        for i in range(lib().ft_num_params(self._h)):
            name, nd, shp = C.c_char_p(), C.c_int32(), (C.c_int64 * 2)()
            self._check(lib().ft_param_info(self._h, i, C.byref(name), C.byref(nd), shp))
            self.params.append((name.value.decode(), (int(shp[0]), int(shp[1])) if nd.value == 2 else (int(shp[0]),)))
        self.index: Dict[str, int] = {n: i for i, (n, _) in enumerate(self.params)}

    def _check(self, st: int):
        if st != FT_OK:
            msg = lib().ft_last_error(self._h).decode() if self._h else "no handle"
            raise ForgeStepError(st, msg)

    def close(self):
        if self._h:
            # the library also works on streams of its own (weight gradients): nothing of this model may still be running
            # when its workspace goes back to the allocator
            import torch
            torch.cuda.synchronize()
            lib().ft_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- steps (device tensors: int32 [B, S], contiguous) -------------------------------------------
    def train_step(self, tokens, labels, want_loss: bool = True):
        B, S = tokens.shape
        loss, gn = C.c_float(), C.c_float()
        st = lib().ft_train_step(self._h, C.c_void_p(tokens.data_ptr()), C.c_void_p(labels.data_ptr()), B, S,
                                 C.byref(loss) if want_loss else None, C.byref(gn) if want_loss else None)
        self._check(st)
        return (loss.value, gn.value) if want_loss else None

    def train_step_host(self, tokens: np.ndarray, labels: np.ndarray):
        """tokens, labels: int32 numpy arrays [B, S] in host memory (copied to the device inside the call)."""
        B, S = tokens.shape
        loss, gn = C.c_float(), C.c_float()
        st = lib().ft_train_step_host(self._h, C.c_void_p(tokens.ctypes.data), C.c_void_p(labels.ctypes.data), B, S,
                                      C.byref(loss), C.byref(gn))
        self._check(st)
        return loss.value, gn.value

    def submit_step_host(self, tokens: np.ndarray, labels: np.ndarray):
        """Enqueue one train step on host int32 arrays [B, S] (ideally pinned) without waiting for it; at most
        MAX_IN_FLIGHT steps may be outstanding.  The arrays must stay unchanged until the step is collected."""
        B, S = tokens.shape
        self._pending.append((tokens, labels))  # keep the buffers alive while the copy may still run
        self._check(lib().ft_submit_step_host(self._h, C.c_void_p(tokens.ctypes.data), C.c_void_p(labels.ctypes.data), B, S))

    def collect_step(self):
        """Wait for the oldest submitted step; returns its (loss, gradient norm)."""
        loss, gn = C.c_float(), C.c_float()
        st = lib().ft_collect_step(self._h, C.byref(loss), C.byref(gn))
        if self._pending:
            self._pending.pop(0)
        self._check(st)
        return loss.value, gn.value

    def forward_loss(self, tokens, labels) -> float:
        B, S = tokens.shape
        loss = C.c_float()
        self._check(lib().ft_forward_loss(self._h, C.c_void_p(tokens.data_ptr()), C.c_void_p(labels.data_ptr()), B, S,
                                          C.byref(loss)))
        return loss.value

    def forward_backward(self, tokens, labels) -> float:
        B, S = tokens.shape
        loss = C.c_float()
        self._check(lib().ft_forward_backward(self._h, C.c_void_p(tokens.data_ptr()), C.c_void_p(labels.data_ptr()), B,
                                              S, C.byref(loss)))
        return loss.value

    def apply_update(self) -> float:
        gn = C.c_float()
        self._check(lib().ft_apply_update(self._h, C.byref(gn)))
        return gn.value

    # ---- state ------------------------------------------------------------------------------------------
    def get_param(self, name: str, kind: int = KIND_MASTER) -> np.ndarray:
        i = self.index[name]
        shape = self.params[i][1]
        out = np.empty(shape, dtype=np.uint16 if kind == KIND_BF16 else np.float32)
        self._check(lib().ft_get_param(self._h, i, kind, C.c_void_p(out.ctypes.data), out.nbytes))
        return bf16_bits_to_f32(out) if kind == KIND_BF16 else out

    def set_param(self, name: str, value: np.ndarray, kind: int = KIND_MASTER):
        if kind == KIND_BF16:
            raise ValueError("the bf16 copy is derived from the master; set the master instead")
        i = self.index[name]
        v = np.ascontiguousarray(value, dtype=np.float32).reshape(self.params[i][1])
        self._check(lib().ft_set_param(self._h, i, kind, C.c_void_p(v.ctypes.data), v.nbytes))

    @property
    def step(self) -> int:
        s = C.c_int64()
        self._check(lib().ft_get_step(self._h, C.byref(s)))
        return s.value

    @step.setter
    def step(self, v: int):
        self._check(lib().ft_set_step(self._h, int(v)))

    def get_tap(self, name: str, layer: int = -1) -> np.ndarray:
        """Named intermediate of the last step as a flat float32 array."""
        need, dt = C.c_size_t(), C.c_int32()
        probe = np.empty(1, dtype=np.uint8)
        st = lib().ft_get_tap(self._h, name.encode(), layer, C.c_void_p(probe.ctypes.data), 0, C.byref(need),
                              C.byref(dt))
        if st == FT_ENOTFOUND:
            self._check(st)
        buf = np.empty(need.value, dtype=np.uint8)
        self._check(lib().ft_get_tap(self._h, name.encode(), layer, C.c_void_p(buf.ctypes.data), buf.nbytes,
                                     C.byref(need), C.byref(dt)))
        return buf.view(np.float32).copy() if dt.value == 1 else bf16_bits_to_f32(buf.view(np.uint16))

    def set_fused_update(self, enable: bool):
        """AdamW inside the weight-gradient GEMM epilogues (default on; only takes effect with clipping off)."""
        self._check(lib().ft_set_fused_update(self._h, 1 if enable else 0))

    def set_rope_scaling(self, factors=None, mscale: float = 1.0):
        """LongRoPE-form position tables: per-frequency rescale factors (head_dim / 2 floats, None = 1) and a magnitude
        factor on cos and sin."""
        f = None if factors is None else np.ascontiguousarray(factors, dtype=np.float32)
        self._check(lib().ft_set_rope_scaling(self._h, None if f is None else C.c_void_p(f.ctypes.data), float(mscale)))

    def set_overlap(self, enable: bool):
        """Weight-gradient GEMMs on a second stream, concurrent with the rest of the backward pass (default on)."""
        self._check(lib().ft_set_overlap(self._h, 1 if enable else 0))

    def set_streaming_ce(self, enable: bool):
        """Cross-entropy inside the logits GEMM's epilogues (no logits in memory, the GEMM runs twice); default off."""
        self._check(lib().ft_set_streaming_ce(self._h, 1 if enable else 0))

    def set_attention_stored_ds(self, enable: bool):
        """Attention backward that stores dS^T once and computes dQ as one batched contraction (default on)."""
        self._check(lib().ft_set_attention_stored_ds(self._h, 1 if enable else 0))

    def set_attention_window(self, window: int, n_sinks: int = 0):
        """Sliding-window attention with sink keys in every layer (query i sees key j iff j <= i and (i - j < window or
        j < n_sinks)); window 0: causal over the whole sequence (the default).  Holds the scratch of its backward pass."""
        import torch
        scratch = None
        if window > 0 and n_sinks >= 0:
            window, n_sinks = min(window, self.cfg.max_seq), min(n_sinks, self.cfg.max_seq)
            nbytes = int(lib().ft_attention_window_bytes(self._h, window, n_sinks))
            scratch = torch.empty(nbytes, dtype=torch.uint8, device=self.workspace.device)
        self._check(lib().ft_set_attention_window(self._h, window, n_sinks, C.c_void_p(scratch.data_ptr()) if scratch is not None else None,
                                                  scratch.numel() if scratch is not None else 0))
        torch.cuda.synchronize(self.workspace.device)  # steps in flight still use the old scratch
        self._attn_window_scratch = scratch

    def set_fused_swiglu_bwd(self, enable: bool):
        """SwiGLU backward in the epilogue of the down projection's data-gradient GEMM (default on; bit-identical)."""
        self._check(lib().ft_set_fused_swiglu_bwd(self._h, 1 if enable else 0))

    def set_graph(self, enable: bool):
        """Capture the whole step into a CUDA graph on its second run and replay it afterwards."""
        self._check(lib().ft_set_graph(self._h, 1 if enable else 0))

    @property
    def graph_replays(self) -> int:
        return int(lib().ft_graph_replays(self._h))

    def set_profiling(self, enable: bool):
        self._check(lib().ft_set_profiling(self._h, 1 if enable else 0))

    def get_profile(self) -> Dict[str, Dict[str, float]]:
        """Per kernel class: device milliseconds, algorithmic work (FLOPs or bytes) and kernel count."""
        out = {}
        for cls, name in enumerate(PROF_CLASSES):
            ms, work, n = C.c_double(), C.c_double(), C.c_int64()
            self._check(lib().ft_get_profile(self._h, cls, C.byref(ms), C.byref(work), C.byref(n)))
            out[name] = dict(ms=ms.value, work=work.value, launches=int(n.value))
        return out

    def get_gemm_profile(self):
        """List of dicts (M, N, K, a_mn, b_mn, epi, M2, N2, ms, launches, tflops) for every GEMM shape seen while profiling;
        M2 x N2: the second output of a launch that computed two weight gradients at once (0 otherwise)."""
        out, i = [], 0
        while True:
            shp, ms, n = (C.c_int32 * 8)(), C.c_double(), C.c_int64()
            st = lib().ft_get_gemm_profile(self._h, i, shp, C.byref(ms), C.byref(n))
            if st == FT_ENOTFOUND:
                break
            self._check(st)
            M, N, K, M2, N2 = shp[0], shp[1], shp[2], shp[6], shp[7]
            out.append(dict(M=M, N=N, K=K, a_mn=shp[3], b_mn=shp[4], epi=shp[5], M2=M2, N2=N2, ms=ms.value, launches=int(n.value),
                            tflops=2.0 * (M * N + M2 * N2) * K * n.value / (ms.value * 1e-3) / 1e12 if ms.value > 0 else 0.0))
            i += 1
        return out

    @property
    def launch_count(self) -> int:
        return int(lib().ft_launch_count(self._h))


# ---- single kernels (torch device tensors) ---------------------------------------------------------------
def k_gemm(A, a_mn: int, B, b_mn: int, Cout, out_kind: int, M: int, N: int, K: int, err, resid=None):
    """C[M,N] = sum_k A[m,k] B[n,k] on device tensors; leading dimensions are the tensors' row strides."""
    st = lib().ft_k_gemm(C.c_void_p(A.data_ptr()), a_mn, A.stride(0), C.c_void_p(B.data_ptr()), b_mn, B.stride(0),
                         C.c_void_p(Cout.data_ptr()), Cout.stride(0),
                         C.c_void_p(resid.data_ptr()) if resid is not None else None, out_kind, M, N, K,
                         C.c_void_p(err.data_ptr()), _stream_ptr())
    if st != FT_OK:
        raise ForgeStepError(st, "ft_k_gemm")


def k_gemm_ws(A, a_mn: int, B, b_mn: int, Cout, out_kind: int, M: int, N: int, K: int, scratch, err, resid=None):
    """k_gemm with an fp32 device scratch tensor, which enables the deterministic split-K / balanced-K schedules."""
    st = lib().ft_k_gemm_ws(C.c_void_p(A.data_ptr()), a_mn, A.stride(0), C.c_void_p(B.data_ptr()), b_mn, B.stride(0),
                            C.c_void_p(Cout.data_ptr()), Cout.stride(0),
                            C.c_void_p(resid.data_ptr()) if resid is not None else None, out_kind, M, N, K,
                            C.c_void_p(scratch.data_ptr()), scratch.numel() * 4, C.c_void_p(err.data_ptr()),
                            _stream_ptr())
    if st != FT_OK:
        raise ForgeStepError(st, "ft_k_gemm_ws")


def k_attention_fwd(qkv, o, lse, B, S, n_heads, n_kv, d):
    st = lib().ft_k_attention_fwd(C.c_void_p(qkv.data_ptr()), C.c_void_p(o.data_ptr()), C.c_void_p(lse.data_ptr()), B,
                                  S, n_heads, n_kv, d, _stream_ptr())
    if st != FT_OK:
        raise ForgeStepError(st, "ft_k_attention_fwd")


def k_attention_bwd(qkv, o, d_o, lse, delta, dqkv, B, S, n_heads, n_kv, d, cos=None, sin=None):
    st = lib().ft_k_attention_bwd(C.c_void_p(qkv.data_ptr()), C.c_void_p(o.data_ptr()), C.c_void_p(d_o.data_ptr()),
                                  C.c_void_p(lse.data_ptr()), C.c_void_p(delta.data_ptr()),
                                  C.c_void_p(dqkv.data_ptr()), C.c_void_p(cos.data_ptr()) if cos is not None else None,
                                  C.c_void_p(sin.data_ptr()) if sin is not None else None, B, S, n_heads, n_kv, d,
                                  _stream_ptr())
    if st != FT_OK:
        raise ForgeStepError(st, "ft_k_attention_bwd")


def k_attention_bwd_ws(qkv, o, d_o, lse, delta, dqkv, ds, B, S, n_heads, n_kv, d, cos=None, sin=None):
    """Attention backward with a dS^T scratch tensor `ds` (bf16, at least B * n_heads * S * S elements) or None."""
    st = lib().ft_k_attention_bwd_ws(C.c_void_p(qkv.data_ptr()), C.c_void_p(o.data_ptr()), C.c_void_p(d_o.data_ptr()),
                                     C.c_void_p(lse.data_ptr()), C.c_void_p(delta.data_ptr()),
                                     C.c_void_p(dqkv.data_ptr()), C.c_void_p(cos.data_ptr()) if cos is not None else None,
                                     C.c_void_p(sin.data_ptr()) if sin is not None else None,
                                     C.c_void_p(ds.data_ptr()) if ds is not None else None,
                                     ds.numel() * ds.element_size() if ds is not None else 0, B, S, n_heads, n_kv, d,
                                     _stream_ptr())
    if st != FT_OK:
        raise ForgeStepError(st, "ft_k_attention_bwd_ws")


def k_attention_bwd_noalloc(qkv, o, d_o, lse, dqkv, B, S, n_heads, n_kv, d, cos=None, sin=None):
    """Attention backward whose scratch lives inside the library: for callers that may not allocate device memory.
    Returns the status code instead of raising, so a caller can tell "too large for the built-in scratch" apart."""
    return lib().ft_k_attention_bwd_noalloc(
        C.c_void_p(qkv.data_ptr()), C.c_void_p(o.data_ptr()), C.c_void_p(d_o.data_ptr()), C.c_void_p(lse.data_ptr()),
        C.c_void_p(dqkv.data_ptr()), C.c_void_p(cos.data_ptr()) if cos is not None else None,
        C.c_void_p(sin.data_ptr()) if sin is not None else None, B, S, n_heads, n_kv, d, _stream_ptr())


# ---- decoder-block operators -------------------------------------------------------------------------------
# Unlike the calls above these check the tensors they are given (type, shape, layout, device) before anything is launched;
# a refused call raises ForgeStepError with status FT_EINVAL.
_INT32_MAX = 2 ** 31 - 1


def _refuse(what: str):
    raise ForgeStepError(FT_EINVAL, what)


def _check_flat(name, t, dtype, numel, index):
    """The address of a contiguous tensor of exactly `numel` elements on device `index`."""
    if t.dtype is not dtype or t.numel() != numel or not t.is_contiguous() or t.get_device() != index:
        _refuse(f"{name}: expected {numel} contiguous {dtype} elements on cuda:{index}, got {tuple(t.shape)} {t.dtype} on {t.device}, "
                f"strides {t.stride()}")
    return t.data_ptr()


def _check_rows(name, t, dtype, rows, h, index):
    """(address, row stride) of a [rows, h] tensor whose rows are contiguous."""
    if t.dtype is not dtype or t.shape != (rows, h) or t.get_device() != index:
        _refuse(f"{name}: expected [{rows}, {h}] {dtype} on cuda:{index}, got {tuple(t.shape)} {t.dtype} on {t.device}")
    ld, one = t.stride()
    if one != 1 and h > 1:
        _refuse(f"{name}: the elements of a row have to be contiguous, got strides {t.stride()}")
    if rows == 1:
        ld = h
    elif ld < h:
        _refuse(f"{name}: rows overlap, strides {t.stride()}")
    return t.data_ptr(), ld


def _current_device(t):
    """Index of the device of the call's tensors, which has to be the current one (kernels run on its current stream)."""
    index = t.get_device()
    if index < 0:
        _refuse(f"tensors on {t.device}: a CUDA device is needed")
    current = (_torch or _import_torch()).cuda.current_device()
    if index != current:
        _refuse(f"tensors on {t.device}, current device cuda:{current}")
    return index


def _row_dtype(t):
    torch = _torch or _import_torch()
    if t.dtype == torch.bfloat16:
        return 0
    if t.dtype == torch.float32:
        return 1
    _refuse(f"{t.dtype}: bf16 and fp32 are supported")


def _window_shape(B, S, n_heads, n_kv, d, window, n_sinks):
    if min(B, S, n_heads, n_kv, window) < 1 or n_sinks < 0 or n_heads % n_kv or d not in (64, 128):
        _refuse(f"B {B}, S {S}, heads {n_heads} / {n_kv} of {d}, window {window}, sinks {n_sinks}")
    return min(window, S), min(n_sinks, S)  # a mask beyond the sequence is one that covers it


def attention_window_scratch_bytes(B, S, n_heads, n_kv, d, window, n_sinks) -> int:
    """Bytes of device scratch k_attention_window_bwd needs."""
    window, n_sinks = _window_shape(B, S, n_heads, n_kv, d, window, n_sinks)
    if max(B, S, n_heads) > _INT32_MAX:
        _refuse(f"B {B}, S {S}, heads {n_heads}: more than 32 bits hold")
    return int(lib().ft_k_attention_window_scratch_bytes(B, S, n_heads, n_kv, d, window, n_sinks))


def k_attention_window_fwd(qkv, o, lse, B, S, n_heads, n_kv, d, window, n_sinks=0):
    """Causal attention in which query i sees key j iff j <= i and (i - j < window or j < n_sinks)."""
    torch = _torch or _import_torch()
    window, n_sinks = _window_shape(B, S, n_heads, n_kv, d, window, n_sinks)
    dev = _current_device(qkv)
    T = B * S
    st = lib().ft_k_attention_window_fwd(_check_flat("qkv", qkv, torch.bfloat16, T * (n_heads + 2 * n_kv) * d, dev),
                                         _check_flat("o", o, torch.bfloat16, T * n_heads * d, dev),
                                         _check_flat("lse", lse, torch.float32, T * n_heads, dev),
                                         B, S, n_heads, n_kv, d, window, n_sinks, _stream_of(dev))
    if st != FT_OK:
        raise ForgeStepError(st, "ft_k_attention_window_fwd")


def k_attention_window_bwd(qkv, o, d_o, lse, dqkv, scratch, B, S, n_heads, n_kv, d, window, n_sinks=0, cos=None, sin=None):
    """Gradient of k_attention_window_fwd; scratch: a uint8 tensor of attention_window_scratch_bytes(...) bytes; cos, sin: fp32
    [S, d / 2] tables by which d_q and d_k are rotated back, or None."""
    torch = _torch or _import_torch()
    window, n_sinks = _window_shape(B, S, n_heads, n_kv, d, window, n_sinks)
    dev, bf16, f32 = _current_device(qkv), torch.bfloat16, torch.float32
    T = B * S
    if (cos is None) != (sin is None):
        _refuse("cos and sin: both or neither")
    st = lib().ft_k_attention_window_bwd(
        _check_flat("qkv", qkv, bf16, T * (n_heads + 2 * n_kv) * d, dev), _check_flat("o", o, bf16, T * n_heads * d, dev),
        _check_flat("d_o", d_o, bf16, T * n_heads * d, dev), _check_flat("lse", lse, f32, T * n_heads, dev),
        _check_flat("dqkv", dqkv, bf16, T * (n_heads + 2 * n_kv) * d, dev),
        _check_flat("cos", cos, f32, S * d // 2, dev) if cos is not None else None,
        _check_flat("sin", sin, f32, S * d // 2, dev) if sin is not None else None,
        _check_flat("scratch", scratch, torch.uint8, scratch.numel(), dev), scratch.numel(), B, S, n_heads, n_kv, d, window, n_sinks,
        _stream_of(dev))
    if st != FT_OK:
        raise ForgeStepError(st, "ft_k_attention_window_bwd")


def _rows_of(x):
    if x.dim() != 2:
        _refuse(f"x: expected [rows, h], got {tuple(x.shape)}")
    rows, h = x.shape
    if rows > _INT32_MAX or h > _INT32_MAX:
        _refuse(f"x: {rows} x {h}, more than 32 bits hold")  # which ctypes would cut off without a word
    return rows, h


def k_layernorm_fwd(x, gain, bias, y, mean, rstd, eps=1e-5):
    """y = (x - mean) rstd gain + bias over the rows of x [rows, h] (bf16 or fp32, any row stride); bias may be None."""
    torch = _torch or _import_torch()
    dt, dev, dtype = _row_dtype(x), _current_device(x), x.dtype
    rows, h = _rows_of(x)
    px, ldx = _check_rows("x", x, dtype, rows, h, dev)
    py, ldy = _check_rows("y", y, dtype, rows, h, dev)
    st = lib().ft_k_layernorm_fwd(px, ldx, _check_flat("gain", gain, dtype, h, dev),
                                  _check_flat("bias", bias, dtype, h, dev) if bias is not None else None, py, ldy,
                                  _check_flat("mean", mean, torch.float32, rows, dev),
                                  _check_flat("rstd", rstd, torch.float32, rows, dev), rows, h, eps, dt, _stream_of(dev))
    if st != FT_OK:
        raise ForgeStepError(st, "ft_k_layernorm_fwd")


def layernorm_scratch_bytes(rows, h) -> int:
    """Bytes of device scratch k_layernorm_bwd needs (0: the shape is refused)."""
    if max(rows, h) > _INT32_MAX:
        return 0
    return int(lib().ft_k_layernorm_scratch_bytes(rows, h))


def k_layernorm_bwd(dy, x, mean, rstd, gain, resid, dx, dgain, dbias, scratch):
    """dx = R(LayerNorm's input gradient + resid), dgain and dbias in fp32; resid and dbias may be None; scratch: a uint8
    tensor of layernorm_scratch_bytes(rows, h) bytes."""
    torch = _torch or _import_torch()
    dt, dev, dtype, f32 = _row_dtype(x), _current_device(x), x.dtype, torch.float32
    rows, h = _rows_of(x)
    px, ldx = _check_rows("x", x, dtype, rows, h, dev)
    pdy, lddy = _check_rows("dy", dy, dtype, rows, h, dev)
    pdx, lddx = _check_rows("dx", dx, dtype, rows, h, dev)
    pr, ldr = _check_rows("resid", resid, dtype, rows, h, dev) if resid is not None else (None, 0)
    st = lib().ft_k_layernorm_bwd(pdy, lddy, px, ldx, _check_flat("mean", mean, f32, rows, dev), _check_flat("rstd", rstd, f32, rows, dev),
                                  _check_flat("gain", gain, dtype, h, dev), pr, ldr, pdx, lddx, _check_flat("dgain", dgain, f32, h, dev),
                                  _check_flat("dbias", dbias, f32, h, dev) if dbias is not None else None,
                                  _check_flat("scratch", scratch, torch.uint8, scratch.numel(), dev), scratch.numel(), rows, h, dt,
                                  _stream_of(dev))
    if st != FT_OK:
        raise ForgeStepError(st, "ft_k_layernorm_bwd")


def k_dropout_add(x, resid, y, p, seed, site, step=None, scale=1.0):
    """y = R(resid + scale / (1 - p) keep x) over [rows, h] tensors; the mask is a function of (seed, site, step, element), so
    the backward pass is this call on the gradient with resid None.  step: int64 tensor of one element, read when the
    kernel runs."""
    torch = _torch or _import_torch()
    dt, dev, dtype = _row_dtype(x), _current_device(x), x.dtype
    rows, h = _rows_of(x)
    if not 0 <= site <= _INT32_MAX:
        _refuse(f"site {site}")
    px, ldx = _check_rows("x", x, dtype, rows, h, dev)
    py, ldy = _check_rows("y", y, dtype, rows, h, dev)
    pr, ldr = _check_rows("resid", resid, dtype, rows, h, dev) if resid is not None else (None, 0)
    st = lib().ft_k_dropout_add(px, ldx, pr, ldr, py, ldy, rows, h, p, scale, seed & 0xFFFFFFFFFFFFFFFF, site,
                                _check_flat("step", step, torch.int64, 1, dev) if step is not None else None, dt, _stream_of(dev))
    if st != FT_OK:
        raise ForgeStepError(st, "ft_k_dropout_add")


# ---- operators of a train step over packed documents ---------------------------------------------------------
def _packed_shape(T, n_heads, n_kv, d, longest=1):
    if not (1 <= T <= _INT32_MAX and 1 <= n_kv <= n_heads <= _INT32_MAX and 1 <= longest <= _INT32_MAX) or n_heads % n_kv or (d != 64 and d != 128):
        _refuse(f"T {T}, heads {n_heads} / {n_kv} of {d}, longest document {longest}")


def k_packed_bounds(offsets, bounds, T, longest=None):
    """The bounds of every row's document in a packed batch of T rows, once a batch.  offsets: int32 [documents + 1], the first rows of
    the documents and the end of the last, ascending from 0 to at most T (on the device; what breaks this is reported by k_status);
    bounds: int32 [3, T]: first row, row behind the last, position in the document; longest: rows of a document, at most (None: T)."""
    torch = _torch or _import_torch()
    longest = T if longest is None else min(longest, T)
    if not 1 <= T <= _INT32_MAX or longest < 1:
        _refuse(f"T {T}, longest document {longest}")
    dev = _current_device(offsets)
    n = offsets.numel()
    if n < 1 or n > _INT32_MAX:
        _refuse(f"offsets: {n} elements")
    st = lib().ft_k_packed_bounds(_check_flat("offsets", offsets, torch.int32, n, dev), n - 1, T, longest,
                                  _check_flat("bounds", bounds, torch.int32, 3 * T, dev), _stream_of(dev))
    if st != FT_OK:
        raise ForgeStepError(st, "ft_k_packed_bounds")


def attention_packed_scratch_bytes(T, n_heads, n_kv, d, longest=None) -> int:
    """Bytes of device scratch k_attention_packed_bwd needs; longest: rows of a document, at most (None: T)."""
    longest = T if longest is None else min(longest, T)
    _packed_shape(T, n_heads, n_kv, d, longest)
    return int(lib().ft_k_attention_packed_scratch_bytes(T, n_heads, n_kv, d, longest))


def k_attention_packed_fwd(qkv, o, lse, bounds, T, n_heads, n_kv, d):
    """Causal attention inside the documents of a packed batch: a row sees the rows from its document's first one to itself.  qkv
    [T, (n_heads + 2 n_kv) d], o [T, n_heads d] (bf16), lse [n_heads, T] (fp32), bounds: what k_packed_bounds left.  Rows behind the
    last document are left as they were."""
    torch = _torch or _import_torch()
    _packed_shape(T, n_heads, n_kv, d)
    dev = _current_device(qkv)
    st = lib().ft_k_attention_packed_fwd(_check_flat("qkv", qkv, torch.bfloat16, T * (n_heads + 2 * n_kv) * d, dev),
                                         _check_flat("o", o, torch.bfloat16, T * n_heads * d, dev),
                                         _check_flat("lse", lse, torch.float32, T * n_heads, dev),
                                         _check_flat("bounds", bounds, torch.int32, 3 * T, dev), T, n_heads, n_kv, d, _stream_of(dev))
    if st != FT_OK:
        raise ForgeStepError(st, "ft_k_attention_packed_fwd")


def k_attention_packed_bwd(qkv, o, d_o, lse, dqkv, bounds, scratch, T, n_heads, n_kv, d, longest=None, cos=None, sin=None):
    """Gradient of k_attention_packed_fwd; scratch: a uint8 tensor of attention_packed_scratch_bytes(...) bytes; longest: as given to
    k_packed_bounds, or more (a longer document in the bounds is reported by k_status); cos, sin: fp32 [longest or more, d / 2] tables by which d_q and d_k are rotated back at their rows'
    positions, or None.  Rows of dqkv behind the last document are left as they were."""
    torch = _torch or _import_torch()
    longest = T if longest is None else min(longest, T)
    _packed_shape(T, n_heads, n_kv, d, longest)
    dev, bf16, f32 = _current_device(qkv), torch.bfloat16, torch.float32
    if (cos is None) != (sin is None):
        _refuse("cos and sin: both or neither")
    if cos is not None and (cos.numel() < longest * d // 2 or cos.shape != sin.shape):
        _refuse(f"cos {tuple(cos.shape)}, sin {tuple(sin.shape)}: [{longest} or more, {d // 2}] are needed")
    st = lib().ft_k_attention_packed_bwd(
        _check_flat("qkv", qkv, bf16, T * (n_heads + 2 * n_kv) * d, dev), _check_flat("o", o, bf16, T * n_heads * d, dev),
        _check_flat("d_o", d_o, bf16, T * n_heads * d, dev), _check_flat("lse", lse, f32, T * n_heads, dev),
        _check_flat("dqkv", dqkv, bf16, T * (n_heads + 2 * n_kv) * d, dev), _check_flat("bounds", bounds, torch.int32, 3 * T, dev),
        _check_flat("cos", cos, f32, cos.numel(), dev) if cos is not None else None,
        _check_flat("sin", sin, f32, sin.numel(), dev) if sin is not None else None,
        _check_flat("scratch", scratch, torch.uint8, scratch.numel(), dev), scratch.numel(), T, n_heads, n_kv, d, longest, _stream_of(dev))
    if st != FT_OK:
        raise ForgeStepError(st, "ft_k_attention_packed_bwd")


def k_status():
    """Waits for the current stream and raises if a call since the last k_status met a wait that ran out (FT_ETIMEOUT) or a value on
    the device that it refuses (FT_EINVAL): offsets of documents, documents over the limit of a backward pass, positions."""
    st = lib().ft_k_status(_stream_ptr())
    if st != FT_OK:
        raise ForgeStepError(st, "a call on the device")


def _check_tables(cos, sin, index):
    torch = _torch or _import_torch()
    shape = cos.shape
    if len(shape) != 2 or sin.shape != shape or not 0 < shape[0] <= _INT32_MAX or not 0 < shape[1] <= 1 << 20:
        _refuse(f"cos {tuple(shape)}, sin {tuple(sin.shape)}: [positions, pairs] are needed")
    n = shape[0] * shape[1]
    return _check_flat("cos", cos, torch.float32, n, index), _check_flat("sin", sin, torch.float32, n, index)


def k_rotary(x, y, cos, sin, n_heads, d, positions=None, interleaved=False, inverse=False):
    """Rotary positions on the heads of x [rows, n_heads d] (bf16 or fp32, any row stride) into y, which may be x.  cos, sin: fp32
    [positions, pairs] tables; the first 2 pairs elements of each head are rotated, as (i, i + pairs) or, interleaved, as
    (2 i, 2 i + 1), the others passed on.  positions: int32 [rows] (None: the row's number); one outside the tables is reported by
    k_status and its row not written.  inverse: the transpose, which is the backward pass."""
    torch = _torch or _import_torch()
    dt, dev, dtype = _row_dtype(x), _current_device(x), x.dtype
    rows, h = _rows_of(x)
    if n_heads < 1 or d < 1 or n_heads * d != h:
        _refuse(f"x: {h} columns are not {n_heads} heads of {d}")
    px, ldx = _check_rows("x", x, dtype, rows, h, dev)
    py, ldy = (px, ldx) if y is x else _check_rows("y", y, dtype, rows, h, dev)
    pc, ps = _check_tables(cos, sin, dev)
    st = lib().ft_k_rotary(px, ldx, py, ldy, _check_flat("positions", positions, torch.int32, rows, dev) if positions is not None else None,
                           pc, ps, cos.shape[0], rows, n_heads, d, 2 * cos.shape[1], 1 if interleaved else 0, 1 if inverse else 0, dt,
                           _stream_of(dev))
    if st != FT_OK:
        raise ForgeStepError(st, "ft_k_rotary")


def k_rotary_tables(cos, sin, theta=1e4, factors=None, mscale=1.0):
    """Fills cos and sin (fp32 [positions, pairs]) with mscale times those of p theta^(-i / pairs) / factors[i] (fp32 [pairs], None: 1)."""
    torch = _torch or _import_torch()
    dev = _current_device(cos)
    pc, ps = _check_tables(cos, sin, dev)
    st = lib().ft_k_rotary_tables(pc, ps, _check_flat("factors", factors, torch.float32, cos.shape[1], dev) if factors is not None else None,
                                  cos.shape[0], 2 * cos.shape[1], theta, mscale, _stream_of(dev))
    if st != FT_OK:
        raise ForgeStepError(st, "ft_k_rotary_tables")


class AdamWPlan:
    """The tensors that k_adamw steps through, handed over once.  Lists of equal length: params (all bf16 or all fp32), grads (all
    bf16 or all fp32), first and second moments (all fp32, or all torch.float8_e4m3fn: m and the square root of v over the scales
    m_scales, v_scales, fp32, one for every 256 elements begun), weight_decay (a number or a list), copies (bf16, or None).  All
    contiguous and on one device.  The plan keeps them alive and steps through their memory as it is now: give gradients that
    stay where they are (zeroed, not set to None), for a plan takes 4 us a tensor to make and waits for the GPU's copy."""

    def __init__(self, params, grads, m, v, weight_decay=0.0, m_scales=None, v_scales=None, copies=None):
        torch = _torch or _import_torch()
        n = len(params)
        decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else [weight_decay] * n
        lists = [list(t) if t is not None else None for t in (params, grads, m, v, m_scales, v_scales, copies)]
        if n == 0 or any(len(t) != n for t in lists if t is not None) or len(decay) != n:
            _refuse("params, grads, m, v, weight_decay, scales and copies: lists of one length")
        params, grads, m, v, m_scales, v_scales, copies = lists
        if any(t is None for of in (params, grads, m, v) for t in of):
            _refuse("params, grads, m and v: a tensor is missing")
        pt, gt, mt = params[0].dtype, grads[0].dtype, m[0].dtype
        param_dtype, grad_dtype = _row_dtype(params[0]), _row_dtype(grads[0])
        if mt not in (torch.float32, torch.float8_e4m3fn):
            _refuse(f"{mt}: moments are fp32 or float8_e4m3fn")
        bits = 32 if mt == torch.float32 else 8
        if (bits == 8) != (m_scales is not None) or (bits == 8) != (v_scales is not None):
            _refuse("m_scales and v_scales belong to moments in 8 bits")
        self.device_index = params[0].get_device()
        if self.device_index < 0:
            _refuse(f"tensors on {params[0].device}: a CUDA device is needed")
        table = (FtAdamWTensor * n)()
        for i in range(n):
            e = params[i].numel()
            runs = (e + 255) // 256
            for field, what, t, dtype, count in (("param", "params", params, pt, e), ("grad", "grads", grads, gt, e), ("m", "m", m, mt, e),
                                                 ("v", "v", v, mt, e), ("m_scale", "m_scales", m_scales, torch.float32, runs),
                                                 ("v_scale", "v_scales", v_scales, torch.float32, runs),
                                                 ("copy", "copies", copies, torch.bfloat16, e)):
                if t is not None and t[i] is not None:
                    setattr(table[i], field, _check_flat(f"{what}[{i}]", t[i], dtype, count, self.device_index))
            table[i].numel, table[i].weight_decay = e, decay[i]
        size = int(lib().ft_k_adamw_plan_bytes(table, n, param_dtype, grad_dtype, bits))
        if size == 0:
            _refuse("AdamWPlan: buffers that are missing, misaligned or overlap")
        self.host = np.zeros((size + 7) // 8, dtype=np.uint64)
        st = lib().ft_k_adamw_plan(table, n, param_dtype, grad_dtype, bits, self.host.ctypes.data, size)
        if st != FT_OK:
            raise ForgeStepError(st, "ft_k_adamw_plan")
        self.bytes = size
        self.device = torch.from_numpy(self.host.view(np.uint8)).to(params[0].device)
        self._host_address, self._device_address = self.host.ctypes.data, self.device.data_ptr()
        self._streams = {_stream_of(self.device_index)}  # those that torch's allocator knows to use the device's copy
        self.tensors = lists


def k_adamw(plan, lr, beta1, beta2, eps, step, lr_tensor=None, grad_scale=None, seed=0):
    """One AdamW step over the tensors of an AdamWPlan.  step: int64 tensor of one element, the number of this step, from 1 on;
    lr_tensor and grad_scale: fp32 tensors of one element (None: lr, 1); all three are read when the kernel runs.  seed: of the
    roundings of moments in 8 bits, with which eps is at least 2^-64."""
    torch = _torch or _import_torch()
    dev = _current_device(step)
    if plan.device_index != dev:
        _refuse(f"a plan of cuda:{plan.device_index}, current device cuda:{dev}")
    stream = _stream_of(dev)
    if stream not in plan._streams:  # a plan that is dropped while a step runs there keeps its memory until the step is through
        plan.device.record_stream(torch.cuda.current_stream(dev))
        plan._streams.add(stream)
    st = lib().ft_k_adamw(plan._host_address, plan._device_address, plan.bytes, lr, beta1, beta2, eps,
                          _check_flat("step", step, torch.int64, 1, dev),
                          _check_flat("lr_tensor", lr_tensor, torch.float32, 1, dev) if lr_tensor is not None else None,
                          _check_flat("grad_scale", grad_scale, torch.float32, 1, dev) if grad_scale is not None else None,
                          seed & 0xFFFFFFFFFFFFFFFF, stream)
    if st != FT_OK:
        raise ForgeStepError(st, "ft_k_adamw")
