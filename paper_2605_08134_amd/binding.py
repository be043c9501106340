"""ctypes binding of libdare.so: same names as the C ABI, argument marshalling only.

Tensors are torch tensors on the GPU (torch provides device memory and streams);
every computation happens in the library's HIP kernels.  There is no fallback:
if libdare.so is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
import struct

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG_DIR, "libdare.so")

DARE_OK, DARE_ERR_INVALID_ARG, DARE_ERR_UNSUPPORTED, DARE_ERR_OOM, DARE_ERR_HIP = range(5)
DARE_F32, DARE_BF16 = 0, 1
MODE_DENSE, MODE_KV, MODE_O, MODE_KVO = 0, 1, 2, 3
MODE_NAMES = {MODE_DENSE: "dense", MODE_KV: "kv", MODE_O: "o", MODE_KVO: "kvo"}

EXPORTS = (
    "dare_create", "dare_layer_step", "dare_destroy", "dare_last_error", "dare_version",
    "dare_static_init", "dare_layer_step_static",
    "dare_k_pack_weight", "dare_k_gemm", "dare_k_score", "dare_k_compact",
    "dare_k_attention", "dare_k_copy_rows",
    "dare_block_attach", "dare_block_step", "dare_k_gemm_rope", "dare_k_rope_table",
    "dare_k_norm", "dare_k_residual_add",
    "dare_set_threshold_rule", "dare_get_thresholds", "dare_drift_stats_enable", "dare_drift_stats_read",
    "dare_allocate_quantiles", "dare_policy_mode", "dare_k_quantile_mask", "dare_set_prefix",
    "dare_model_create", "dare_model_set_layer", "dare_model_set_io", "dare_model_set_rule",
    "dare_model_set_prefix", "dare_model_step", "dare_model_logits", "dare_model_layer",
    "dare_model_destroy", "dare_model_last_error",
    "dare_k_linear", "dare_k_rope", "dare_k_rope_freqs", "dare_k_attention_packed", "dare_k_attention_packed_workspace",
    "dare_k_norm_q8", "dare_k_linear_q8", "dare_k_logprobs", "dare_k_logprobs_workspace",
)
RULE_SCORE, RULE_QUANTILE = 0, 1
NORM_NONE, NORM_LAYER, NORM_RMS = 0, 1, 2
ACTIVATIONS = {None: 0, "silu": 1, "gelu": 2, "gelu_tanh": 3}
ROPE_LAYOUTS = {"half": 0, "pairs": 1}
ROPE_SCALINGS = {None: 0, "linear": 1, "base": 2, "turns": 3}
NORM_KINDS = {None: NORM_NONE, "layer": NORM_LAYER, "rms": NORM_RMS}


class DareConfig(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32),
        ("hidden", ctypes.c_int32),
        ("n_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("max_batch", ctypes.c_int32),
        ("max_seq", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("score_head", ctypes.c_int32),
        ("device", ctypes.c_int32),
        ("flags", ctypes.c_uint32),
    ]


class DareBlockConfig(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32),
        ("norm", ctypes.c_int32),
        ("eps", ctypes.c_float),
        ("rope_base", ctypes.c_float),
        ("residual", ctypes.c_int32),
    ]


class DareModelConfig(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32),
        ("n_layers", ctypes.c_int32), ("hidden", ctypes.c_int32), ("n_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("ffn", ctypes.c_int32), ("vocab", ctypes.c_int32),
        ("max_batch", ctypes.c_int32), ("max_seq", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("norm_eps", ctypes.c_float),
        ("rope_base", ctypes.c_float),
        ("device", ctypes.c_int32),
        ("flags", ctypes.c_uint32),
    ]


class DareError(RuntimeError):
    def __init__(self, status, text):
        super().__init__("libdare status %d: %s" % (status, text))
        self.status = status


_lib = None


def lib():
    """The loaded library (loaded on first use; raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError("libdare.so is not built: run `python -m paper_2605_08134_amd.build`")
    L = ctypes.CDLL(LIB_PATH)
    vp, i32, f32, u64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_uint64
    L.dare_create.argtypes = [ctypes.POINTER(DareConfig), vp, vp, vp, vp, vp, ctypes.POINTER(vp)]
    L.dare_create.restype = i32
    L.dare_layer_step.argtypes = [vp, i32, f32, i32, i32] + [vp] * 11
    L.dare_layer_step.restype = i32
    L.dare_static_init.argtypes = [i32]
    L.dare_static_init.restype = i32
    L.dare_layer_step_static.argtypes = [ctypes.POINTER(DareConfig), vp, vp, i32, f32, i32, i32] + [vp] * 11
    L.dare_layer_step_static.restype = i32
    L.dare_destroy.argtypes = [vp]
    L.dare_destroy.restype = i32
    L.dare_last_error.argtypes = [vp]
    L.dare_last_error.restype = ctypes.c_char_p
    L.dare_version.argtypes = []
    L.dare_version.restype = ctypes.c_char_p
    L.dare_k_pack_weight.argtypes = [i32, vp, i32, i32, vp, i32, vp]
    L.dare_k_pack_weight.restype = i32
    L.dare_k_gemm.argtypes = [i32, vp, i32, vp, i32, i32, i32, vp, vp, ctypes.POINTER(vp), i32, i32,
                              vp, i32, i32, ctypes.c_long, vp]
    L.dare_k_gemm.restype = i32
    L.dare_k_score.argtypes = [vp, i32, i32, i32, ctypes.c_long, vp, i32, f32, i32, vp, vp, vp]
    L.dare_k_score.restype = i32
    L.dare_k_compact.argtypes = [vp, i32, i32, vp, vp, vp, vp]
    L.dare_k_compact.restype = i32
    L.dare_k_attention.argtypes = [i32, vp, vp, vp, vp, i32, i32, i32, i32, vp, vp, vp]
    L.dare_k_attention.restype = i32
    L.dare_k_copy_rows.argtypes = [vp, vp, i32, i32, vp, vp, vp]
    L.dare_k_copy_rows.restype = i32
    L.dare_block_attach.argtypes = [vp, ctypes.POINTER(DareBlockConfig), vp, vp, vp]
    L.dare_block_attach.restype = i32
    L.dare_block_step.argtypes = [vp, i32, f32, i32, i32] + [vp] * 11
    L.dare_block_step.restype = i32
    L.dare_k_gemm_rope.argtypes = [i32, vp, i32, vp, i32, i32, i32, vp, vp, ctypes.POINTER(vp), i32, i32,
                                   vp, i32, vp, i32, i32, i32, vp]
    L.dare_k_gemm_rope.restype = i32
    L.dare_k_rope_table.argtypes = [vp, i32, i32, ctypes.c_double]
    L.dare_k_rope_table.restype = i32
    L.dare_k_norm.argtypes = [i32, i32, vp, vp, vp, f32, i32, i32, vp, vp]
    L.dare_k_norm.restype = i32
    L.dare_k_residual_add.argtypes = [i32, vp, vp, vp, ctypes.c_long, vp]
    L.dare_k_residual_add.restype = i32
    dbl_p = ctypes.POINTER(ctypes.c_double)
    L.dare_set_threshold_rule.argtypes = [vp, i32]
    L.dare_set_threshold_rule.restype = i32
    L.dare_get_thresholds.argtypes = [vp, vp, i32, vp]
    L.dare_get_thresholds.restype = i32
    L.dare_drift_stats_enable.argtypes = [vp, i32, vp]
    L.dare_drift_stats_enable.restype = i32
    L.dare_drift_stats_read.argtypes = [vp, dbl_p, ctypes.POINTER(ctypes.c_int64), vp]
    L.dare_drift_stats_read.restype = i32
    L.dare_allocate_quantiles.argtypes = [i32, dbl_p, ctypes.c_double, ctypes.c_double, dbl_p]
    L.dare_allocate_quantiles.restype = i32
    L.dare_policy_mode.argtypes = [i32] * 5
    L.dare_policy_mode.restype = i32
    L.dare_model_create.argtypes = [ctypes.POINTER(DareModelConfig), vp, ctypes.POINTER(vp)]
    L.dare_model_create.restype = i32
    L.dare_model_set_layer.argtypes = [vp, i32] + [vp] * 10
    L.dare_model_set_layer.restype = i32
    L.dare_model_set_io.argtypes = [vp, vp, vp, vp, vp]
    L.dare_model_set_io.restype = i32
    L.dare_model_set_rule.argtypes = [vp, i32]
    L.dare_model_set_rule.restype = i32
    L.dare_model_set_prefix.argtypes = [vp, i32]
    L.dare_model_set_prefix.restype = i32
    L.dare_model_step.argtypes = [vp, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_float), i32, i32,
                                  vp, vp, vp, vp, vp]
    L.dare_model_step.restype = i32
    L.dare_model_logits.argtypes = [vp, vp, vp, i32, vp, vp]
    L.dare_model_logits.restype = i32
    L.dare_model_layer.argtypes = [vp, i32]
    L.dare_model_layer.restype = vp
    L.dare_model_destroy.argtypes = [vp]
    L.dare_model_destroy.restype = i32
    L.dare_model_last_error.argtypes = [vp]
    L.dare_model_last_error.restype = ctypes.c_char_p
    L.dare_set_prefix.argtypes = [vp, i32]
    L.dare_set_prefix.restype = i32
    L.dare_k_quantile_mask.argtypes = [vp, i32, i32, f32, i32, vp, vp, vp, vp, vp]
    L.dare_k_quantile_mask.restype = i32
    lng = ctypes.c_long
    L.dare_k_logprobs.argtypes = [vp, vp, ctypes.c_size_t, vp]
    L.dare_k_logprobs.restype = i32
    L.dare_k_logprobs_workspace.argtypes = [vp, ctypes.POINTER(ctypes.c_size_t)]
    L.dare_k_logprobs_workspace.restype = i32
    for name in ("dare_k_norm_q8", "dare_k_linear_q8"):
        getattr(L, name).argtypes = [vp, vp]
        getattr(L, name).restype = i32
    L.dare_k_linear.argtypes = [i32, vp, lng, vp, i32, i32, i32, vp, i32, vp, lng, vp, lng, vp]
    L.dare_k_linear.restype = i32
    L.dare_k_rope.argtypes = [vp, vp]
    L.dare_k_rope.restype = i32
    L.dare_k_rope_freqs.argtypes = [vp, i32, ctypes.c_double, i32] + [ctypes.c_double] * 4
    L.dare_k_rope_freqs.restype = i32
    L.dare_k_attention_packed.argtypes = [vp, vp, ctypes.c_size_t, vp]
    L.dare_k_attention_packed.restype = i32
    L.dare_k_attention_packed_workspace.argtypes = [vp, ctypes.POINTER(ctypes.c_size_t)]
    L.dare_k_attention_packed_workspace.restype = i32
    _lib = L
    return L


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    assert t.is_contiguous(), "tensor must be contiguous"
    return t.data_ptr()


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    import torch
    # the handle alone where torch has it: the Stream object around it takes 2.5 us of a call of 24
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    return raw(torch.cuda.current_device())


def _torch_dtype(dtype):
    import torch
    return torch.bfloat16 if dtype == DARE_BF16 else torch.float32


def _check(st, ctx=None):
    if st != DARE_OK:
        msg = lib().dare_last_error(ctx)
        raise DareError(st, msg.decode() if msg else "")


def dare_version():
    return lib().dare_version().decode()


STATIC_MAX_ROW_BYTES = 8 << 20      # DARE_STATIC_MAX_ROW_BYTES
STATIC_MAX_SCORE_ELEMS = 1 << 20    # DARE_STATIC_MAX_SCORE_ELEMS


def dare_static_init(device=0):
    _check(lib().dare_static_init(device), None)


def dare_layer_step_static(wqkv_t, wo_t, n_heads, mode, threshold, hidden, q_prev, k_cache, v_cache, o_cache, out,
                           reuse_mask, sel_idx=None, sel_count=None, scores=None, score_head=0, stream=None):
    """dare_layer_step_static: the layer step without a context and without any allocation.
    wqkv_t [3d, d] and wo_t [d, d] are the packed weights (dare_k_pack_weight)."""
    import torch
    batch, seq, d = hidden.shape
    dtype = DARE_BF16 if hidden.dtype == torch.bfloat16 else DARE_F32
    cfg = DareConfig(ctypes.sizeof(DareConfig), d, n_heads, d // n_heads, batch, seq, dtype, score_head,
                     hidden.device.index or 0, 0)
    st = lib().dare_layer_step_static(ctypes.byref(cfg), _ptr(wqkv_t), _ptr(wo_t), mode, threshold, batch, seq,
                                      _ptr(hidden), _ptr(q_prev), _ptr(k_cache), _ptr(v_cache), _ptr(o_cache),
                                      _ptr(out), _ptr(reuse_mask), _ptr(sel_idx), _ptr(sel_count), _ptr(scores),
                                      _stream(stream))
    _check(st, None)


class DareLayer:
    """dare_create / dare_layer_step / dare_destroy for one layer's weights."""

    @classmethod
    def view(cls, ctx_ptr, device):
        """A non-owning handle on a context that something else owns (a model's layer)."""
        self = cls.__new__(cls)
        self._ctx = ctypes.c_void_p(ctx_ptr)
        self.device = device
        self._borrowed = True
        return self

    def __init__(self, wq, wk, wv, wo, n_heads, max_batch, max_seq, score_head=0, stream=None):
        import torch
        d = wq.shape[0]
        dtype = DARE_BF16 if wq.dtype == torch.bfloat16 else DARE_F32
        for w in (wq, wk, wv, wo):
            assert w.is_cuda and w.shape == (d, d) and w.dtype == wq.dtype
        self.cfg = DareConfig(ctypes.sizeof(DareConfig), d, n_heads, d // n_heads, max_batch, max_seq,
                              dtype, score_head, wq.device.index or 0, 0)
        self.dtype = dtype
        self.hidden, self.n_heads, self.head_dim = d, n_heads, d // n_heads
        self.score_width = d if score_head < 0 else self.head_dim
        self.device = wq.device
        self._ctx = ctypes.c_void_p()
        st = lib().dare_create(ctypes.byref(self.cfg), _ptr(wq), _ptr(wk), _ptr(wv), _ptr(wo),
                               _stream(stream), ctypes.byref(self._ctx))
        _check(st, None)

    def new_state(self, batch, seq):
        """Zeroed caches for dare_layer_step (a DENSE step fills them)."""
        import torch
        td = _torch_dtype(self.dtype)
        z = lambda *s, dt=td: torch.zeros(*s, dtype=dt, device=self.device)
        return {
            "q_prev": z(batch, seq, self.score_width, dt=torch.float32),
            "k_cache": z(batch, seq, self.hidden),
            "v_cache": z(batch, seq, self.hidden),
            "o_cache": z(batch, seq, self.hidden),
        }

    def layer_step(self, mode, threshold, hidden, q_prev, k_cache, v_cache, o_cache, out,
                   reuse_mask, sel_idx=None, sel_count=None, scores=None, stream=None):
        batch, seq, _ = hidden.shape
        st = lib().dare_layer_step(self._ctx, mode, threshold, batch, seq, _ptr(hidden), _ptr(q_prev),
                                   _ptr(k_cache), _ptr(v_cache), _ptr(o_cache), _ptr(out),
                                   _ptr(reuse_mask), _ptr(sel_idx), _ptr(sel_count), _ptr(scores),
                                   _stream(stream))
        _check(st, self._ctx)

    def block_attach(self, norm=None, gain=None, bias=None, eps=1e-5, rope_base=0.0, residual=True,
                     stream=None):
        """dare_block_attach: norm is None, "layer" or "rms"."""
        cfg = DareBlockConfig(ctypes.sizeof(DareBlockConfig), NORM_KINDS[norm], eps, rope_base,
                              int(bool(residual)))
        st = lib().dare_block_attach(self._ctx, ctypes.byref(cfg), _ptr(gain), _ptr(bias), _stream(stream))
        _check(st, self._ctx)

    def block_step(self, mode, threshold, x, q_prev, k_cache, v_cache, o_cache, out,
                   reuse_mask, sel_idx=None, sel_count=None, scores=None, stream=None):
        batch, seq, _ = x.shape
        st = lib().dare_block_step(self._ctx, mode, threshold, batch, seq, _ptr(x), _ptr(q_prev),
                                   _ptr(k_cache), _ptr(v_cache), _ptr(o_cache), _ptr(out),
                                   _ptr(reuse_mask), _ptr(sel_idx), _ptr(sel_count), _ptr(scores),
                                   _stream(stream))
        _check(st, self._ctx)

    def set_prefix(self, prefix_len):
        _check(lib().dare_set_prefix(self._ctx, prefix_len), self._ctx)

    def set_threshold_rule(self, rule):
        _check(lib().dare_set_threshold_rule(self._ctx, rule), self._ctx)

    def thresholds(self, batch, stream=None):
        """The per-sequence thresholds of the last quantile step (float32 tensor [batch])."""
        import torch
        out = torch.empty(batch, dtype=torch.float32, device=self.device)
        _check(lib().dare_get_thresholds(self._ctx, _ptr(out), batch, _stream(stream)), self._ctx)
        return out

    def drift_stats_enable(self, on=True, stream=None):
        _check(lib().dare_drift_stats_enable(self._ctx, int(bool(on)), _stream(stream)), self._ctx)

    def drift_stats_read(self, stream=None):
        mean, count = ctypes.c_double(0.0), ctypes.c_int64(0)
        _check(lib().dare_drift_stats_read(self._ctx, ctypes.byref(mean), ctypes.byref(count),
                                           _stream(stream)), self._ctx)
        return mean.value, count.value

    def destroy(self):
        if self._ctx and not getattr(self, "_borrowed", False):
            lib().dare_destroy(self._ctx)
        self._ctx = ctypes.c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


class DareModel:
    """dare_model_*: a masked-diffusion model of DARE layers.  Weights are torch tensors on
    the GPU; they are copied at the set_* calls."""

    def __init__(self, n_layers, hidden, n_heads, ffn, vocab, max_batch, max_seq, dtype, norm_eps=1e-5,
                 rope_base=10000.0, device=None, stream=None):
        import torch
        self.device = device or torch.device("cuda", torch.cuda.current_device())
        self.dtype = dtype
        self.cfg = DareModelConfig(ctypes.sizeof(DareModelConfig), n_layers, hidden, n_heads, hidden // n_heads,
                                   ffn, vocab, max_batch, max_seq, dtype, norm_eps, rope_base,
                                   self.device.index or 0, 0)
        self._m = ctypes.c_void_p()
        st = lib().dare_model_create(ctypes.byref(self.cfg), _stream(stream), ctypes.byref(self._m))
        self._check(st, created=False)

    def _check(self, st, created=True):
        if st != DARE_OK:
            msg = lib().dare_model_last_error(self._m if created else None)
            raise DareError(st, msg.decode() if msg else "")

    def set_layer(self, layer, attn_gain, wq, wk, wv, wo, ffn_gain, w_gate, w_up, w_down, stream=None):
        self._check(lib().dare_model_set_layer(self._m, layer, _ptr(attn_gain), _ptr(wq), _ptr(wk), _ptr(wv),
                                               _ptr(wo), _ptr(ffn_gain), _ptr(w_gate), _ptr(w_up), _ptr(w_down),
                                               _stream(stream)))

    def set_io(self, embed, final_gain, head=None, stream=None):
        self._check(lib().dare_model_set_io(self._m, _ptr(embed), _ptr(final_gain), _ptr(head), _stream(stream)))

    def set_rule(self, rule):
        self._check(lib().dare_model_set_rule(self._m, rule))

    def set_prefix(self, prefix_len):
        self._check(lib().dare_model_set_prefix(self._m, prefix_len))

    def step(self, modes, thresholds, ids, hidden_out=None, refreshed=None, trace=None, stream=None):
        L = self.cfg.n_layers
        batch, seq = ids.shape
        if isinstance(modes, int):
            modes = [modes] * L
        if isinstance(thresholds, (int, float)):
            thresholds = [float(thresholds)] * L
        assert len(modes) == L and len(thresholds) == L
        ma = (ctypes.c_int32 * L)(*modes)
        ta = (ctypes.c_float * L)(*thresholds)
        self._check(lib().dare_model_step(self._m, ma, ta, batch, seq, _ptr(ids), _ptr(hidden_out),
                                          _ptr(refreshed), _ptr(trace), _stream(stream)))

    def logits(self, hidden, rows, stream=None):
        import torch
        out = torch.empty((rows.numel(), self.cfg.vocab), dtype=_torch_dtype(self.dtype), device=self.device)
        self._check(lib().dare_model_logits(self._m, _ptr(hidden), _ptr(rows), rows.numel(), _ptr(out),
                                            _stream(stream)))
        return out

    def layer(self, index):
        ptr = lib().dare_model_layer(self._m, index)
        if not ptr:
            raise IndexError("no such layer, or its weights are not set")
        return DareLayer.view(ptr, self.device)

    def destroy(self):
        if self._m:
            lib().dare_model_destroy(self._m)
            self._m = ctypes.c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def dare_allocate_quantiles(s_layers, phi_bar, eps):
    n = len(s_layers)
    src = (ctypes.c_double * n)(*[float(v) for v in s_layers])
    out = (ctypes.c_double * n)()
    _check(lib().dare_allocate_quantiles(n, src, float(phi_bar), float(eps), out))
    return list(out)


def dare_policy_mode(mode, layer, step, skip_layers=0, refresh_interval=0):
    return lib().dare_policy_mode(mode, layer, step, skip_layers, refresh_interval)


# ---- kernel-level entry points ---------------------------------------------------------

def dare_k_pack_weight(w, stream=None):
    import torch
    k, n = w.shape
    wt = torch.empty((n, k), dtype=w.dtype, device=w.device)
    dtype = DARE_BF16 if w.dtype == torch.bfloat16 else DARE_F32
    _check(lib().dare_k_pack_weight(dtype, _ptr(w), k, n, _ptr(wt), k, _stream(stream)))
    return wt


def dare_k_gemm(a, wt, outs, seg_n, idx=None, m_dev=None, m_max=None, c32=None, k_parts=1, stream=None):
    import torch
    n, k = wt.shape
    dtype = DARE_BF16 if a.dtype == torch.bfloat16 else DARE_F32
    arr = (ctypes.c_void_p * 3)(*[_ptr(o) for o in list(outs) + [None] * (3 - len(outs))])
    ldc = next(o for o in outs if o is not None).shape[-1] if any(o is not None for o in outs) else seg_n
    if m_max is None:
        m_max = a.shape[0] if idx is None else idx.shape[0]
    _check(lib().dare_k_gemm(dtype, _ptr(a), a.shape[-1], _ptr(wt), n, k, m_max, _ptr(idx), _ptr(m_dev),
                             arr, ldc, seg_n, _ptr(c32), 0 if c32 is None else c32.shape[-1],
                             k_parts, 0 if c32 is None else m_max * c32.shape[-1], _stream(stream)))


def dare_k_quantile_mask(scores, phi, mask, tau_out=None, force_refresh=False, stat_sum=None,
                         stat_count=None, stream=None):
    batch, seq = scores.shape
    _check(lib().dare_k_quantile_mask(_ptr(scores), batch, seq, phi, int(force_refresh), _ptr(tau_out),
                                      _ptr(mask), _ptr(stat_sum), _ptr(stat_count), _stream(stream)))


def dare_k_gemm_rope(a, wt, outs, seg_n, rope_table, rope_cols, head_dim, seq, idx=None, m_dev=None,
                     m_max=None, c32=None, stream=None):
    import torch
    n, k = wt.shape
    dtype = DARE_BF16 if a.dtype == torch.bfloat16 else DARE_F32
    arr = (ctypes.c_void_p * 3)(*[_ptr(o) for o in list(outs) + [None] * (3 - len(outs))])
    ldc = next(o for o in outs if o is not None).shape[-1]
    if m_max is None:
        m_max = a.shape[0] if idx is None else idx.shape[0]
    _check(lib().dare_k_gemm_rope(dtype, _ptr(a), a.shape[-1], _ptr(wt), n, k, m_max, _ptr(idx),
                                  _ptr(m_dev), arr, ldc, seg_n, _ptr(c32),
                                  0 if c32 is None else c32.shape[-1], _ptr(rope_table), rope_cols,
                                  head_dim, seq, _stream(stream)))


def dare_k_rope_table(n_pos, head_dim, base, device="cuda"):
    import torch
    table = torch.empty((n_pos, head_dim // 2, 2), dtype=torch.float32, device=device)
    _check(lib().dare_k_rope_table(_ptr(table), n_pos, head_dim, float(base)))
    return table


def dare_k_norm(kind, x, gain, bias, eps, out, stream=None):
    import torch
    dtype = DARE_BF16 if x.dtype == torch.bfloat16 else DARE_F32
    d = x.shape[-1]
    _check(lib().dare_k_norm(dtype, NORM_KINDS[kind], _ptr(x), _ptr(gain), _ptr(bias), eps,
                             x.numel() // d, d, _ptr(out), _stream(stream)))


def dare_k_residual_add(x, o, out, stream=None):
    import torch
    dtype = DARE_BF16 if x.dtype == torch.bfloat16 else DARE_F32
    _check(lib().dare_k_residual_add(dtype, _ptr(x), _ptr(o), _ptr(out), x.numel(), _stream(stream)))


def dare_k_score(q_new, q_prev, threshold, force_refresh, scores, mask, n_parts=1, stream=None):
    n_tokens, width = q_prev.shape[0], q_prev.shape[-1]
    _check(lib().dare_k_score(_ptr(q_new), q_new.shape[-1], width, n_parts, n_tokens * q_new.shape[-1],
                              _ptr(q_prev), n_tokens, threshold,
                              int(force_refresh), _ptr(scores), _ptr(mask), _stream(stream)))


def dare_k_compact(mask, batch, seq, sel_idx, sel_count, sel_off, stream=None):
    _check(lib().dare_k_compact(_ptr(mask), batch, seq, _ptr(sel_idx), _ptr(sel_count), _ptr(sel_off),
                                _stream(stream)))


def dare_k_attention(q, k, v, out, batch, seq, n_heads, head_dim, idx=None, sel_off=None, stream=None):
    import torch
    dtype = DARE_BF16 if q.dtype == torch.bfloat16 else DARE_F32
    _check(lib().dare_k_attention(dtype, _ptr(q), _ptr(k), _ptr(v), _ptr(out), batch, seq, n_heads,
                                  head_dim, _ptr(idx), _ptr(sel_off), _stream(stream)))


def dare_k_copy_rows(src, dst, idx=None, m_dev=None, stream=None):
    n_rows = src.shape[0]
    row_bytes = src.shape[-1] * src.element_size()
    _check(lib().dare_k_copy_rows(_ptr(src), _ptr(dst), n_rows, row_bytes, _ptr(idx), _ptr(m_dev),
                                  _stream(stream)))


# ---- decoder layers with shared key heads ------------------------------------------------
# (A call takes the host about as long as a small kernel the GPU, so every property of a tensor is asked for once, and what
# has many arguments goes over as the bytes of its struct.)

# dare_rope_call: struct_size, dtype, layout, n_tokens, head_dim, rot_dim, n_heads, n_kv_heads, out_rows, magnitude; pos, freqs,
# rows; q, k, v; q_out, k_out, v_out; ldq, ldk, ldv, ldqo, ldko, ldvo
_ROPE_CALL = struct.Struct("@I8ifPPP3P3P6q")
# dare_packed_call: struct_size, dtype, batch, total_q, k_rows, max_q, max_k, n_heads, n_kv_heads, head_dim, causal_block,
# scale; ldq, ldk, ldv, ldo; q, k, v, out, q_off, k_begin, k_end
_PACKED_CALL = struct.Struct("@I10if4q7P")


def _pack(layout, *fields):
    try:
        return layout.pack(layout.size, *fields)
    except struct.error as e:
        raise ValueError("an argument does not fit its type: %s" % e) from None


def _gpu_of(like):
    """Device index and dtype code of the tensor that the others have to match."""
    import torch
    device, dt = like.get_device(), like.dtype
    if device < 0:
        raise ValueError("tensors must be on the GPU")
    if dt is torch.bfloat16:
        return device, dt, DARE_BF16
    if dt is torch.float32:
        return device, dt, DARE_F32
    raise ValueError("dtype must be bfloat16 or float32, not %s" % dt)


def _wrong(name, t, dt, device, wanted):
    raise ValueError("%s must be %s of %s on cuda:%d, is %s of %s on %s" % (name, wanted, dt, device, tuple(t.shape), t.dtype,
                                                                       t.device))


def _ld(name, t, shape, dt, device):
    """Row distance of a [tokens, heads, head_dim] tensor of that shape whose heads lie one behind the other."""
    if t.shape != shape or t.dtype is not dt or t.get_device() != device:
        _wrong(name, t, dt, device, list(shape))
    ld, between, inside = t.stride()
    rows, h, d = shape
    if (inside != 1 and d > 1 or between != d and h > 1) and rows * h * d:
        raise ValueError("the heads of a row of %s must lie one behind the other" % name)
    return ld if rows > 1 else h * d


def _matrix(name, t, dt, device, rows, cols):
    """Pointer and row distance of a [rows, cols] tensor with contiguous rows."""
    if t.shape != (rows, cols) or t.dtype is not dt or t.get_device() != device:
        _wrong(name, t, dt, device, "[%s, %s]" % (rows, cols))
    ld, inside = t.stride()
    if inside != 1 and cols > 1 and rows:
        raise ValueError("the rows of %s must be contiguous" % name)
    return t.data_ptr(), ld if rows > 1 else cols


def _vector(name, t, dt, device, n):
    if t.shape != (n,) or t.dtype is not dt or t.get_device() != device or not t.is_contiguous():
        _wrong(name, t, dt, device, "a contiguous [%s]" % n)
    return t.data_ptr()


def _enqueue(device, stream, fn, *args):
    """fn(*args, stream) with `device` as the current one."""
    import torch
    if stream is not None and stream.device.index != device:
        raise ValueError("the stream belongs to %s, the tensors to cuda:%d" % (stream.device, device))
    if device == torch._C._cuda_getDevice():
        st = fn(*args, torch._C._cuda_getCurrentRawStream(device) if stream is None else stream.cuda_stream)
    else:
        with torch.cuda.device(device):
            st = fn(*args, _stream(stream))
    if st:
        _check(st)


def dare_k_linear(a, wt, out, bias=None, act=None, residual=None, stream=None):
    """out = act(a W + bias) + residual.  a [m, k], out and residual [m, n] with contiguous rows, wt [n, k] packed
    (dare_k_pack_weight), act None, "silu", "gelu" or "gelu_tanh"; out may be residual."""
    device, dt, code = _gpu_of(a)
    if wt.dim() != 2 or a.dim() != 2 or act not in ACTIVATIONS:
        raise ValueError("a and wt must be matrices, act one of %s" % list(ACTIVATIONS))
    n, k = wt.shape
    m = a.shape[0]
    pa, lda = _matrix("a", a, dt, device, m, k)
    po, ldo = _matrix("out", out, dt, device, m, n)
    pr, ldr = (None, 0) if residual is None else _matrix("residual", residual, dt, device, m, n)
    pw, ldw = _matrix("wt", wt, dt, device, n, k)
    if ldw != k:
        raise ValueError("wt must be contiguous")
    pb = None if bias is None else _vector("bias", bias, dt, device, n)
    _enqueue(device, stream, lib().dare_k_linear, code, pa, lda, pw, n, k, m, pb, ACTIVATIONS[act], pr, ldr, po, ldo)


def dare_k_rope_freqs(rot_dim, base=10000.0, scaling=None, factor=1.0, context=8192, low=1.0, high=4.0, device="cuda"):
    """Frequencies (float64 [rot_dim / 2] on the device) for dare_k_rope; scaling None, "linear", "base" or "turns"."""
    import torch
    if scaling not in ROPE_SCALINGS:
        raise ValueError("scaling must be one of %s" % list(ROPE_SCALINGS))
    freqs = torch.empty(max(rot_dim, 2) // 2, dtype=torch.float64, device=device)
    with torch.cuda.device(freqs.device):
        torch.cuda.current_stream().synchronize()  # (the memory may have been that of a tensor still in use there)
        _check(lib().dare_k_rope_freqs(_ptr(freqs), rot_dim, float(base), ROPE_SCALINGS[scaling], float(factor),
                                       float(context), float(low), float(high)))
    return freqs


def dare_k_rope(pos, freqs, layout="half", q=None, q_out=None, k=None, k_out=None, v=None, v_out=None, rows=None,
                magnitude=1.0, stream=None):
    """Rotary embedding of q and k [tokens, heads, head_dim] by the positions pos (int32 [tokens]) into q_out and k_out; v is
    copied into v_out.  rows (int32 [tokens]): the rows of k_out and v_out, for instance of a cache, that the tokens go
    to.  layout "half" or "pairs"."""
    import torch
    first = q if q is not None else k if k is not None else v
    if first is None or first.dim() != 3 or layout not in ROPE_LAYOUTS:
        raise ValueError("q, k or v must be [tokens, heads, head_dim], layout one of %s" % list(ROPE_LAYOUTS))
    if (q is None) != (q_out is None) or (k is None) != (k_out is None) or (v is None) != (v_out is None):
        raise ValueError("an input and its output go together")
    device, dt, code = _gpu_of(first)
    shape = first.shape
    n, h, d = shape
    pq = pqo = pk = pko = pv = pvo = None
    ldq = ldqo = ldk = ldko = ldv = ldvo = kv = out_rows = 0
    if q is not None:
        pq, ldq = q.data_ptr(), _ld("q", q, shape, dt, device)
        pqo, ldqo = q_out.data_ptr(), _ld("q_out", q_out, shape, dt, device)
    if k is not None or v is not None:
        one, one_out = (k, k_out) if k is not None else (v, v_out)
        shape = out_shape = one.shape
        if len(shape) != 3 or shape[0] != n or shape[2] != d:
            raise ValueError("k and v must be [%d, heads, %d], not %s" % (n, d, tuple(shape)))
        kv = shape[1]
        if rows is not None:
            out_shape = one_out.shape
            if len(out_shape) != 3 or out_shape[1] != kv or out_shape[2] != d:
                raise ValueError("k_out and v_out must be [rows, %d, %d], not %s" % (kv, d, tuple(out_shape)))
            out_rows = out_shape[0]
        if k is not None:
            pk, ldk = k.data_ptr(), _ld("k", k, shape, dt, device)
            pko, ldko = k_out.data_ptr(), _ld("k_out", k_out, out_shape, dt, device)
        if v is not None:
            pv, ldv = v.data_ptr(), _ld("v", v, shape, dt, device)
            pvo, ldvo = v_out.data_ptr(), _ld("v_out", v_out, out_shape, dt, device)
    pr = 0 if rows is None else _vector("rows", rows, torch.int32, device, n)
    if freqs.dim() != 1:
        raise ValueError("freqs must be a vector, not %s" % (tuple(freqs.shape),))
    half = freqs.shape[0]
    call = _pack(_ROPE_CALL, code, ROPE_LAYOUTS[layout], n, d, 2 * half, 0 if q is None else h, kv, out_rows, magnitude,
                 _vector("pos", pos, torch.int32, device, n), _vector("freqs", freqs, torch.float64, device, half), pr,
                 pq or 0, pk or 0, pv or 0, pqo or 0, pko or 0, pvo or 0, ldq, ldk, ldv, ldqo, ldko, ldvo)
    _enqueue(device, stream, lib().dare_k_rope, call)


def dare_k_attention_packed(q, k, v, out, q_off, k_begin, k_end, max_q, max_k, causal_block=0, scale=None,
                            workspace=None, stream=None):
    """Attention of packed sequences.  q, out [total_q, n_heads, head_dim], k, v [k_rows, n_kv_heads, head_dim] (parts of one
    buffer, or a cache); int32 q_off [batch + 1], k_begin and k_end [batch].  causal_block 0: every token sees all keys of its
    sequence, b: those up to the end of its block of b positions (1: causal).  scale: 1 / sqrt(head_dim).  max_q, max_k: the largest
    numbers of query tokens and keys of a sequence.  workspace: a uint8 tensor of dare_k_attention_packed_workspace() bytes to
    use instead of one of the call's own."""
    import torch
    device, dt, code = _gpu_of(q)
    shape, kshape, i32 = q.shape, k.shape, torch.int32
    if len(shape) != 3 or len(kshape) != 3 or shape[2] != kshape[2]:
        raise ValueError("q and k must be [tokens, heads, head_dim], not %s and %s" % (tuple(shape), tuple(kshape)))
    total, h, d = shape
    if k_begin.dim() != 1:
        raise ValueError("k_begin must be a vector, not %s" % (tuple(k_begin.shape),))
    batch = k_begin.shape[0]
    call = _pack(_PACKED_CALL, code, batch, total, kshape[0], max_q, max_k, h, kshape[1], d, causal_block,
                 d ** -0.5 if scale is None else scale,
                 _ld("q", q, shape, dt, device), _ld("k", k, kshape, dt, device), _ld("v", v, kshape, dt, device),
                 _ld("out", out, shape, dt, device), q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
                 _vector("q_off", q_off, i32, device, batch + 1), _vector("k_begin", k_begin, i32, device, batch),
                 _vector("k_end", k_end, i32, device, batch))
    if workspace is None:
        need = ctypes.c_size_t()
        st = lib().dare_k_attention_packed_workspace(call, need)
        if st:
            _check(st)
        if need.value:
            workspace = _scratch(need.value, q.device, stream)
    elif workspace.get_device() != device or not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous and on cuda:%d" % device)
    pw, size = (None, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() * workspace.element_size())
    _enqueue(device, stream, lib().dare_k_attention_packed, call, pw, size)


def dare_k_attention_packed_workspace(dtype, batch, total_q, max_q, max_k, n_heads, n_kv_heads, head_dim):
    """Bytes of the workspace of a dare_k_attention_packed call of these sizes (0: none)."""
    wq, wk = n_heads * head_dim, n_kv_heads * head_dim
    call = _pack(_PACKED_CALL, dtype, batch, total_q, 0, max_q, max_k, n_heads, n_kv_heads, head_dim, 0, 1.0, wq, wk, wk, wq,
                 *[0] * 7)
    need = ctypes.c_size_t()
    _check(lib().dare_k_attention_packed_workspace(call, ctypes.byref(need)))
    return need.value


# ---- 8-bit codes, and the output end of a step --------------------------------------------

# dare_norm_q8_call: struct_size, dtype, kind, n_rows, d; eps; ldx, ldo, ldxo, ldc; x, o, gain, bias, x_out, codes, scales
_NORM_Q8_CALL = struct.Struct("@I4id4q7P")
# dare_linear_q8_call: struct_size, dtype, m, n, k, act; lda, ldr, ldo; a, row_scale, wt, col_scale, bias, residual, out
_LINEAR_Q8_CALL = struct.Struct("@I5i3q7P")
# dare_logprobs_call: struct_size, dtype, n_rows, vocab, top, scale; ld; logits, tokens, logprobs, entropy, top_ids, top_logprobs
_LOGPROBS_CALL = struct.Struct("@I4ifq6P")


def dare_k_norm_q8(kind, x, codes, scales, o=None, x_out=None, gain=None, bias=None, eps=1e-5, stream=None):
    """Rows of s = x + o (stored in x_out) or of their norm as 8-bit codes with a scale each: codes[t] * scales[t] stands for the
    row.  kind None, "layer" or "rms"; x, o, x_out [rows, d], codes int8 [rows, d] with contiguous rows, scales float32 [rows], gain and
    bias [d].  x_out may be x or o.  Codes of a weight: kind None of the packed one (dare_k_pack_weight), a scale per column."""
    import torch
    if x.dim() != 2 or kind not in NORM_KINDS:
        raise ValueError("x must be a matrix, kind one of %s" % list(NORM_KINDS))
    device, dt, code = _gpu_of(x)
    rows, d = x.shape
    px, ldx = _matrix("x", x, dt, device, rows, d)
    po, ldo = (0, 0) if o is None else _matrix("o", o, dt, device, rows, d)
    ps, lds = (0, 0) if x_out is None else _matrix("x_out", x_out, dt, device, rows, d)
    pc, ldc = _matrix("codes", codes, torch.int8, device, rows, d)
    call = _pack(_NORM_Q8_CALL, code, NORM_KINDS[kind], rows, d, eps, ldx, ldo, lds, ldc, px, po,
                 0 if gain is None else _vector("gain", gain, dt, device, d),
                 0 if bias is None else _vector("bias", bias, dt, device, d), ps, pc,
                 _vector("scales", scales, torch.float32, device, rows))
    _enqueue(device, stream, lib().dare_k_norm_q8, call)


def dare_k_linear_q8(a, a_scales, wt, wt_scales, out, bias=None, act=None, residual=None, stream=None):
    """out = act(a_scales wt_scales (a W) + bias) + residual.  a int8 [m, k] with contiguous rows, wt int8 [n, k] (the codes of a packed
    weight), a_scales float32 [m], wt_scales float32 [n]; bias [n], residual and out [m, n] bfloat16 or float32; act None, "silu", "gelu" or
    "gelu_tanh"; out may be residual."""
    import torch
    device, dt, code = _gpu_of(out)
    if wt.dim() != 2 or a.dim() != 2 or act not in ACTIVATIONS:
        raise ValueError("a and wt must be matrices, act one of %s" % list(ACTIVATIONS))
    n, k = wt.shape
    m = a.shape[0]
    i8, f32 = torch.int8, torch.float32
    pa, lda = _matrix("a", a, i8, device, m, k)
    pw, ldw = _matrix("wt", wt, i8, device, n, k)
    if ldw != k:
        raise ValueError("wt must be contiguous")
    po, ldo = _matrix("out", out, dt, device, m, n)
    pr, ldr = (0, 0) if residual is None else _matrix("residual", residual, dt, device, m, n)
    call = _pack(_LINEAR_Q8_CALL, code, m, n, k, ACTIVATIONS[act], lda, ldr, ldo, pa, _vector("a_scales", a_scales, f32, device, m), pw,
                 _vector("wt_scales", wt_scales, f32, device, n), 0 if bias is None else _vector("bias", bias, dt, device, n), pr, po)
    _enqueue(device, stream, lib().dare_k_linear_q8, call)


def dare_k_logprobs(logits, tokens=None, logprobs=None, entropy=None, top_ids=None, top_logprobs=None, scale=1.0,
                    workspace=None, stream=None):
    """Of p = softmax(scale logits) per row of logits [rows, vocab]: logprobs = log p of tokens (int32 [rows]), the entropy, and ids and
    log-probabilities of the largest (top_ids int32, top_logprobs [rows, top], top up to 32; equal logits by their ids).  What is not
    wanted is None; outputs are float32 [rows].  workspace: a uint8 tensor of dare_k_logprobs_workspace() bytes to use instead of one of the
    call's own."""
    import torch
    if logits.dim() != 2 or (top_ids is None) != (top_logprobs is None) or (top_ids is not None and top_ids.dim() != 2):
        raise ValueError("logits must be a matrix, top_ids and top_logprobs both matrices or None")
    device, dt, code = _gpu_of(logits)
    rows, vocab = logits.shape
    px, ld = _matrix("logits", logits, dt, device, rows, vocab)
    i32, f32 = torch.int32, torch.float32
    top = 0 if top_ids is None else top_ids.shape[1]
    pi = pt = 0
    if top_ids is not None:
        pi, _ = _matrix("top_ids", top_ids, i32, device, rows, top)
        pt, _ = _matrix("top_logprobs", top_logprobs, f32, device, rows, top)
        if not (top_ids.is_contiguous() and top_logprobs.is_contiguous()):
            raise ValueError("top_ids and top_logprobs must be contiguous")
    call = _pack(_LOGPROBS_CALL, code, rows, vocab, top, scale, ld, px, 0 if tokens is None else _vector("tokens", tokens, i32, device, rows),
                 0 if logprobs is None else _vector("logprobs", logprobs, f32, device, rows),
                 0 if entropy is None else _vector("entropy", entropy, f32, device, rows), pi, pt)
    if workspace is None:
        need = ctypes.c_size_t()
        st = lib().dare_k_logprobs_workspace(call, need)
        if st:
            _check(st)
        if need.value:
            workspace = _scratch(need.value, logits.device, stream)
    elif workspace.get_device() != device or not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous and on cuda:%d" % device)
    pw, size = (None, 0) if workspace is None else (workspace.data_ptr(), workspace.numel() * workspace.element_size())
    _enqueue(device, stream, lib().dare_k_logprobs, call, pw, size)


def dare_k_logprobs_workspace(dtype, rows, vocab, top):
    """Bytes of the workspace of a dare_k_logprobs call of these sizes (0: none)."""
    need = ctypes.c_size_t()
    _check(lib().dare_k_logprobs_workspace(_pack(_LOGPROBS_CALL, dtype, rows, vocab, top, 1.0, vocab, *[0] * 6), ctypes.byref(need)))
    return need.value


def _scratch(n_bytes, device, stream):
    """Memory for one call, from the pool of the stream that the call runs on: what is freed there is used again behind
    the call, not beside it."""
    import torch
    if stream is None:
        return torch.empty(n_bytes, dtype=torch.uint8, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(n_bytes, dtype=torch.uint8, device=device)


# ---- benchmark aids (libdare_bench.so, include/dare_bench.h) ------------------------------

BENCH_LIB_PATH = os.path.join(PKG_DIR, "libdare_bench.so")
BENCH_EXPORTS = ("dare_bench_mfma_loop", "dare_bench_stream")
_bench_lib = None


def bench_lib():
    global _bench_lib
    if _bench_lib is None:
        if not os.path.exists(BENCH_LIB_PATH):
            raise RuntimeError("libdare_bench.so is not built: run `python -m paper_2605_08134_amd.build`")
        L = ctypes.CDLL(BENCH_LIB_PATH)
        L.dare_bench_mfma_loop.argtypes = [ctypes.c_int] * 3 + [ctypes.c_void_p, ctypes.POINTER(ctypes.c_double),
                                                                ctypes.c_void_p]
        L.dare_bench_mfma_loop.restype = ctypes.c_int
        L.dare_bench_stream.argtypes = [ctypes.c_int, ctypes.c_ulonglong, ctypes.c_int, ctypes.c_void_p,
                                        ctypes.c_void_p, ctypes.c_void_p]
        L.dare_bench_stream.restype = ctypes.c_int
        _bench_lib = L
    return _bench_lib


def dare_bench_stream(n_blocks, bytes_per_block, depth, src, stream=None):
    """Enqueue the one-workgroup-per-CU stream over src (a device tensor of at least
    n_blocks * bytes_per_block bytes)."""
    if src.numel() * src.element_size() < n_blocks * bytes_per_block:
        raise ValueError("source buffer too small")
    st = bench_lib().dare_bench_stream(n_blocks, bytes_per_block, depth, _ptr(src), None, _stream(stream))
    if st != 0:
        raise DareError(st, "dare_bench_stream failed")


def dare_bench_mfma_loop(n_blocks, n_iter, pattern, stream=None):
    """Enqueue the register-resident MFMA loop; returns the flop count of the launch."""
    flops = ctypes.c_double(0.0)
    st = bench_lib().dare_bench_mfma_loop(n_blocks, n_iter, pattern, None, ctypes.byref(flops), _stream(stream))
    if st != 0:
        raise DareError(st, "dare_bench_mfma_loop failed")
    return flops.value
