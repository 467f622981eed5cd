"""ctypes binding of the C ABI in include/elasto.h (argument marshalling only).

Every computation runs in the HIP library; this module converts numpy host
arrays and torch device tensors into the plain pointers and sizes the C ABI
takes, and turns status codes into exceptions.  If the library is not built
this module raises: there is no CPU fallback.
"""
from __future__ import annotations

import ctypes
import math
import os
from typing import Dict, Optional

import numpy as np

from .inputs import BF16, FP32, DNTable, ModelConfig

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_lib", "libelasto.so")

c_i32, c_i64, c_f32, c_f64, c_vp = (ctypes.c_int32, ctypes.c_int64, ctypes.c_float,
                                     ctypes.c_double, ctypes.c_void_p)

STATUS = {0: "OK", 1: "INVALID_ARG", 2: "BAD_CONFIG", 3: "BAD_TABLE", 4: "OUT_OF_MEMORY",
          5: "HIP", 6: "MODE_RANGE", 7: "BATCH_RANGE", 8: "INFEASIBLE"}

# Tensor ids (elasto_tensor_t).
T_PATCH_W, T_PATCH_B, T_CLS, T_POS, T_NORM_G, T_NORM_B, T_HEAD_W, T_HEAD_B = range(8)
(T_LN1_G, T_LN1_B, T_WQKV, T_BQKV, T_WO, T_BO, T_LN2_G, T_LN2_B, T_W1, T_B1, T_W2,
 T_B2) = range(8, 20)
# Kernel classes (elasto_kernel_t).
KERNELS = ["patch", "ln", "qkv", "attn", "proj", "fc1", "fc2", "head"]
# Epilogues (elasto_epilogue_t).
EPI_BIAS, EPI_BIAS_GELU, EPI_BIAS_RESID, EPI_BIAS_F32OUT = range(4)

WEIGHT_FIELDS = ["patch_w", "patch_b", "cls", "pos", "ln1_g", "ln1_b", "qkv_w", "qkv_b",
                 "proj_w", "proj_b", "ln2_g", "ln2_b", "fc1_w", "fc1_b", "fc2_w", "fc2_b",
                 "norm_g", "norm_b", "head_w", "head_b"]


class ElastoError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"elasto {STATUS.get(status, status)}: {msg}")
        self.status = status


class Config(ctypes.Structure):
    _fields_ = [(n, c_i32) for n in ("img", "patch", "in_chans", "dim", "depth", "heads",
                                     "mlp_hidden", "num_classes", "max_batch", "dtype")] + \
               [("ln_eps", c_f32)]


class Weights(ctypes.Structure):
    _fields_ = [(n, c_vp) for n in WEIGHT_FIELDS]


class Table(ctypes.Structure):
    _fields_ = [("num_modes", c_i32), ("depth", c_i32), ("n_heads", c_vp), ("n_mlp", c_vp),
                ("head_order", c_vp), ("mlp_order", c_vp), ("n_embed", c_vp),
                ("embed_order", c_vp)]


class DNLut(ctypes.Structure):
    _fields_ = [("num_modes", c_i32), ("flops", ctypes.POINTER(c_f64)),
                ("latency_ms", ctypes.POINTER(c_f64)), ("memory_bytes", ctypes.POINTER(c_f64)),
                ("accuracy", ctypes.POINTER(c_f64)), ("power_w", ctypes.POINTER(c_f64))]


class CNNConfig(ctypes.Structure):
    _fields_ = [("img", c_i32), ("in_chans", c_i32), ("stem", c_i32), ("num_stages", c_i32),
                ("widths", c_i32 * 8), ("blocks", c_i32 * 8), ("expansion", c_i32),
                ("num_classes", c_i32), ("max_batch", c_i32), ("dtype", c_i32)]


class CNNWeights(ctypes.Structure):
    _fields_ = [("num_tensors", c_i32), ("tensors", ctypes.POINTER(ctypes.c_void_p))]


class CNNTableC(ctypes.Structure):
    _fields_ = [("num_modes", c_i32), ("num_blocks", c_i32), ("n_width", c_vp),
                ("order1", c_vp), ("order2", c_vp)]


class Heads(ctypes.Structure):
    _fields_ = [("data", c_vp), ("batch_stride", c_i64), ("token_stride", c_i64),
                ("head_stride", c_i64)]


class QkNorm(ctypes.Structure):
    _fields_ = [(n, c_i32) for n in ("dtype", "batch", "tokens", "q_heads", "kv_heads", "head_dim",
                                     "rot_dim", "interleaved", "table_rows")] + \
               [("eps", c_f32)] + \
               [(n, c_vp) for n in ("positions", "lens", "cos", "sin", "q_gamma", "k_gamma")]


class Window(ctypes.Structure):
    _fields_ = [(n, c_i32) for n in ("dtype", "batch", "q_tokens", "k_tokens", "heads", "kv_heads",
                                     "head_dim", "causal", "window", "sinks")] + \
               [("scale", c_f32), ("q_lens", c_vp), ("k_lens", c_vp)]


_lib: Optional[ctypes.CDLL] = None


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise ImportError(f"{path} is not built; run __graft_entry__.build() or "
                          f"python -m paper_2609_10018_amd.build")
    lib = ctypes.CDLL(path)
    P = ctypes.POINTER
    sig = {
        "elasto_create": [P(Config), P(Weights), P(Table), P(c_vp)],
        "elasto_destroy": [c_vp],
        "elasto_set_mode": [c_vp, c_i32],
        "elasto_get_mode": [c_vp, P(c_i32)],
        "elasto_forward": [c_vp, c_vp, c_i32, c_vp, c_vp],
        "elasto_forward_static": [c_vp, c_vp, c_i32, c_vp, c_vp],
        "elasto_mode_info": [c_vp, c_i32, P(c_f64), P(c_i64)],
        "elasto_memory_info": [c_vp, P(c_i64), P(c_i64)],
        "elasto_validate": [P(Config), P(Table)],
        "elasto_packed_bytes": [P(Config), P(c_i64)],
        "elasto_packed_layout": [P(Config), c_i32, c_i32, P(c_i64), P(c_i64), P(c_i64), P(c_i32)],
        "elasto_pack_weights": [P(Config), P(Weights), P(Table), c_vp, c_i64],
        "elasto_kernel_timing": [c_vp, c_i32, c_i32],
        "elasto_kernel_timing_read": [c_vp, P(c_f64), P(c_i64)],
        "elasto_kernel_work": [c_vp, c_i32, c_i32, c_i32, P(c_f64), P(c_f64), P(c_i32)],
        "elasto_op_layernorm": [c_i32, c_vp, c_i64, c_vp, c_i32, c_vp, c_i64, c_i32, c_vp, c_vp,
                                c_f32, c_vp],
        "elasto_op_linear": [c_i32, c_i32, c_vp, c_i64, c_vp, c_i64, c_vp, c_i64, c_vp, c_i32,
                             c_vp, c_i64, c_i32, c_i32, c_vp],
        "elasto_op_linear_ln": [c_i32, c_vp, c_i64, c_vp, c_i64, c_vp, c_i64, c_vp, c_i32, c_vp,
                                c_i64, c_i32, c_i32, c_vp, c_vp, c_i64, c_vp, c_f32, c_vp],
        "elasto_op_attention": [c_i32, c_vp, c_i64, c_vp, c_i64, c_i32, c_i32, c_i32, c_i32,
                                c_f32, c_vp],
        "elasto_op_conv2d": [c_vp, c_i32, c_i32, c_i32, c_i32, c_i32, c_i32, c_i32, c_i32, c_i32,
                             c_vp, c_i64, c_i64, c_vp, c_vp, c_i64, c_i32, c_i32, c_vp],
        "elasto_op_qk_norm_rotate": [P(QkNorm)] + [P(Heads)] * 4 + [c_vp],
        "elasto_op_qk_norm_rotate_bwd": [P(QkNorm)] + [P(Heads)] * 6 + [c_vp, c_vp, c_vp, c_i64, c_vp],
        "elasto_qk_norm_rotate_workspace": [P(QkNorm), P(c_i64)],
        "elasto_op_window_attention": [P(Window)] + [P(Heads)] * 4 + [c_vp, c_vp, c_i64, c_vp],
        "elasto_op_window_attention_bwd": [P(Window)] + [P(Heads)] * 4 + [c_vp] + [P(Heads)] * 4 +
                                          [c_vp, c_i64, c_vp],
        "elasto_window_attention_workspace": [P(Window), c_i32, P(c_i64)],
        "elasto_op_top_logits": [c_i32, c_vp, c_i64, c_i64, c_i32, c_i32, c_vp, c_vp, c_vp],
        "elasto_op_distill": [c_i32, c_vp, c_i64, c_i64, c_i32, c_vp, c_vp, c_i32, c_vp, c_vp, c_f32,
                              c_f32, c_f32, c_vp, c_i32, c_vp, c_i64, c_vp],
        "elasto_select_mode": [P(DNLut), c_f64, c_f64, c_f64, c_f64, P(c_i32)],
        "elasto_growth_create": [c_vp, c_i32, P(c_vp)],
        "elasto_growth_destroy": [c_vp],
        "elasto_growth_step": [c_vp, c_i32, c_vp, c_vp, c_i32, c_f32, c_f32, c_vp, c_vp],
        "elasto_growth_step_distill": [c_vp, c_i32, c_vp, c_vp, c_vp, c_vp, c_i32, c_f32, c_f32,
                                       c_i32, c_f32, c_f32, c_vp, c_vp],
        "elasto_growth_read": [c_vp, c_i32, c_vp, c_i64],
        "elasto_profile_modes": [c_vp, c_vp, c_i32, c_vp, c_i32, c_i32, c_vp, P(c_f64), P(c_f64),
                                 P(c_f64)],
        "elasto_cnn_validate": [P(CNNConfig), P(CNNTableC)],
        "elasto_cnn_create": [P(CNNConfig), P(CNNWeights), P(CNNTableC), P(c_vp)],
        "elasto_cnn_destroy": [c_vp],
        "elasto_cnn_set_mode": [c_vp, c_i32],
        "elasto_cnn_get_mode": [c_vp, P(c_i32)],
        "elasto_cnn_forward": [c_vp, c_vp, c_i32, c_vp, c_vp],
        "elasto_cnn_mode_info": [c_vp, c_i32, P(c_f64), P(c_i64)],
    }
    for name, args in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = c_i32
    lib.elasto_last_error.argtypes = []
    lib.elasto_last_error.restype = ctypes.c_char_p
    _lib = lib
    return lib


def last_error() -> str:
    return load_library().elasto_last_error().decode()


def check(status: int) -> None:
    if status != 0:
        raise ElastoError(status, last_error())


def make_config(cfg: ModelConfig, max_batch: int) -> Config:
    return Config(cfg.img, cfg.patch, cfg.in_chans, cfg.dim, cfg.depth, cfg.heads,
                  cfg.mlp_hidden, cfg.num_classes, max_batch, cfg.dtype, cfg.ln_eps)


class _HostWeights:
    """Keeps contiguous fp32 copies alive while the C struct points at them."""

    def __init__(self, w: Dict[str, np.ndarray]):
        self.arrays = {k: np.ascontiguousarray(w[k], dtype=np.float32) for k in WEIGHT_FIELDS}
        self.struct = Weights(*[a.ctypes.data for a in (self.arrays[k] for k in WEIGHT_FIELDS)])


class _HostTable:
    """Keeps int32 copies alive while the C struct points at them; the
    embedding columns are optional (None: every mode keeps all channels,
    identity order)."""

    def __init__(self, t: DNTable):
        cols = (t.n_heads, t.n_mlp, t.head_order, t.mlp_order,
                getattr(t, "n_embed", None), getattr(t, "embed_order", None))
        self.arrays = [None if a is None else np.ascontiguousarray(a, dtype=np.int32)
                       for a in cols]
        self.struct = Table(int(t.n_heads.shape[0]), int(t.n_heads.shape[1]),
                            *[None if a is None else a.ctypes.data for a in self.arrays])


def validate(cfg: ModelConfig, table: DNTable, max_batch: int = 1) -> int:
    c = make_config(cfg, max_batch)
    t = _HostTable(table)
    return load_library().elasto_validate(ctypes.byref(c), ctypes.byref(t.struct))


def packed_bytes(cfg: ModelConfig) -> int:
    out = c_i64()
    check(load_library().elasto_packed_bytes(ctypes.byref(make_config(cfg, 1)), ctypes.byref(out)))
    return out.value


def packed_layout(cfg: ModelConfig, tensor: int, layer: int = 0):
    off, rows, cols, eb = c_i64(), c_i64(), c_i64(), c_i32()
    check(load_library().elasto_packed_layout(ctypes.byref(make_config(cfg, 1)), tensor, layer,
                                              ctypes.byref(off), ctypes.byref(rows),
                                              ctypes.byref(cols), ctypes.byref(eb)))
    return off.value, rows.value, cols.value, eb.value


def pack_weights(cfg: ModelConfig, w: Dict[str, np.ndarray], table: DNTable) -> np.ndarray:
    n = packed_bytes(cfg)
    dst = np.zeros(n, dtype=np.uint8)
    hw, ht = _HostWeights(w), _HostTable(table)
    check(load_library().elasto_pack_weights(ctypes.byref(make_config(cfg, 1)),
                                             ctypes.byref(hw.struct), ctypes.byref(ht.struct),
                                             dst.ctypes.data, n))
    return dst


_raw_stream = None      # torch's (device index) -> hipStream_t of its current stream


def _stream_ptr(stream, device: Optional[int] = None) -> int:
    """The hipStream_t of `stream`; None: torch's current stream (of the current device, which
    `device` is where the caller has asked for it already).

    Asked for as a pointer: building torch's Stream object to read it from took
    3.0 of the 7.8 us of host time of a small call."""
    if stream is not None:
        return int(getattr(stream, "cuda_stream", stream))
    global _raw_stream
    if device is not None and _raw_stream is not None:
        return _raw_stream(device)
    import torch
    if _raw_stream is None:
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda device: torch.cuda.current_stream(device).cuda_stream)
    return _raw_stream(torch.cuda.current_device())


class ElasticViT:
    """One library handle: packed weights on the current device + scratch."""

    def __init__(self, cfg: ModelConfig, w: Dict[str, np.ndarray], table: DNTable,
                 max_batch: int):
        self.lib = load_library()
        self.cfg = cfg
        self.max_batch = max_batch
        self.num_modes = int(table.n_heads.shape[0])
        c = make_config(cfg, max_batch)
        hw, ht = _HostWeights(w), _HostTable(table)
        h = c_vp()
        check(self.lib.elasto_create(ctypes.byref(c), ctypes.byref(hw.struct),
                                     ctypes.byref(ht.struct), ctypes.byref(h)))
        self.h = h

    def close(self) -> None:
        if getattr(self, "h", None) is not None and self.h.value:
            check(self.lib.elasto_destroy(self.h))
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_mode(self, k: int) -> None:
        check(self.lib.elasto_set_mode(self.h, int(k)))

    def get_mode(self) -> int:
        k = c_i32()
        check(self.lib.elasto_get_mode(self.h, ctypes.byref(k)))
        return k.value

    def forward(self, images, logits, stream=None) -> None:
        """images: device tensor NCHW (bf16 or fp32 per the path); logits: fp32 device tensor."""
        if not images.is_contiguous() or not logits.is_contiguous():
            raise ValueError("images and logits must be contiguous")
        check(self.lib.elasto_forward(self.h, images.data_ptr(), int(images.shape[0]),
                                      logits.data_ptr(), _stream_ptr(stream)))

    def forward_static(self, images, logits, stream=None) -> None:
        """The forward with its activations in the library's static scratch
        (elasto_forward_static: allocates nothing)."""
        if not images.is_contiguous() or not logits.is_contiguous():
            raise ValueError("images and logits must be contiguous")
        check(self.lib.elasto_forward_static(self.h, images.data_ptr(), int(images.shape[0]),
                                             logits.data_ptr(), _stream_ptr(stream)))

    def mode_info(self, k: int):
        f, b = c_f64(), c_i64()
        check(self.lib.elasto_mode_info(self.h, int(k), ctypes.byref(f), ctypes.byref(b)))
        return f.value, b.value

    def profile_modes(self, images, logits, warmup: int = 3, iters: int = 10, stream=None):
        """Per-mode (latency_ms, memory_bytes, flops) arrays at images.shape[0]."""
        n = self.num_modes
        lat, mem, fl = (np.zeros(n, dtype=np.float64) for _ in range(3))
        dp = ctypes.POINTER(c_f64)
        check(self.lib.elasto_profile_modes(
            self.h, images.data_ptr(), int(images.shape[0]), logits.data_ptr(), int(warmup),
            int(iters), _stream_ptr(stream), lat.ctypes.data_as(dp), mem.ctypes.data_as(dp),
            fl.ctypes.data_as(dp)))
        return lat, mem, fl

    def memory_info(self):
        wb, sb = c_i64(), c_i64()
        check(self.lib.elasto_memory_info(self.h, ctypes.byref(wb), ctypes.byref(sb)))
        return wb.value, sb.value

    def kernel_timing(self, kernel: str, max_launches: int) -> None:
        kc = -1 if kernel is None else KERNELS.index(kernel)
        check(self.lib.elasto_kernel_timing(self.h, kc, int(max_launches)))

    def kernel_timing_read(self):
        ms, n = c_f64(), c_i64()
        check(self.lib.elasto_kernel_timing_read(self.h, ctypes.byref(ms), ctypes.byref(n)))
        return ms.value, n.value

    def kernel_work(self, k: int, batch: int, kernel: str):
        f, b, n = c_f64(), c_f64(), c_i32()
        check(self.lib.elasto_kernel_work(self.h, int(k), int(batch), KERNELS.index(kernel),
                                          ctypes.byref(f), ctypes.byref(b), ctypes.byref(n)))
        return f.value, b.value, n.value


def _ptr(t):
    return None if t is None else t.data_ptr()


def op_layernorm(dtype: int, x, x_stride: int, out, rows: int, d: int, g, b, eps: float,
                 x_cls=None, tokens: int = 1, stream=None) -> None:
    check(load_library().elasto_op_layernorm(dtype, x.data_ptr(), x_stride, _ptr(x_cls), tokens,
                                             out.data_ptr(), rows, d, g.data_ptr(), b.data_ptr(),
                                             eps, _stream_ptr(stream)))


def op_linear(dtype: int, epilogue: int, A, lda: int, W, ldw: int, C, ldc: int, bias,
              M: int, N: int, K: int, C_cls=None, tokens: int = 1, stream=None) -> None:
    check(load_library().elasto_op_linear(dtype, epilogue, A.data_ptr(), lda, W.data_ptr(), ldw,
                                          C.data_ptr(), ldc, _ptr(C_cls), tokens, bias.data_ptr(),
                                          M, N, K, _stream_ptr(stream)))


def op_linear_ln(epilogue: int, A, lda: int, W, ldw: int, C, ldc: int, bias, M: int, N: int,
                 K: int, stats_ld: int, stats_out=None, stats_in=None, colsum=None,
                 eps: float = 1e-6, C_cls=None, tokens: int = 1, stream=None) -> None:
    check(load_library().elasto_op_linear_ln(epilogue, A.data_ptr(), lda, W.data_ptr(), ldw,
                                             C.data_ptr(), ldc, _ptr(C_cls), tokens,
                                             bias.data_ptr(), M, N, K, _ptr(stats_out),
                                             _ptr(stats_in), stats_ld, _ptr(colsum), eps,
                                             _stream_ptr(stream)))


def op_attention(dtype: int, qkv, qkv_stride: int, o, o_stride: int, batch: int, tokens: int,
                 heads: int, head_dim: int, scale: float, stream=None) -> None:
    check(load_library().elasto_op_attention(dtype, qkv.data_ptr(), qkv_stride, o.data_ptr(),
                                             o_stride, batch, tokens, heads, head_dim, scale,
                                             _stream_ptr(stream)))


# Per-call work of the operators below is kept small: a call on a few tokens
# takes less time on the GPU than these checks would if they formatted names.
_torch = None        # torch's element types and its cuda module, at the first use


class _Torch:
    def __init__(self):
        import torch
        self.f32, self.i32, self.u8 = torch.float32, torch.int32, torch.uint8
        self.types = {torch.bfloat16: BF16, torch.float32: FP32}
        self.cuda = torch.cuda


def _tt() -> _Torch:
    global _torch
    if _torch is None:
        _torch = _Torch()
    return _torch


def _same_device(*tensors) -> int:
    """Refuse tensors that do not all lie on the current device: the kernels run there."""
    d = _tt().cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != d:
            raise ValueError(f"a tensor lies on {t.device}, the current device is cuda:{d}")
    return d


_MAX = 2 ** 31 - 1


def _fits(*sizes) -> None:
    """Refuse sizes of more than the C ABI's 32-bit integers, which ctypes would cut off."""
    if max(sizes) > _MAX:
        raise ValueError(f"a size of {max(sizes)} does not fit 32 bits")


def _int(n) -> int:
    """n for the C ABI's own checks: one that it refuses where n does not fit 32 bits."""
    return max(-1, min(int(n), _MAX))


def _dtype(t) -> int:
    try:
        return _tt().types[t.dtype]
    except KeyError:
        raise ValueError(f"{t.dtype} is not supported: bfloat16 or float32") from None


def _plain(t, want, name: str, numel: int = -1):
    """The address of a contiguous device tensor of one element type (None: NULL)."""
    if t is None:
        return None
    if t.dtype is not want or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous and {want}, not {t.dtype}")
    if numel >= 0 and t.numel() != numel:
        raise ValueError(f"{name} has {t.numel()} elements, not {numel}")
    return t.data_ptr()


def _heads(t, shape, dtype, name: str):
    """A [batch, tokens, heads, head_dim] tensor as the C ABI takes it (None: no heads)."""
    if t is None:
        return None
    if t.shape != shape or t.dtype is not dtype:
        raise ValueError(f"{name} is {tuple(t.shape)} {t.dtype}, not {tuple(shape)} {dtype}")
    return _strided(t, shape, name)


def _strided(t, shape, name: str):
    """The same of a tensor that the shape was taken from."""
    b, r, h, f = t.stride()
    nb, nr, nh, n = shape
    if f != 1 and n > 1:
        raise ValueError(f"the features of {name} must be contiguous")
    # The stride of an axis of one element means nothing; torch may give any.
    return Heads(t.data_ptr(), b if nb > 1 else n, r if nr > 1 else n, h if nh > 1 else n)


def _space(workspace):
    """Address and bytes of a workspace (None: none)."""
    if workspace is None:
        return None, 0
    return _plain(workspace, _tt().u8, "workspace"), workspace.numel()


def _qk_desc(q, k, cos, sin, q_gamma, k_gamma, positions, lens, eps, interleaved):
    """The description, and the shapes of q and of k."""
    x = q if q is not None else k
    if x.dim() != 4:
        raise ValueError(f"q and k must be [batch, tokens, heads, head_dim], not {tuple(x.shape)}")
    tt = _tt()
    shape = x.shape
    b, t, n, d = shape
    other = 0 if q is None or k is None else k.shape[2]
    nq, nk = (0, n) if q is None else (n, other)
    rot = rows = 0
    if cos is not None:
        rows, rot = cos.shape
        rot *= 2
    if (cos is None) != (sin is None) or (cos is not None and cos.shape != sin.shape):
        raise ValueError("cos and sin must be given together, of one shape")
    _fits(b, t, n, d, other, rows, rot)
    if positions is not None and positions.shape != (b, t):
        raise ValueError(f"positions is {tuple(positions.shape)}, not {(b, t)}")
    f32, i32 = tt.f32, tt.i32
    a = QkNorm(_dtype(x), b, t, nq, nk, d, rot, 1 if interleaved else 0, rows, eps,
               _plain(positions, i32, "positions"), _plain(lens, i32, "lens", b),
               _plain(cos, f32, "cos"), _plain(sin, f32, "sin"),
               _plain(q_gamma, f32, "q_gamma", d), _plain(k_gamma, f32, "k_gamma", d))
    return a, (b, t, nq, d), (b, t, nk, d), x.dtype


def qk_norm_rotate_workspace(q, k) -> int:
    """Workspace bytes of op_qk_norm_rotate_bwd for these q and k."""
    n = c_i64()
    a = _qk_desc(q, k, None, None, None, None, None, None, 1.0, False)[0]
    check(load_library().elasto_qk_norm_rotate_workspace(a, ctypes.byref(n)))
    return n.value


def op_qk_norm_rotate(q, k, q_out, k_out, cos=None, sin=None, q_gamma=None, k_gamma=None,
                      positions=None, lens=None, eps: float = 1e-6, interleaved: bool = False,
                      stream=None) -> None:
    """q, q_out: [batch, tokens, heads, head_dim] device tensors of any strides (the features
    contiguous); k, k_out likewise with their own heads; either pair may be None.  cos, sin: fp32
    [rows, rot_dim / 2] (None: no rotation).  positions: int32 [batch, tokens]; lens: int32
    [batch]."""
    dev = _same_device(q, k, q_out, k_out, cos, sin, q_gamma, k_gamma, positions, lens)
    a, sq, sk, dt = _qk_desc(q, k, cos, sin, q_gamma, k_gamma, positions, lens, eps, interleaved)
    check(load_library().elasto_op_qk_norm_rotate(
        a, None if q is None else _strided(q, sq, "q"), _heads(k, sk, dt, "k"),
        _heads(q_out, sq, dt, "q_out"), _heads(k_out, sk, dt, "k_out"), _stream_ptr(stream, dev)))


def op_qk_norm_rotate_bwd(q, k, dq_out, dk_out, dq, dk, dq_gamma=None, dk_gamma=None,
                          workspace=None, cos=None, sin=None, q_gamma=None, k_gamma=None,
                          positions=None, lens=None, eps: float = 1e-6, interleaved: bool = False,
                          stream=None) -> None:
    """dq_out, dk_out: the gradients of op_qk_norm_rotate's results; dq, dk: those of q and k;
    dq_gamma, dk_gamma: fp32 [head_dim] or None.  workspace: a uint8 device tensor of
    qk_norm_rotate_workspace() bytes where a weight gradient is asked for."""
    dev = _same_device(q, k, dq_out, dk_out, dq, dk, dq_gamma, dk_gamma, workspace, cos, sin,
                       q_gamma, k_gamma, positions, lens)
    a, sq, sk, dt = _qk_desc(q, k, cos, sin, q_gamma, k_gamma, positions, lens, eps, interleaved)
    f32 = _tt().f32
    check(load_library().elasto_op_qk_norm_rotate_bwd(
        a, None if q is None else _strided(q, sq, "q"), _heads(k, sk, dt, "k"),
        _heads(dq_out, sq, dt, "dq_out"), _heads(dk_out, sk, dt, "dk_out"),
        _heads(dq, sq, dt, "dq"), _heads(dk, sk, dt, "dk"),
        _plain(dq_gamma, f32, "dq_gamma", sq[3]), _plain(dk_gamma, f32, "dk_gamma", sq[3]),
        *_space(workspace), _stream_ptr(stream, dev)))


def _window_desc(q, k, window, sinks, causal, scale, q_lens, k_lens):
    """The description, and the shapes of q and of k."""
    sq, sk = q.shape, k.shape
    if len(sq) != 4 or len(sk) != 4 or sq[0] != sk[0] or sq[3] != sk[3]:
        raise ValueError(f"q {tuple(sq)} and k {tuple(sk)} do not go together")
    b, tq, h, d = sq
    _fits(*sq, *sk)
    i32 = _tt().i32
    if scale is None:
        scale = 1.0 / math.sqrt(d or 1)
    a = Window(_dtype(q), b, tq, sk[1], h, sk[2], d, 1 if causal else 0,
               _int(window), _int(sinks), scale,
               _plain(q_lens, i32, "q_lens", b), _plain(k_lens, i32, "k_lens", b))
    return a, sq, sk, q.dtype


def window_attention_workspace(q, k, window: int, sinks: int = 0, causal: bool = True,
                               backward: bool = False) -> int:
    """Workspace bytes of op_window_attention (backward: op_window_attention_bwd) for tensors of
    these shapes."""
    n = c_i64()
    a = _window_desc(q, k, window, sinks, causal, None, None, None)[0]
    check(load_library().elasto_window_attention_workspace(a, int(bool(backward)), ctypes.byref(n)))
    return n.value


def op_window_attention(q, k, v, o, window: int, sinks: int = 0, causal: bool = True,
                        scale: Optional[float] = None, lse=None, q_lens=None, k_lens=None,
                        workspace=None, stream=None) -> None:
    """q, o: [batch, q_tokens, heads, head_dim] device tensors of any strides (the features
    contiguous); k, v: [batch, k_tokens, kv_heads, head_dim].  lse: fp32 [batch, heads, q_tokens]
    or None.  q_lens, k_lens: int32 [batch] or None.  scale: None for 1 / sqrt(head_dim).
    workspace: a uint8 device tensor of window_attention_workspace() bytes."""
    dev = _same_device(q, k, v, o, lse, q_lens, k_lens, workspace)
    a, sq, sk, dt = _window_desc(q, k, window, sinks, causal, scale, q_lens, k_lens)
    check(load_library().elasto_op_window_attention(
        a, _strided(q, sq, "q"), _heads(k, sk, dt, "k"), _heads(v, sk, dt, "v"),
        _heads(o, sq, dt, "o"), _plain(lse, _tt().f32, "lse", sq[0] * sq[1] * sq[2]),
        *_space(workspace), _stream_ptr(stream, dev)))


def op_window_attention_bwd(q, k, v, o, lse, dout, dq, dk, dv, window: int, sinks: int = 0,
                            causal: bool = True, scale: Optional[float] = None, q_lens=None,
                            k_lens=None, workspace=None, stream=None) -> None:
    """The gradients dq, dk, dv (shaped like q, k, v) from dout (like o), with op_window_attention's
    o and lse."""
    dev = _same_device(q, k, v, o, lse, dout, dq, dk, dv, q_lens, k_lens, workspace)
    a, sq, sk, dt = _window_desc(q, k, window, sinks, causal, scale, q_lens, k_lens)
    check(load_library().elasto_op_window_attention_bwd(
        a, _strided(q, sq, "q"), _heads(k, sk, dt, "k"), _heads(v, sk, dt, "v"),
        _heads(o, sq, dt, "o"), _plain(lse, _tt().f32, "lse", sq[0] * sq[1] * sq[2]),
        _heads(dout, sq, dt, "dout"), _heads(dq, sq, dt, "dq"), _heads(dk, sk, dt, "dk"),
        _heads(dv, sk, dt, "dv"), *_space(workspace), _stream_ptr(stream, dev)))


def _rows(t, name: str):
    """A [rows, classes] tensor with contiguous rows: (rows, classes, row stride)."""
    shape, stride = t.shape, t.stride()
    if len(shape) != 2 or (stride[1] != 1 and shape[1] > 1):
        raise ValueError(f"{name} must be [rows, classes] with contiguous rows")
    r, c = shape
    _fits(c)
    return r, c, stride[0] if r > 1 else c


def op_top_logits(logits, values, indices, stream=None) -> None:
    """logits: bf16 or fp32 [rows, classes] device tensor (any row stride); values: fp32 and
    indices: int32, [rows, top]."""
    dev = _same_device(logits, values, indices)
    r, c, ld = _rows(logits, "logits")
    shape = values.shape
    if len(shape) != 2 or shape != indices.shape or shape[0] != r:
        raise ValueError(f"values {tuple(shape)} and indices {tuple(indices.shape)} must be "
                         f"[{r}, top]")
    _fits(shape[1])
    check(load_library().elasto_op_top_logits(
        _dtype(logits), logits.data_ptr(), ld, r, c, shape[1], _plain(values, _tt().f32, "values"),
        _plain(indices, _tt().i32, "indices"), _stream_ptr(stream, dev)))


def op_distill(logits, teacher_values, teacher_indices, loss, dlogits=None, labels=None,
               temperature: float = 1.0, alpha: float = 1.0, row_weight=None, scale: float = 1.0,
               stream=None) -> None:
    """logits: bf16 or fp32 [rows, classes] device tensor (any row stride); teacher_values: fp32
    and teacher_indices: int32, [rows, top] (None with alpha 0); loss: fp32 [rows]; dlogits: bf16
    or fp32 [rows, classes] or None; labels: int32 [rows] or None; row_weight: fp32 [rows] or
    None."""
    dev = _same_device(logits, teacher_values, teacher_indices, loss, dlogits, labels, row_weight)
    r, c, ld = _rows(logits, "logits")
    top = 0
    if teacher_values is not None:
        shape = teacher_values.shape
        if (teacher_indices is None or len(shape) != 2 or shape[0] != r
                or shape != teacher_indices.shape):
            raise ValueError(f"teacher values and indices must both be [{r}, top]")
        top = shape[1]
        _fits(top)
    dt = gd = _dtype(logits)
    ldg, grad = ld, None
    if dlogits is not None:
        rg, cg, ldg = _rows(dlogits, "dlogits")
        if (rg, cg) != (r, c):
            raise ValueError(f"dlogits is {(rg, cg)}, not {(r, c)}")
        gd, grad = _dtype(dlogits), dlogits.data_ptr()
    f32, i32 = _tt().f32, _tt().i32
    check(load_library().elasto_op_distill(
        dt, logits.data_ptr(), ld, r, c, _plain(teacher_values, f32, "teacher_values"),
        _plain(teacher_indices, i32, "teacher_indices"), top, _plain(labels, i32, "labels", r),
        _plain(row_weight, f32, "row_weight", r), temperature, alpha, scale,
        _plain(loss, f32, "loss", r), gd, grad, ldg, _stream_ptr(stream, dev)))


class GrowthContext:
    """Growth-step state of a bf16 ElasticViT handle (fp32 masters, saved
    activations, gradients) for batches of up to max_batch images."""

    def __init__(self, vit: "ElasticViT", max_batch: int):
        self.lib = load_library()
        self.vit = vit                      # the handle must outlive the context
        g = c_vp()
        check(self.lib.elasto_growth_create(vit.h, int(max_batch), ctypes.byref(g)))
        self.g = g

    def step(self, mode: int, images, labels, lr: float, clip: float, stats=None,
             stream=None) -> None:
        """images: bf16 device tensor NCHW; labels: int32 device tensor [batch];
        stats: fp32 device tensor with 3 elements (loss, |G grad|, clip factor) or None."""
        if not images.is_contiguous() or not labels.is_contiguous():
            raise ValueError("images and labels must be contiguous")
        check(self.lib.elasto_growth_step(self.g, int(mode), images.data_ptr(), labels.data_ptr(),
                                          int(images.shape[0]), float(lr), float(clip),
                                          _ptr(stats), _stream_ptr(stream)))

    def step_distill(self, mode: int, images, labels, teacher_values, teacher_indices, lr: float,
                     clip: float, temperature: float = 1.0, alpha: float = 1.0, stats=None,
                     stream=None) -> None:
        """The growth step with op_distill's loss: teacher_values (fp32) and teacher_indices
        (int32) are [batch, top] device tensors; labels may be None with alpha 1."""
        if not images.is_contiguous() or (labels is not None and not labels.is_contiguous()):
            raise ValueError("images and labels must be contiguous")
        n = int(images.shape[0])
        if teacher_values.dim() != 2 or teacher_values.shape != teacher_indices.shape or \
                teacher_values.shape[0] != n:
            raise ValueError(f"teacher values and indices must be [{n}, top]")
        _fits(n, teacher_values.shape[1])
        _same_device(images, labels, teacher_values, teacher_indices, stats)
        check(self.lib.elasto_growth_step_distill(
            self.g, int(mode), images.data_ptr(), _plain(labels, _tt().i32, "labels", n),
            _plain(teacher_values, _tt().f32, "teacher_values"),
            _plain(teacher_indices, _tt().i32, "teacher_indices"), int(teacher_values.shape[1]),
            float(temperature), float(alpha), n, float(lr), float(clip), _ptr(stats),
            _stream_ptr(stream)))

    def read(self, which: int) -> np.ndarray:
        """which 0: packed weights (uint8); 1: fp32 masters (float32, one per bf16 element)."""
        total = packed_bytes(self.vit.cfg)
        n = total if which == 0 else total // 2 * 4
        buf = np.empty(n, dtype=np.uint8)
        check(self.lib.elasto_growth_read(self.g, int(which), buf.ctypes.data, n))
        return buf if which == 0 else buf.view(np.float32)

    def close(self) -> None:
        if getattr(self, "g", None) is not None and self.g.value:
            check(self.lib.elasto_growth_destroy(self.g))
            self.g = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def op_conv2d(x, batch: int, H: int, W: int, cs: int, ca: int, kh: int, kw: int, stride: int,
              pad: int, w, ldw: int, wseg: int, bias, y, ldy: int, n: int, relu: bool = False,
              stream=None) -> None:
    check(load_library().elasto_op_conv2d(x.data_ptr(), batch, H, W, cs, ca, kh, kw, stride, pad,
                                          w.data_ptr(), ldw, wseg, bias.data_ptr(), y.data_ptr(),
                                          ldy, n, int(relu), _stream_ptr(stream)))


class _HostCNN:
    """Keeps the host arrays alive while the C structs point at them."""

    def __init__(self, cfg, w, table, max_batch: int):
        from .inputs_cnn import conv_shapes
        self.cfg = CNNConfig()
        self.cfg.img, self.cfg.in_chans, self.cfg.stem = cfg.img, cfg.in_chans, cfg.stem
        self.cfg.num_stages = len(cfg.widths)
        for i, (wd, nb) in enumerate(zip(cfg.widths, cfg.blocks)):
            self.cfg.widths[i], self.cfg.blocks[i] = wd, nb
        self.cfg.expansion, self.cfg.num_classes = cfg.expansion, cfg.num_classes
        self.cfg.max_batch, self.cfg.dtype = max_batch, cfg.dtype
        self.tensors = [] if w is None else [
            np.ascontiguousarray(w[key], dtype=np.float32) for key in conv_shapes(cfg)]
        self.ptrs = (ctypes.c_void_p * max(1, len(self.tensors)))(
            *[t.ctypes.data for t in self.tensors])
        self.weights = CNNWeights(len(self.tensors), self.ptrs)
        self.n_width = np.ascontiguousarray(table.n_width, dtype=np.int32)
        self.order1 = np.ascontiguousarray(np.concatenate(table.order1), dtype=np.int32)
        self.order2 = np.ascontiguousarray(np.concatenate(table.order2), dtype=np.int32)
        self.table = CNNTableC(int(self.n_width.shape[0]), int(self.n_width.shape[1]),
                               self.n_width.ctypes.data, self.order1.ctypes.data,
                               self.order2.ctypes.data)


def cnn_validate(cfg, table, max_batch: int = 1) -> int:
    hc = _HostCNN(cfg, None, table, max_batch)
    return load_library().elasto_cnn_validate(ctypes.byref(hc.cfg), ctypes.byref(hc.table))


class ElasticResNet:
    """One elastic bottleneck-ResNet handle (bf16, NHWC on the device)."""

    def __init__(self, cfg, w, table, max_batch: int):
        self.lib = load_library()
        self.cfg = cfg
        self.num_modes = int(table.n_width.shape[0])
        hc = _HostCNN(cfg, w, table, max_batch)
        h = c_vp()
        check(self.lib.elasto_cnn_create(ctypes.byref(hc.cfg), ctypes.byref(hc.weights),
                                         ctypes.byref(hc.table), ctypes.byref(h)))
        self.h = h

    def close(self) -> None:
        if getattr(self, "h", None) is not None and self.h.value:
            check(self.lib.elasto_cnn_destroy(self.h))
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_mode(self, k: int) -> None:
        check(self.lib.elasto_cnn_set_mode(self.h, int(k)))

    def get_mode(self) -> int:
        k = c_i32()
        check(self.lib.elasto_cnn_get_mode(self.h, ctypes.byref(k)))
        return k.value

    def forward(self, images, logits, stream=None) -> None:
        check(self.lib.elasto_cnn_forward(self.h, images.data_ptr(), int(images.shape[0]),
                                          logits.data_ptr(), _stream_ptr(stream)))

    def mode_info(self, k: int):
        f, b = c_f64(), c_i64()
        check(self.lib.elasto_cnn_mode_info(self.h, int(k), ctypes.byref(f), ctypes.byref(b)))
        return f.value, b.value


def select_mode(flops, latency_ms, memory_bytes, accuracy=None, power_w=None,
                max_latency_ms=math.inf, max_memory_bytes=math.inf, min_accuracy=-math.inf,
                max_power_w=math.inf):
    """Eq. 11 over a DN table (host only).  Returns the mode, or None when no
    mode meets the bounds."""
    cols = [np.ascontiguousarray(c, dtype=np.float64) if c is not None else None
            for c in (flops, latency_ms, memory_bytes, accuracy, power_w)]
    n = len(cols[0])
    if any(c is not None and len(c) != n for c in cols):
        raise ValueError("table columns differ in length")
    dp = ctypes.POINTER(c_f64)
    ptr = [c.ctypes.data_as(dp) if c is not None else None for c in cols]
    lut = DNLut(n, *ptr)
    k = c_i32(-1)
    st = load_library().elasto_select_mode(ctypes.byref(lut), float(max_latency_ms),
                                           float(max_memory_bytes), float(min_accuracy),
                                           float(max_power_w), ctypes.byref(k))
    if st == 8:
        return None
    check(st)
    return k.value


__all__ = ["ElasticViT", "ElasticResNet", "cnn_validate", "select_mode", "ElastoError", "load_library", "validate", "packed_bytes",
           "packed_layout", "pack_weights", "op_layernorm", "op_linear", "op_linear_ln", "op_attention",
           "op_qk_norm_rotate", "op_qk_norm_rotate_bwd", "qk_norm_rotate_workspace",
           "op_window_attention", "op_window_attention_bwd", "window_attention_workspace",
           "op_top_logits", "op_distill",
           "KERNELS", "FP32", "BF16"]
