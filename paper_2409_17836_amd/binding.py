"""ctypes binding of liblmgc (include/lmgc.h): argument marshalling only.

PyTorch supplies device memory (tensors) and streams; every step of the
LM-GC hot path runs in the library.  If liblmgc.so is missing the import of
this module still works, but every call raises: there is no fallback path.
"""
import ctypes
import math
import os
from typing import List, Optional, Sequence, Tuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblmgc.so")

LMGC_OK = 0
ERRORS = {-1: "EINVAL", -2: "ENOMEM", -3: "EDEVICE", -4: "ESIZE", -5: "ECORRUPT",
          -6: "EUNSUPPORTED"}
NALPHA, NSYM = 17, 18          # with one separator token (A = 17 + escape)
HEADER_BYTES = 128

KINDS = ["embed", "norm", "gemm_qkv", "attn", "gemm_o", "gemm_up", "gemm_down", "gemm_head",
         "lse_cdf"]
KIND = {k: i for i, k in enumerate(KINDS)}


class LMGCError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{ERRORS.get(code, code)}: {msg}")
        self.code = code


class SerialParams(ctypes.Structure):
    _fields_ = [("bytes_per_value", ctypes.c_int32), ("bytes_per_group", ctypes.c_int32),
                ("msb_first", ctypes.c_int32), ("window", ctypes.c_int32),
                ("bos_id", ctypes.c_int32), ("pad_id", ctypes.c_int32),
                ("sep_id", ctypes.c_int32), ("hex_ids", ctypes.c_int32 * 16),
                ("sep2_id", ctypes.c_int32), ("renorm", ctypes.c_int32)]


class ModelConfig(ctypes.Structure):
    _fields_ = [("arch", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("n_layers", ctypes.c_int32), ("d_model", ctypes.c_int32),
                ("n_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("d_ff", ctypes.c_int32), ("vocab", ctypes.c_int32),
                ("max_pos", ctypes.c_int32), ("rope_theta", ctypes.c_float),
                ("norm_eps", ctypes.c_float)]


class DecoderState(ctypes.Structure):
    _fields_ = [("opaque", ctypes.c_uint64 * 8)]


_lib = None


def lib():
    """The loaded library; raises if liblmgc.so has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is not built; run __graft_entry__.build() "
                           "(there is no fallback implementation)")
    L = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, u32, u64, sz = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64,
                                  ctypes.c_uint32, ctypes.c_uint64, ctypes.c_size_t)
    P, f64 = ctypes.POINTER, ctypes.c_double
    sig = {
        "lmgc_last_error": (ctypes.c_char_p, []),
        "lmgc_version": (ctypes.c_char_p, []),
        "lmgc_alphabet_size": (i32, [P(SerialParams)]),
        "lmgc_num_tokens": (i64, [i64, P(SerialParams)]),
        "lmgc_num_windows": (i64, [i64, P(SerialParams)]),
        "lmgc_serialize": (ctypes.c_int, [vp, i64, P(SerialParams), i64, i64, vp, vp, vp]),
        "lmgc_deserialize": (ctypes.c_int, [vp, i64, i64, P(SerialParams), vp]),
        "lmgc_keep_count": (i64, [i64, i32]),
        "lmgc_lossy_workspace": (i64, [i64]),
        "lmgc_sparsify_topk": (ctypes.c_int, [vp, i64, i64, vp, vp, sz, vp]),
        "lmgc_sparsify_topk_noalloc": (ctypes.c_int, [vp, i64, i64, vp, vp]),
        "lmgc_quantize_linear": (ctypes.c_int, [vp, i64, i32, vp, P(ctypes.c_float), vp, sz, vp]),
        "lmgc_sign_pack": (ctypes.c_int, [vp, i64, vp, vp]),
        "lmgc_model_num_tensors": (i32, [P(ModelConfig)]),
        "lmgc_model_tensor_info": (ctypes.c_int, [P(ModelConfig), i32, ctypes.c_char_p, sz,
                                                  P(i32), P(i64)]),
        "lmgc_model_create": (ctypes.c_int, [P(ModelConfig), P(vp), vp, P(vp)]),
        "lmgc_model_destroy": (None, [vp]),
        "lmgc_probs_workspace": (sz, [vp, i32, i32]),
        "lmgc_probs": (ctypes.c_int, [vp, vp, i32, i32, P(SerialParams), u32, vp, vp, vp, sz, vp]),
        "lmgc_step_workspace": (sz, [vp, i32, i32]),
        "lmgc_probs_stepwise": (ctypes.c_int, [vp, vp, i32, i32, P(SerialParams), u32, vp, vp, vp, sz,
                                               vp]),
        "lmgc_encode_bound": (sz, [i32, i32]),
        "lmgc_encode": (ctypes.c_int, [vp, i32, vp, vp, i32, i32, vp, sz, vp, P(sz), i32]),
        "lmgc_decode_init": (ctypes.c_int, [P(DecoderState), vp, u64]),
        "lmgc_decode_symbol": (ctypes.c_int, [P(DecoderState), vp, i32, P(i32)]),
        "lmgc_container_bound": (sz, [i64, P(SerialParams)]),
        "lmgc_codec_workspace": (sz, [vp, i64, P(SerialParams), i32]),
        "lmgc_compress": (ctypes.c_int, [vp, vp, i64, P(SerialParams), u32, i32, u64, i64, i64,
                                         vp, sz, vp, sz, P(sz), vp]),
        "lmgc_decode": (ctypes.c_int, [vp, vp, sz, i32, u64, vp, sz, vp, vp]),
        "lmgc_container_info": (ctypes.c_int, [vp, sz, P(i64), P(i32), P(i64), P(u64)]),
        "lmgc_op_gemm_bf16": (ctypes.c_int, [vp, vp, vp, i32, i32, i32, vp]),
        "lmgc_op_gemm_bf16_blocked": (ctypes.c_int, [vp, vp, vp, i32, i32, i32, i32, vp]),
        "lmgc_op_gemm_bf16_tile": (ctypes.c_int, [vp, vp, vp, i32, i32, i32, i32, i32, vp]),
        "lmgc_gemm_tile": (i32, [i32, i32, i32, i32]),
        "lmgc_op_gemm_f32": (ctypes.c_int, [vp, vp, vp, i32, i32, i32, vp]),
        "lmgc_op_block_weights": (ctypes.c_int, [vp, vp, i32, i32, vp]),
        "lmgc_op_attention_bf16": (ctypes.c_int, [vp, vp, vp, vp, i32, i32, i32, i32, i32, vp]),
        "lmgc_mx_code_bytes": (i64, [i32, i64, i64]),
        "lmgc_mx_scale_bytes": (i64, [i64, i64]),
        "lmgc_mx_block_code_bytes": (i64, [i64, i64]),
        "lmgc_mx_block_scale_bytes": (i64, [i64, i64]),
        "lmgc_op_mx_quantize": (ctypes.c_int, [vp, i32, i64, i64, i64, i32, vp, vp, vp]),
        "lmgc_op_mx_dequantize": (ctypes.c_int, [vp, vp, i32, i64, i64, vp, i32, i64, vp]),
        "lmgc_op_mx_block": (ctypes.c_int, [vp, vp, i64, i64, vp, vp, vp]),
        "lmgc_op_add_norm_mx": (ctypes.c_int, [vp, i32, vp, i32, vp, i32, ctypes.c_float, i64, i64, i32,
                                               vp, vp, vp, vp]),
        "lmgc_op_gemm_mx": (ctypes.c_int, [vp, vp, i32, vp, vp, vp, vp, i32, i32, i32, i32, vp]),
        "lmgc_op_gemm_mx_tile": (ctypes.c_int, [vp, vp, i32, vp, vp, vp, vp, i32, i32, i32, i32, i32, vp]),
        "lmgc_op_kv8_append": (ctypes.c_int, [vp, vp, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp]),
        "lmgc_kv8_workspace": (i64, [i32, i32, i32, i32, i32, i32]),
        "lmgc_op_attention_kv8": (ctypes.c_int, [vp, i32, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp,
                                                 i32, i32, vp, vp, sz, vp]),
        "lmgc_rope_frequencies": (ctypes.c_int, [f64, i32, i32, f64, f64, f64, f64, P(f64)]),
        "lmgc_op_rope_table": (ctypes.c_int, [P(f64), i32, f64, i64, vp, vp]),
        "lmgc_op_rope": (ctypes.c_int, [vp, i32, i64, i32, i32, i64, i64, vp, vp, i64, i32, i32, i32, vp, i64, i64, vp]),
        "lmgc_op_paged_append": (ctypes.c_int, [vp, vp, i32, i64, i64, i32, i32, i32, i32, vp, vp, i32, i32, vp, i32,
                                                vp, vp, vp, i64, i32, i32, vp, i64, i32, vp, i64, vp]),
        "lmgc_paged_workspace": (i64, [i32, i32, i32, i32, i32, i32, i32, i32]),
        "lmgc_op_attention_paged": (ctypes.c_int, [vp, i64, i32, i32, i32, i32, i32, vp, vp, i32, i32, vp, i32, vp, vp,
                                                   i32, i32, i32, i32, ctypes.c_float, vp, vp, sz, vp]),
        "lmgc_timing_enable": (ctypes.c_int, [i32]),
        "lmgc_timing_kinds": (ctypes.c_int, [u32]),
        "lmgc_timing_read": (ctypes.c_int, [i32, P(ctypes.c_double), P(i64)]),
        "lmgc_probs_flops": (ctypes.c_double, [vp, i32, i32, i32]),
    }
    for name, (res, args) in sig.items():
        f = getattr(L, name)
        f.restype = res
        f.argtypes = args
    _lib = L
    return L


def exported_symbols() -> List[str]:
    return [n for n in dir(lib()) if n.startswith("lmgc_")]


def _check(rc: int):
    if rc != LMGC_OK:
        raise LMGCError(rc, lib().lmgc_last_error().decode())


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, np.ndarray):
        return t.ctypes.data
    return t.data_ptr()


def _stream(stream=None):
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


# ------------------------------------------------------------ conversions --
def serial_params(spec) -> SerialParams:
    """From any object with the SerialParams field names (e.g. synth.SerialSpec)."""
    p = SerialParams()
    for f, _ in SerialParams._fields_:
        if f == "hex_ids":
            ids = list(spec.hex_ids)
            assert len(ids) == 16
            p.hex_ids = (ctypes.c_int32 * 16)(*ids)
        elif f == "sep2_id":
            p.sep2_id = int(getattr(spec, "sep2_id", -1))
        elif f == "renorm":
            p.renorm = int(getattr(spec, "renorm", 0))
        else:
            setattr(p, f, int(getattr(spec, f)))
    return p


def alphabet_size(sp: SerialParams) -> int:
    """Coded alphabet size A (17, or 18 with a second separator token)."""
    n = int(lib().lmgc_alphabet_size(ctypes.byref(sp)))
    if n < 0:
        raise LMGCError(-1, lib().lmgc_last_error().decode())
    return n


def model_config(shape) -> ModelConfig:
    """From any object with ModelShape fields (arch "llama"/"gpt2", dtype "f32"/"bf16")."""
    c = ModelConfig()
    c.arch = {"llama": 0, "gpt2": 1}[shape.arch]
    c.dtype = {"f32": 0, "bf16": 1}[shape.dtype]
    for f in ("n_layers", "d_model", "n_heads", "n_kv_heads", "d_ff", "vocab", "max_pos"):
        setattr(c, f, int(getattr(shape, f)))
    c.rope_theta = float(shape.rope_theta)
    c.norm_eps = float(shape.norm_eps)
    return c


# ---------------------------------------------------------- serialisation --
def num_tokens(n_values: int, sp: SerialParams) -> int:
    return int(lib().lmgc_num_tokens(n_values, ctypes.byref(sp)))


def num_windows(n_values: int, sp: SerialParams) -> int:
    return int(lib().lmgc_num_windows(n_values, ctypes.byref(sp)))


def serialize(values, sp: SerialParams, first_window: int = 0, n_windows: int = None,
              tokens=None, sym=None, want_sym: bool = True, stream=None):
    """values: 1-D CUDA tensor (float32 / uint8 / int16) -> (tokens [nw, W] int32, sym [nw, W] uint8)."""
    import torch
    n = values.numel()
    assert values.element_size() == sp.bytes_per_value and values.is_contiguous()
    if n_windows is None:
        n_windows = num_windows(n, sp) - first_window
    W = sp.window
    if tokens is None:
        tokens = torch.empty((n_windows, W), dtype=torch.int32, device=values.device)
    if sym is None and want_sym:
        sym = torch.empty((n_windows, W), dtype=torch.uint8, device=values.device)
    _check(lib().lmgc_serialize(_ptr(values), n, ctypes.byref(sp), first_window, n_windows,
                                _ptr(tokens), _ptr(sym), _stream(stream)))
    return tokens, sym


def deserialize(sym: np.ndarray, n_values: int, sp: SerialParams, dtype) -> np.ndarray:
    s = np.ascontiguousarray(sym, dtype=np.uint8)
    out = np.empty(n_values * sp.bytes_per_value, np.uint8)
    _check(lib().lmgc_deserialize(s.ctypes.data, s.size, n_values, ctypes.byref(sp),
                                  out.ctypes.data))
    return out.view(dtype)


# ------------------------------------------------------------ lossy steps --
def keep_count(n_values: int, percent: int) -> int:
    """Values sparsification keeps at `percent` percent (Sec. 5.4)."""
    k = int(lib().lmgc_keep_count(n_values, percent))
    if k < 0:
        _check(k)
    return k


def lossy_workspace(n_values: int) -> int:
    n = int(lib().lmgc_lossy_workspace(n_values))
    if n < 0:
        _check(n)
    return n


def sparsify_topk(values, k: int, out=None, ws=None, stream=None):
    """Keep the k largest-magnitude values of a CUDA float32 vector (Sec. 5.4);
    out may be values itself."""
    import torch
    assert values.dtype == torch.float32 and values.is_contiguous()
    n = values.numel()
    if out is None:
        out = torch.empty_like(values)
    if ws is None:
        ws = workspace(lossy_workspace(n), values.device)
    _check(lib().lmgc_sparsify_topk(_ptr(values), n, int(k), _ptr(out), _ptr(ws), ws.numel(),
                                    _stream(stream)))
    return out


def sparsify_topk_noalloc(values, k: int, out, stream=None):
    """sparsify_topk on the library's own device scratch: no workspace, and
    the call allocates nothing (out must be given; it may be values)."""
    import torch
    assert values.dtype == torch.float32 and values.is_contiguous()
    assert out.dtype == torch.float32 and out.numel() == values.numel()
    _check(lib().lmgc_sparsify_topk_noalloc(_ptr(values), values.numel(), int(k), _ptr(out),
                                            _stream(stream)))
    return out


def quantize_linear(values, bits: int, out=None, ws=None, stream=None):
    """Eq. 4 indices of a CUDA float32 vector -> (indices, min, max).  Indices
    are uint8 for bits <= 8, else int16 storage holding uint16 values."""
    import torch
    assert values.dtype == torch.float32 and values.is_contiguous()
    n = values.numel()
    if out is None:
        out = torch.empty(n, dtype=torch.uint8 if bits <= 8 else torch.int16, device=values.device)
    if ws is None:
        ws = workspace(lossy_workspace(n), values.device)
    mm = (ctypes.c_float * 2)()
    _check(lib().lmgc_quantize_linear(_ptr(values), n, int(bits), _ptr(out), mm, _ptr(ws), ws.numel(),
                                      _stream(stream)))
    return out, float(mm[0]), float(mm[1])


def sign_pack(values, out=None, stream=None):
    """SignSGD bits of a CUDA float32 vector, eight per byte, first value in bit 7."""
    import torch
    assert values.dtype == torch.float32 and values.is_contiguous()
    n = values.numel()
    if out is None:
        out = torch.empty((n + 7) // 8, dtype=torch.uint8, device=values.device)
    _check(lib().lmgc_sign_pack(_ptr(values), n, _ptr(out), _stream(stream)))
    return out


def lossy_prepare(values, steps, stream=None):
    """Apply lossy steps [(kind, arg)] left to right on the GPU: ("sparsify",
    percent), ("quantize", bits), ("sign", 0).  Returns the value stream."""
    x = values
    ws = None
    for kind, arg in steps:
        if kind == "sparsify":
            if ws is None:
                ws = workspace(lossy_workspace(x.numel()), x.device)
            x = sparsify_topk(x, keep_count(x.numel(), int(arg)), ws=ws, stream=stream)
        elif kind == "quantize":
            if ws is None:
                ws = workspace(lossy_workspace(x.numel()), x.device)
            x = quantize_linear(x, int(arg), ws=ws, stream=stream)[0]
        elif kind == "sign":
            x = sign_pack(x, stream=stream)
        else:
            raise ValueError(f"unknown lossy step {kind!r}")
    return x


# ------------------------------------------------------------------ model --
def manifest(cfg: ModelConfig) -> List[Tuple[str, Tuple[int, ...]]]:
    L = lib()
    n = L.lmgc_model_num_tensors(ctypes.byref(cfg))
    if n < 0:
        _check(-1)
    out = []
    name = ctypes.create_string_buffer(128)
    nd = ctypes.c_int32()
    shape = (ctypes.c_int64 * 2)()
    for i in range(n):
        _check(L.lmgc_model_tensor_info(ctypes.byref(cfg), i, name, 128, ctypes.byref(nd), shape))
        out.append((name.value.decode(), tuple(shape[:nd.value])))
    return out


class Model:
    """A decoder on the GPU.  weights: CUDA tensors in manifest order (bf16
    models: torch.bfloat16 or int16/uint16 bit patterns; f32: float32)."""

    def __init__(self, cfg: ModelConfig, weights: Sequence, stream=None):
        man = manifest(cfg)
        assert len(weights) == len(man), (len(weights), len(man))
        for (name, shape), w in zip(man, weights):
            assert tuple(w.shape) == tuple(shape), (name, tuple(w.shape), shape)
            assert w.is_contiguous()
        arr = (ctypes.c_void_p * len(man))(*[_ptr(w) for w in weights])
        h = ctypes.c_void_p()
        _check(lib().lmgc_model_create(ctypes.byref(cfg), arr, _stream(stream), ctypes.byref(h)))
        self.cfg = cfg
        self.handle = h

    def close(self):
        if self.handle:
            lib().lmgc_model_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def probs_workspace(self, B: int, W: int) -> int:
        return int(lib().lmgc_probs_workspace(self.handle, B, W))

    def step_workspace(self, B: int, W: int) -> int:
        return int(lib().lmgc_step_workspace(self.handle, B, W))

    def codec_workspace(self, n_values: int, sp: SerialParams, batch: int) -> int:
        return int(lib().lmgc_codec_workspace(self.handle, n_values, ctypes.byref(sp), batch))

    def flops(self, B: int, W: int, kind: str) -> float:
        return float(lib().lmgc_probs_flops(self.handle, B, W, KIND[kind]))


def workspace(nbytes: int, device="cuda"):
    import torch
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def probs(model: Model, tokens, sp: SerialParams, total: int = 1 << 16, want_logp: bool = True,
          ws=None, cdf=None, logp=None, stream=None):
    """tokens: CUDA int32 [B, W] -> (cdf int32 [B, W, A + 2] holding uint32 values,
    logp float32 [B, W, A]) with A = alphabet_size(sp)."""
    import torch
    B, W = tokens.shape
    assert tokens.dtype == torch.int32 and tokens.is_contiguous()
    na = alphabet_size(sp)
    need = model.probs_workspace(B, W)
    if ws is None:
        ws = workspace(need, tokens.device)
    if cdf is None:
        cdf = torch.empty((B, W, na + 2), dtype=torch.int32, device=tokens.device)
    if logp is None and want_logp:
        logp = torch.empty((B, W, na), dtype=torch.float32, device=tokens.device)
    _check(lib().lmgc_probs(model.handle, _ptr(tokens), B, W, ctypes.byref(sp), total, _ptr(cdf),
                            _ptr(logp), _ptr(ws), ws.numel(), _stream(stream)))
    return cdf, logp


def probs_stepwise(model: Model, tokens, sp: SerialParams, total: int = 1 << 16,
                   want_logp: bool = True, ws=None, stream=None):
    """lmgc_probs_stepwise: the same outputs as probs(), computed position by
    position through the K/V cache (the decoder's path); B <= 32."""
    import torch
    B, W = tokens.shape
    assert tokens.dtype == torch.int32 and tokens.is_contiguous()
    na = alphabet_size(sp)
    if ws is None:
        ws = workspace(model.step_workspace(B, W), tokens.device)
    cdf = torch.empty((B, W, na + 2), dtype=torch.int32, device=tokens.device)
    logp = torch.empty((B, W, na), dtype=torch.float32, device=tokens.device) if want_logp else None
    _check(lib().lmgc_probs_stepwise(model.handle, _ptr(tokens), B, W, ctypes.byref(sp), total,
                                     _ptr(cdf), _ptr(logp), _ptr(ws), ws.numel(), _stream(stream)))
    return cdf, logp


# ------------------------------------------------------------------ coder --
def encode(cdf: np.ndarray, sym: np.ndarray, lens: np.ndarray, n_threads: int = 0):
    """cdf [n_win, W, nsym+1] uint32, sym [n_win, W] uint8, lens [n_win] -> (payloads bytes, bits uint32[n_win])."""
    cdf = np.ascontiguousarray(cdf, dtype=np.uint32)
    sym = np.ascontiguousarray(sym, dtype=np.uint8)
    lens = np.ascontiguousarray(lens, dtype=np.int32)
    n_win, W = sym.shape
    nsym = cdf.shape[-1] - 1
    cap = int(lib().lmgc_encode_bound(n_win, W))
    out = np.empty(max(cap, 1), np.uint8)
    bits = np.zeros(n_win, np.uint32)
    used = ctypes.c_size_t()
    _check(lib().lmgc_encode(cdf.ctypes.data, nsym, sym.ctypes.data, lens.ctypes.data, n_win, W,
                             out.ctypes.data, cap, bits.ctypes.data, ctypes.byref(used), n_threads))
    return out[:used.value].tobytes(), bits


class StepDecoder:
    def __init__(self, payload: bytes, nbits: int):
        self._buf = np.frombuffer(payload, np.uint8).copy() if len(payload) else np.zeros(1, np.uint8)
        self._st = DecoderState()
        _check(lib().lmgc_decode_init(ctypes.byref(self._st), self._buf.ctypes.data, nbits))

    def decode(self, cdf_row: np.ndarray) -> int:
        row = np.ascontiguousarray(cdf_row, dtype=np.uint32)
        out = ctypes.c_int32()
        _check(lib().lmgc_decode_symbol(ctypes.byref(self._st), row.ctypes.data, row.size - 1,
                                        ctypes.byref(out)))
        return out.value


# ------------------------------------------------------------------ codec --
def compress(model: Model, values, sp: SerialParams, total: int = 1 << 16, batch: int = 8,
             model_tag: int = 0, first_window: int = 0, n_windows: int = -1, ws=None,
             stream=None) -> bytes:
    n = values.numel()
    nw = num_windows(n, sp)
    cnt = (nw - first_window) if n_windows < 0 else n_windows
    cap = 128 + 4 * cnt + int(lib().lmgc_encode_bound(max(cnt, 1), sp.window))
    out = np.empty(cap, np.uint8)
    if ws is None:
        ws = workspace(model.codec_workspace(n, sp, batch), values.device)
    used = ctypes.c_size_t()
    _check(lib().lmgc_compress(model.handle, _ptr(values), n, ctypes.byref(sp), total, batch,
                               model_tag, first_window, n_windows, _ptr(ws), ws.numel(),
                               out.ctypes.data, cap, ctypes.byref(used), _stream(stream)))
    return out[:used.value].tobytes()


def container_info(buf: bytes):
    a = np.frombuffer(buf, np.uint8)
    nv, bpv, nw, tag = ctypes.c_int64(), ctypes.c_int32(), ctypes.c_int64(), ctypes.c_uint64()
    _check(lib().lmgc_container_info(a.ctypes.data, a.size, ctypes.byref(nv), ctypes.byref(bpv),
                                     ctypes.byref(nw), ctypes.byref(tag)))
    return dict(n_values=nv.value, bytes_per_value=bpv.value, n_windows=nw.value,
                model_tag=tag.value)


def decode(model: Model, buf: bytes, batch: int = 8, model_tag: int = 0, ws=None,
           stream=None, dtype=np.float32) -> np.ndarray:
    info = container_info(buf)
    a = np.frombuffer(buf, np.uint8).copy()
    out = np.empty(info["n_values"] * info["bytes_per_value"], np.uint8)
    W = int.from_bytes(buf[28:32], "little")
    sp = SerialParams()
    sp.window = W
    if ws is None:
        ws = workspace(model.codec_workspace(info["n_values"], sp, batch))
    _check(lib().lmgc_decode(model.handle, a.ctypes.data, a.size, batch, model_tag, _ptr(ws),
                             ws.numel(), out.ctypes.data, _stream(stream)))
    return out.view(dtype)


# ----------------------------------------------------------- kernel level --
def op_gemm_bf16(a, b, c=None, stream=None):
    """a [M, K], b [N, K] bf16 CUDA tensors -> c [M, N] float32 = a b^T."""
    import torch
    M, K = a.shape
    N = b.shape[0]
    if c is None:
        c = torch.empty((M, N), dtype=torch.float32, device=a.device)
    _check(lib().lmgc_op_gemm_bf16(_ptr(a), _ptr(b), _ptr(c), M, N, K, _stream(stream)))
    return c


def op_gemm_f32(a, b, stream=None):
    """a [M, K], b [N, K] float32 CUDA tensors -> [M, N] float32 = a b^T."""
    import torch
    M, K = a.shape
    N = b.shape[0]
    c = torch.empty((M, N), dtype=torch.float32, device=a.device)
    _check(lib().lmgc_op_gemm_f32(_ptr(a), _ptr(b), _ptr(c), M, N, K, _stream(stream)))
    return c


OP_KINDS = {"store": 0, "resid": 1, "swiglu": 2}
TILES = ["32x32", "64x64", "128x64", "128x128", "256x128", "256x256"]


def gemm_tile(M: int, N: int, K: int, head: bool = False) -> str:
    """The tile the library takes for a bf16 product of whole windows."""
    t = int(lib().lmgc_gemm_tile(int(head), M, N, K))
    if t < 0:
        _check(t)
    return TILES[t]


def op_block_weights(b, stream=None):
    """b [N, K] bf16 CUDA tensor (row-major) -> the same matrix in MFMA blocks."""
    import torch
    N, K = b.shape
    out = torch.empty_like(b)
    _check(lib().lmgc_op_block_weights(_ptr(b), _ptr(out), N, K, _stream(stream)))
    return out


def op_gemm_bf16_blocked(a, b_blocked, kind: str, out=None, stream=None, tile: str = None):
    """The model's blocked-weight product with its epilogue: "store" (float32
    [M, N] = a b^T), "resid" (out += a b^T; out given), "swiglu" (bf16
    [M, N/2], b's rows gate/up interleaved in groups of 32).  tile: one of
    TILES instead of the library's choice."""
    import torch
    M, K = a.shape
    N = b_blocked.shape[0]
    if out is None:
        out = (torch.empty((M, N // 2), dtype=torch.bfloat16, device=a.device) if kind == "swiglu"
               else torch.zeros((M, N), dtype=torch.float32, device=a.device))
    _check(lib().lmgc_op_gemm_bf16_tile(_ptr(a), _ptr(b_blocked), _ptr(out), M, N, K, OP_KINDS[kind],
                                        -1 if tile is None else TILES.index(tile), _stream(stream)))
    return out


def op_attention_bf16(q, k, vt, o=None, stream=None):
    """q [B, Hq, W, hd], k [B, Hkv, W, hd], vt = V transposed [B, Hkv, hd, W],
    all bf16 -> o [B*W, Hq*hd] bf16."""
    import torch
    B, Hq, W, hd = q.shape
    Hkv = k.shape[1]
    if o is None:
        o = torch.empty((B * W, Hq * hd), dtype=torch.bfloat16, device=q.device)
    _check(lib().lmgc_op_attention_bf16(_ptr(q), _ptr(k), _ptr(vt), _ptr(o), B, Hq, Hkv, W, hd,
                                        _stream(stream)))
    return o


# ------------------------------------------- decoder steps in fewer bits --
MX_FORMATS = {"fp8": 0, "fp4": 1}


def _size(n: int) -> int:
    if n < 0:
        _check(n)
    return int(n)


def _dtype(t) -> int:
    """LMGC_DTYPE_* of a float32 or bfloat16 tensor."""
    import torch
    assert t.dtype in (torch.float32, torch.bfloat16), t.dtype
    return 1 if t.dtype == torch.bfloat16 else 0


_cuda = None  # (current device, its current stream's handle): torch's own calls without the objects around them


def _cuda_calls():
    global _cuda
    if _cuda is None:
        import torch
        dev = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        _cuda = dev, raw or (lambda d: torch.cuda.current_stream(d).cuda_stream)
    return _cuda


def _on(stream, *tensors):
    """The stream to launch on (the current one unless given) and the tensors'
    addresses.  Every tensor has to be on the current device, as for every call
    of the library."""
    current, raw = _cuda_calls()
    dev = current()
    at = []
    for t in tensors:
        if t is None:
            at.append(None)
            continue
        if t.get_device() != dev:
            raise ValueError(f"a tensor is on {t.device}, the current device is cuda:{dev}")
        at.append(t.data_ptr())
    if stream is None:
        return raw(dev), at
    if stream.device_index != dev:
        raise ValueError(f"a stream of cuda:{stream.device_index}, the current device is cuda:{dev}")
    return stream.cuda_stream, at


def _empty(shape, dtype, like, stream):
    """A tensor on like's device that is free for `stream` to write: with a stream
    other than the current one it is allocated there, as torch.cuda.stream(stream)
    would."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    import torch
    with torch.cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


def _mx_sizes(rows: int, cols: int, fmt: str) -> Tuple[int, int]:
    """Bytes of a row's codes and scales (lmgc_mx_code_bytes, lmgc_mx_scale_bytes)."""
    kp = -(-cols // 128) * 128
    return kp if MX_FORMATS[fmt] == 0 else kp // 2, 16 * -(-cols // 512)


def _mx_empty(rows, cols, fmt, codes, scales, like, stream):
    """Code and scale tensors of the rows layout: uint8 [rows, bytes of a row]."""
    import torch
    nc, ns = _mx_sizes(rows, cols, fmt)
    if codes is None:
        codes = _empty((rows, nc), torch.uint8, like, stream)
    else:
        assert codes.dtype == torch.uint8 and codes.is_contiguous() and codes.numel() == rows * nc, (tuple(codes.shape), rows, cols, fmt)
    if scales is None:
        scales = _empty((rows, ns), torch.uint8, like, stream)
    else:
        assert scales.dtype == torch.uint8 and scales.is_contiguous() and scales.numel() == rows * ns, (tuple(scales.shape), rows, cols)
    return codes, scales


def _mx_check(codes, scales, rows, cols, fmt):
    assert codes is not None and scales is not None
    _mx_empty(rows, cols, fmt, codes, scales, None, None)


def op_mx_quantize(x, fmt: str, codes=None, scales=None, stream=None):
    """x [rows, cols] float32 or bf16 CUDA tensor (rows may be strided) ->
    (codes uint8 [rows, Kp or Kp / 2], scales uint8 [rows, 16 ceil(cols / 512)]),
    fmt "fp8" (e4m3) or "fp4" (e2m1)."""
    rows, cols = x.shape
    assert cols == 1 or x.stride(1) == 1
    codes, scales = _mx_empty(rows, cols, fmt, codes, scales, x, stream)
    ld = x.stride(0) if rows > 1 else cols
    st, (px, pc, ps) = _on(stream, x, codes, scales)
    _check(lib().lmgc_op_mx_quantize(px, _dtype(x), rows, cols, ld, MX_FORMATS[fmt], pc, ps, st))
    return codes, scales


def op_mx_dequantize(codes, scales, fmt: str, cols: int, dtype=None, out=None, stream=None):
    """The values of a microscaled matrix: float32 (or dtype=torch.bfloat16) [rows, cols]."""
    import torch
    rows = codes.shape[0]
    _mx_check(codes, scales, rows, cols, fmt)
    if out is None:
        out = _empty((rows, cols), dtype or torch.float32, codes, stream)
    assert out.shape == (rows, cols) and (cols == 1 or out.stride(1) == 1)
    ld = out.stride(0) if rows > 1 else cols
    st, (pc, ps, po) = _on(stream, codes, scales, out)
    _check(lib().lmgc_op_mx_dequantize(pc, ps, MX_FORMATS[fmt], rows, cols, po, _dtype(out), ld, st))
    return out


def op_mx_block(codes, scales, cols: int, stream=None):
    """4-bit weights from the rows layout -> (codes, scales) in blocks, flat uint8."""
    import torch
    rows = codes.shape[0]
    _mx_check(codes, scales, rows, cols, "fp4")
    bc = _empty(_size(lib().lmgc_mx_block_code_bytes(rows, cols)), torch.uint8, codes, stream)
    bs = _empty(_size(lib().lmgc_mx_block_scale_bytes(rows, cols)), torch.uint8, codes, stream)
    st, (pc, ps, pbc, pbs) = _on(stream, codes, scales, bc, bs)
    _check(lib().lmgc_op_mx_block(pc, ps, rows, cols, pbc, pbs, st))
    return bc, bs


def op_add_norm_mx(h, x, gain, eps: float, fmt: str, out=None, codes=None, scales=None, stream=None):
    """t = h + x (x may be None), RMSNorm of t times gain, microscaled: h and x
    [M, d] float32 or bf16 -> (codes, scales); t goes to `out` (h itself: in
    place; None: not stored)."""
    M, d = h.shape
    assert h.is_contiguous() and gain.is_contiguous() and gain.numel() == d
    assert x is None or (x.is_contiguous() and x.shape == (M, d))
    assert out is None or (out.is_contiguous() and out.shape == (M, d) and out.dtype == h.dtype)
    codes, scales = _mx_empty(M, d, fmt, codes, scales, h, stream)
    st, (ph, px, pg, po, pc, ps) = _on(stream, h, x, gain, out, codes, scales)
    _check(lib().lmgc_op_add_norm_mx(ph, _dtype(h), px, _dtype(x) if x is not None else 0, pg, _dtype(gain), float(eps),
                                     M, d, MX_FORMATS[fmt], po, pc, ps, st))
    return codes, scales


MX_KINDS = {"store": 0, "bf16": 3}
MX_TILES = ("16x16", "16x32", "16x64", "64x64", "128x64", "128x128", "128x256", "256x256")  # LMGC_MX_TILE_*


def op_gemm_mx(a, a_scales, a_fmt: str, b, b_scales, N: int, K: int, kind: str = "store", add=None, out=None,
               tile: str = None, stream=None):
    """a (rows layout, "fp8" or "fp4") times the 4-bit weights b [N, K] (blocks
    layout), transposed -> [M, N] float32 ("store") or bf16 ("bf16"), plus the
    float32 `add` [M, N] if given (out may be add).  tile (MX_TILES): the tile
    of the output, for comparing them; by itself the library takes one by shape."""
    import torch
    M = a.shape[0]
    _mx_check(a, a_scales, M, K, a_fmt)
    nc, ns = _mx_sizes(N, K, "fp4")
    n16 = -(-N // 16) * 16
    assert b.dtype == torch.uint8 and b.is_contiguous() and b.numel() == n16 * nc
    assert b_scales.dtype == torch.uint8 and b_scales.is_contiguous() and b_scales.numel() == n16 * ns
    dt = torch.bfloat16 if kind == "bf16" else torch.float32
    if out is None:
        out = _empty((M, N), dt, a, stream)
    else:
        assert out.dtype == dt and out.is_contiguous() and out.shape == (M, N)
    if add is not None:
        assert add.dtype == torch.float32 and add.is_contiguous() and add.shape == (M, N)
    st, (pa, psa, pb, psb, padd, po) = _on(stream, a, a_scales, b, b_scales, add, out)
    _check(lib().lmgc_op_gemm_mx_tile(pa, psa, MX_FORMATS[a_fmt], pb, psb, padd, po, M, N, K, MX_KINDS[kind],
                                      -1 if tile is None else MX_TILES.index(tile), st))
    return out


def kv8_cache(B: int, Hkv: int, cap: int, hd: int, device="cuda"):
    """An empty 8-bit key/value cache of one layer: (key codes, key scales,
    value codes, value scales)."""
    import torch
    assert cap % 64 == 0
    return tuple(t for _ in range(2) for t in
                 (torch.zeros((B, Hkv, cap // 64, 64 * hd), dtype=torch.uint8, device=device),
                  torch.ones((B, Hkv, cap // 64), dtype=torch.float32, device=device)))


def _kv8_check(cache, B, Hkv, hd):
    """The cache's tokens, its tensors checked."""
    import torch
    kc, ks, vc, vs = cache
    n = kc.shape[2]
    assert kc.dtype == vc.dtype == torch.uint8 and kc.shape == vc.shape == (B, Hkv, n, 64 * hd)
    assert ks.dtype == vs.dtype == torch.float32 and ks.shape == vs.shape == (B, Hkv, n)
    assert kc.is_contiguous() and ks.is_contiguous() and vc.is_contiguous() and vs.is_contiguous()
    return 64 * n


def _kv8_lens(lens, counts, B):
    import torch
    assert lens.dtype == torch.int32 and lens.is_contiguous() and lens.numel() == B
    assert counts is None or (counts.dtype == torch.int32 and counts.is_contiguous() and counts.numel() == B)


def op_kv8_append(cache, k, v, lens, counts=None, stream=None):
    """Stores k, v (bf16 [B, Hkv, T, hd]) at positions lens[b] .. of each
    sequence (lens, counts: CUDA int32 [B])."""
    import torch
    B, Hkv, T, hd = k.shape
    cap = _kv8_check(cache, B, Hkv, hd)
    assert k.dtype == v.dtype == torch.bfloat16 and k.is_contiguous() and v.is_contiguous() and v.shape == k.shape
    _kv8_lens(lens, counts, B)
    st, (pk, pv, *rest) = _on(stream, k, v, lens, counts, *cache)
    _check(lib().lmgc_op_kv8_append(pk, pv, B, Hkv, T, hd, cap, *rest, st))


def kv8_workspace(B: int, Hq: int, Hkv: int, T: int, hd: int, cap: int) -> int:
    return _size(lib().lmgc_kv8_workspace(B, Hq, Hkv, T, hd, cap))


def op_attention_kv8(q, cache, lens, counts=None, window: int = 0, sinks: int = 0, out=None, ws=None, stream=None):
    """Attention of the T tokens just appended over the 8-bit cache: q bf16
    [B, Hq, T, hd] -> bf16 [B T, Hq hd].  window, sinks: any size (ctypes would
    keep the low 32 bits of a larger one)."""
    import torch
    B, Hq, T, hd = q.shape
    Hkv = cache[0].shape[1]
    cap = _kv8_check(cache, B, Hkv, hd)
    assert q.dtype == torch.bfloat16 and q.is_contiguous()
    _kv8_lens(lens, counts, B)
    if out is None:
        out = _empty((B * T, Hq * hd), torch.bfloat16, q, stream)
    else:
        assert out.dtype == torch.bfloat16 and out.is_contiguous() and out.numel() == q.numel()
    if ws is None:
        ws = _empty(kv8_workspace(B, Hq, Hkv, T, hd, cap), torch.uint8, q, stream)
    else:
        assert ws.is_contiguous()  # its bytes lie one behind the other
    st, (pq, po, pw, *rest) = _on(stream, q, out, ws, lens, counts, *cache)
    window, sinks = int(window), int(sinks)
    if not (0 <= window < 2 ** 31 and 0 <= sinks < 2 ** 31):
        window, sinks = max(-1, min(window, 2 ** 31 - 1)), max(-1, min(sinks, 2 ** 31 - 1))
    _check(lib().lmgc_op_attention_kv8(pq, B, Hq, Hkv, T, hd, cap, *rest, window, sinks, po, pw,
                                       ws.numel() * ws.element_size(), st))
    return out


# ----------------------------------------- ragged batches over a paged cache --
ROPE_LAYOUTS = {"half": 0, "interleaved": 1}
ROPE_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3}


def _int32(x):
    """A size for the library: the nearest of [-1, 2^31) (ctypes would keep the low 32
    bits of another), and it refuses what it does not take."""
    return max(-1, min(int(x), 2 ** 31 - 1))


def rope_frequencies(rot: int, theta: float = 10000.0, scaling: str = "none", factor: float = 1.0, orig: float = 4096,
                     slow: float = 1.0, fast: float = 32.0) -> np.ndarray:
    """float64 [rot / 2]: the frequencies of lmgc_rope_frequencies."""
    return np.array(_frequencies(rot, theta, scaling, factor, orig, slow, fast))


def _frequencies(rot, theta, scaling, factor, orig, slow, fast):
    rot = _int32(rot)
    out = (ctypes.c_double * max(min(rot, 512) // 2, 1))()  # (no rot past 512 is taken)
    _check(lib().lmgc_rope_frequencies(float(theta), rot, ROPE_SCALINGS[scaling], float(factor), float(orig), float(slow),
                                       float(fast), out))
    return out


def rope_table(n_pos: int, rot: int, theta: float = 10000.0, scaling: str = "none", factor: float = 1.0, orig: float = 4096,
               slow: float = 1.0, fast: float = 32.0, mscale: float = None, out=None, stream=None):
    """(cos, sin) of positions 0 .. n_pos - 1: float32 CUDA tensor [n_pos, rot / 2,
    2].  mscale multiplies both; YaRN's 0.1 ln(factor) + 1 with that scaling
    unless given, else 1."""
    import torch
    f = _frequencies(rot, theta, scaling, factor, orig, slow, fast)
    if mscale is None:
        mscale = 0.1 * math.log(factor) + 1.0 if scaling == "yarn" else 1.0
    shape = (n_pos, rot // 2, 2)
    if out is None:
        if stream is None:
            out = torch.empty(shape, dtype=torch.float32, device="cuda")
        else:
            with torch.cuda.stream(stream):
                out = torch.empty(shape, dtype=torch.float32, device="cuda")
    else:
        assert out.dtype == torch.float32 and out.is_contiguous() and out.shape == shape
    st, (po,) = _on(stream, out)
    _check(lib().lmgc_op_rope_table(f, rot, float(mscale), n_pos, po, st))
    return out


def _rope_check(table):
    """Positions and dims of a table."""
    import torch
    assert table.dtype == torch.float32 and table.is_contiguous() and table.dim() == 3 and table.shape[2] == 2
    return table.shape[0], 2 * table.shape[1]


def op_rope(x, positions, table, layout: str = "half", backward: bool = False, out=None, stream=None):
    """Rotates x [n, heads, hd] (float32 or bf16 CUDA tensor, any strides of rows
    and heads) by the table's row of each position (CUDA int32 [n]); backward: the
    transpose.  The result goes to `out` (x itself: in place; None: a new tensor,
    whose rows at positions outside the table hold anything)."""
    import torch
    n, heads, hd = x.shape
    n_pos, rot = _rope_check(table)
    assert positions.dtype == torch.int32 and positions.is_contiguous() and positions.numel() == n
    if out is None:
        out = _empty((n, heads, hd), x.dtype, x, stream)
    else:
        assert out.dtype == x.dtype and out.shape == x.shape
    assert x.stride(2) == 1 and out.stride(2) == 1
    dt = _dtype(x)

    def strides(t):  # of a single row or head: what a contiguous tensor has
        rows, h, _ = t.stride()
        h = h if heads > 1 else hd
        return (rows if n > 1 else heads * h), h
    st, (px, pp, pt, po) = _on(stream, x, positions, table, out)
    _check(lib().lmgc_op_rope(px, dt, n, heads, hd, *strides(x), pp, pt, n_pos, rot, ROPE_LAYOUTS[layout],
                              int(backward), po, *strides(out), st))
    return out


def paged_cache(n_pages: int, Hkv: int, page: int, hd: int, device="cuda"):
    """An empty paged key/value cache of one layer: (keys, values), bf16 [n_pages,
    Hkv, page, hd] in the order of lmgc.h."""
    import torch
    return tuple(torch.zeros((n_pages, Hkv, page, hd), dtype=torch.bfloat16, device=device) for _ in range(2))


def _paged_check(cache, pages, starts, lens, Hkv, hd):
    """(n_pages, page, B, max_pages) of a cache and a batch, their tensors checked."""
    import torch
    kc, vc = cache
    shape, i32 = kc.shape, torch.int32
    assert kc.dtype == vc.dtype == torch.bfloat16 and shape == vc.shape and kc.is_contiguous() and vc.is_contiguous()
    assert len(shape) == 4 and shape[1] == Hkv and shape[3] == hd, (tuple(shape), Hkv, hd)
    B, most = pages.shape
    assert pages.dtype == i32 and pages.is_contiguous()
    assert starts.dtype == i32 and starts.is_contiguous() and starts.numel() == B + 1
    assert lens.dtype == i32 and lens.is_contiguous() and lens.numel() == B
    return shape[0], shape[2], B, most


def _row_stride(t):
    """Numbers between rows of t [n, heads, hd], whose heads lie side by side."""
    n, heads, hd = t.shape
    rows, of_heads, dims = t.stride()
    assert dims == 1 and (heads == 1 or of_heads == hd), t.stride()
    return rows if n > 1 else heads * hd


def op_paged_append(cache, k, v, pages, starts, lens, rope=None, layout: str = "half", q=None, q_out=None, stream=None):
    """Stores k, v [n, Hkv, hd] (float32 or bf16, rows may be strided) of a ragged
    batch (pages [B, max_pages], starts [B + 1], lens [B]: CUDA int32), k rotated
    by the table `rope` if given.  q [n, Hq, hd]: rotated too, into q_out (a new
    bf16 tensor, rows of no token left as they are, unless given), which is
    returned."""
    import torch
    n, Hkv, hd = k.shape
    n_pages, page, B, most = _paged_check(cache, pages, starts, lens, Hkv, hd)
    assert v.shape == k.shape and v.dtype == k.dtype
    n_pos, rot = _rope_check(rope) if rope is not None else (0, 0)
    Hq, ldq, ldqo, ldk, ldv = 0, 0, 0, _row_stride(k), _row_stride(v)
    if q is not None:
        Hq = q.shape[1]
        assert q.dtype == k.dtype and q.shape == (n, Hq, hd)
        if q_out is None:
            q_out = _empty((n, Hq, hd), torch.bfloat16, q, stream)
        assert q_out.dtype == torch.bfloat16 and q_out.shape == q.shape
        ldq, ldqo = _row_stride(q), _row_stride(q_out)
    else:
        assert q_out is None
    st, (pk, pv, pq, pqo, pr, pp, ps, pl, pkc, pvc) = _on(stream, k, v, q, q_out, rope, pages, starts, lens, *cache)
    _check(lib().lmgc_op_paged_append(pk, pv, _dtype(k), ldk, ldv, n, B, Hkv, hd, pkc, pvc, n_pages,
                                      page, pp, most, ps, pl, pr, n_pos, rot, ROPE_LAYOUTS[layout], pq, ldq, Hq, pqo, ldqo, st))
    return q_out


def paged_workspace(n: int, B: int, Hq: int, Hkv: int, hd: int, max_new: int, tokens: int, shared: int = 0) -> int:
    return _size(lib().lmgc_paged_workspace(*map(_int32, (n, B, Hq, Hkv, hd, max_new, tokens, shared))))


def op_attention_paged(q, cache, pages, starts, lens, max_new: int, window: int = 0, sinks: int = 0, shared: int = 0,
                       scale: float = None, out=None, ws=None, stream=None):
    """Attention of the tokens just appended over the paged cache: q bf16 [n, Hq,
    hd] (rows may be strided) -> bf16 [n, Hq hd].  max_new: the most new tokens
    that a sequence has; shared: leading tokens that all sequences have in common;
    scale: 1 / sqrt(hd) unless given."""
    import torch
    n, Hq, hd = q.shape
    Hkv = cache[0].shape[1]
    n_pages, page, B, most = _paged_check(cache, pages, starts, lens, Hkv, hd)
    assert q.dtype == torch.bfloat16
    ldq = _row_stride(q)
    if out is None:
        out = _empty((n, Hq * hd), torch.bfloat16, q, stream)
    else:
        assert out.dtype == torch.bfloat16 and out.is_contiguous() and out.numel() == q.numel()
    if not (0 <= max_new <= 1 << 24 and 0 <= window < 1 << 31 and 0 <= sinks < 1 << 31 and 0 <= shared < 1 << 31):
        max_new, window, sinks, shared = map(_int32, (max_new, window, sinks, shared))
        max_new = min(max_new, 1 << 24)
    if ws is None:
        ws = _empty(paged_workspace(n, B, Hq, Hkv, hd, max_new, most * page, shared), torch.uint8, q, stream)
    else:
        assert ws.is_contiguous()  # its bytes lie one behind the other
    st, (pq, pkc, pvc, pp, ps, pl, po, pw) = _on(stream, q, *cache, pages, starts, lens, out, ws)
    _check(lib().lmgc_op_attention_paged(pq, ldq, n, B, Hq, Hkv, hd, pkc, pvc, n_pages, page, pp, most, ps, pl,
                                         max_new, window, sinks, shared,
                                         hd ** -0.5 if scale is None else float(scale), po, pw,
                                         ws.numel() * ws.element_size(), st))
    return out


# ----------------------------------------------------------------- timing --
def timing_enable(on: bool = True):
    _check(lib().lmgc_timing_enable(1 if on else 0))


def timing_kinds(kinds=None):
    """lmgc_timing_kinds: record events only for these kinds (None: all)."""
    names = list(KIND) if kinds is None else list(kinds)
    mask = 0
    for k in names:
        mask |= 1 << KIND[k]
    _check(lib().lmgc_timing_kinds(mask))


def timing_read(kind: str) -> Tuple[float, int]:
    ms, n = ctypes.c_double(), ctypes.c_int64()
    _check(lib().lmgc_timing_read(KIND[kind], ctypes.byref(ms), ctypes.byref(n)))
    return ms.value, n.value
