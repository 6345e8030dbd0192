"""Thin ctypes binding of libpwdec.so (include/pwdec.h).

Argument marshalling only: every step of the decoder runs in the library's HIP kernels.
Device buffers are torch tensors on the decoder's GPU; torch supplies memory and streams.
"""
from __future__ import annotations

import ctypes
import os
import re
import struct

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libpwdec.so")
HEADER = os.path.join(os.path.dirname(HERE), "include", "pwdec.h")

PWD_OK, PWD_EINVAL, PWD_EUNSUPPORTED, PWD_EBLOB, PWD_ENOMEM, PWD_EHIP, PWD_EBATCH, PWD_EDEVICE = (
    0, -1, -2, -3, -4, -5, -6, -7)
DTYPE_F32, DTYPE_BF16, DTYPE_MXFP8 = 0, 1, 2
BLOB_MAGIC = 0x31445750
BLOB_VERSION = 1


class PwdError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"pwdec error {code}: {msg}")
        self.code = code


class Geometry(ctypes.Structure):
    _fields_ = [("distance", ctypes.c_int32), ("window_rounds", ctypes.c_int32),
                ("max_windows", ctypes.c_int32)]


class ModelDims(ctypes.Structure):
    _fields_ = [("d_model", ctypes.c_int32), ("n_layers", ctypes.c_int32), ("n_heads", ctypes.c_int32),
                ("mlp_ratio", ctypes.c_int32), ("dtype", ctypes.c_int32), ("token_set", ctypes.c_int32),
                ("embedder", ctypes.c_int32), ("conv_dilation", ctypes.c_int32 * 3)]


class RotaryDims(ctypes.Structure):
    _fields_ = [("pairs", ctypes.c_int32 * 2), ("theta", ctypes.c_float), ("qk_norm", ctypes.c_int32),
                ("norm_eps", ctypes.c_float), ("window", ctypes.c_int32), ("sinks", ctypes.c_int32)]


def rotary_dims(pairs=(0, 0), theta: float = 10000.0, qk_norm: bool = False, norm_eps: float = 1e-6, window: int = -1,
                sinks: int = 0) -> RotaryDims:
    """Attention options of a rotary network (decoder_create_rotary): feature pairs of a head turned by the
    token's lattice row and column, RMS norm of Q and K heads, window of tokens and sinks."""
    return RotaryDims((ctypes.c_int32 * 2)(*pairs), theta, int(qk_norm), norm_eps, window, sinks)


NUM_STAGES = 12
STAGE_NAMES = ["embed_qkv", "attention", "post_qkv", "post_embed_qkv", "post", "readout", "fp32_window",
               "stream_split", "stream_combine", "out_proj", "dilated_conv", "resident"]
SCHEDULE_AUTO, SCHEDULE_LAYERS, SCHEDULE_RESIDENT = 0, 1, 2


class StageTimes(ctypes.Structure):
    _fields_ = [("ms", ctypes.c_double * NUM_STAGES), ("launches", ctypes.c_int64 * NUM_STAGES)]


class LinearArgs(ctypes.Structure):
    _fields_ = [("m", ctypes.c_int64), ("n", ctypes.c_int64), ("k", ctypes.c_int64),
                ("d_x", ctypes.c_void_p), ("ld_x", ctypes.c_int64), ("d_w", ctypes.c_void_p), ("ld_w", ctypes.c_int64),
                ("d_bias", ctypes.c_void_p), ("d_residual", ctypes.c_void_p), ("ld_residual", ctypes.c_int64),
                ("d_y", ctypes.c_void_p), ("ld_y", ctypes.c_int64),
                ("dtype", ctypes.c_int32), ("out_dtype", ctypes.c_int32), ("activation", ctypes.c_int32),
                ("d_workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


class RopeArgs(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("q_heads", ctypes.c_int32), ("k_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32)] + \
        [f for t in ("q", "k", "q_out", "k_out")
         for f in ((f"d_{t}", ctypes.c_void_p), (f"{t}_token_stride", ctypes.c_int64), (f"{t}_head_stride", ctypes.c_int64))] + \
        [("d_positions", ctypes.c_void_p), ("axes", ctypes.c_int32), ("pairs", ctypes.c_int32 * 3),
         ("layout", ctypes.c_int32), ("frequencies", ctypes.c_int32), ("inverse", ctypes.c_int32),
         ("theta", ctypes.c_double)]


class AttentionArgs(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("q_len", ctypes.c_int64), ("k_len", ctypes.c_int64),
                ("q_heads", ctypes.c_int32), ("k_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32)] + \
        [f for t, s in (("d_q", "q"), ("d_k", "k"), ("d_v", "v"), ("d_out", "out"))
         for f in ((t, ctypes.c_void_p), (f"{s}_stride", ctypes.c_int64 * 3))] + \
        [("d_q_lengths", ctypes.c_void_p), ("d_k_lengths", ctypes.c_void_p), ("window_left", ctypes.c_int64),
         ("window_right", ctypes.c_int64), ("sinks", ctypes.c_int64), ("scale", ctypes.c_double),
         ("d_workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


_lib = None


def load_library() -> ctypes.CDLL:
    """Loads the in-tree libpwdec.so; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with paper_2601_09921_amd.build.build()")
    _lib = bind(ctypes.CDLL(LIB_PATH))
    return _lib


def bind(lib: ctypes.CDLL) -> ctypes.CDLL:
    """Declares the argument and result types of the include/pwdec.h entry points on `lib`."""
    P, I64, VP = ctypes.POINTER, ctypes.c_int64, ctypes.c_void_p
    sig = {
        "decoder_blob_floats": (ctypes.c_size_t, [P(Geometry), P(ModelDims)]),
        "decoder_validate_config": (ctypes.c_int, [P(Geometry), P(ModelDims)]),
        "decoder_create": (ctypes.c_int, [P(Geometry), P(ModelDims), ctypes.c_void_p, ctypes.c_size_t, P(VP)]),
        "decode_windows": (ctypes.c_int, [VP, VP, VP, I64, VP, VP, VP]),
        "decode_windows_recurrent": (ctypes.c_int, [VP, VP, VP, I64, VP, VP, VP]),
        "decode_windows_noalloc": (ctypes.c_int, [VP, VP, VP, I64, VP, VP, VP]),
        "decoder_detection_events": (ctypes.c_int, [VP, VP, VP, I64, VP, VP]),
        "decode_stream": (ctypes.c_int, [VP, VP, I64, VP, VP, VP, VP, VP, VP]),
        "decoder_sync_status": (ctypes.c_int, [VP, VP]),
        "decoder_last_error": (ctypes.c_char_p, []),
        "decoder_destroy": (ctypes.c_int, [VP]),
        "decoder_profile": (ctypes.c_int, [VP, ctypes.c_int]),
        "decoder_schedule": (ctypes.c_int, [VP, ctypes.c_int]),
        "decoder_profile_read": (ctypes.c_int, [VP, P(StageTimes)]),
        "decoder_rotary_blob_floats": (ctypes.c_size_t, [P(Geometry), P(ModelDims), P(RotaryDims)]),
        "decoder_validate_rotary": (ctypes.c_int, [P(Geometry), P(ModelDims), P(RotaryDims)]),
        "decoder_create_rotary": (ctypes.c_int, [P(Geometry), P(ModelDims), P(RotaryDims), ctypes.c_void_p,
                                                 ctypes.c_size_t, P(VP)]),
        "pwd_linear_workspace": (ctypes.c_size_t, [P(LinearArgs)]),
        "pwd_linear": (ctypes.c_int, [P(LinearArgs), VP]),
        "pwd_rope": (ctypes.c_int, [P(RopeArgs), VP]),
        "pwd_qk_norm_rope": (ctypes.c_int, [P(RopeArgs), VP, VP, ctypes.c_double, VP]),
        "pwd_attention_workspace": (ctypes.c_size_t, [P(AttentionArgs)]),
        "pwd_attention": (ctypes.c_int, [P(AttentionArgs), VP]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    return lib


def header_functions() -> list[str]:
    """Names of the functions declared in include/pwdec.h."""
    text = open(HEADER).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return re.findall(r"^\s*(?:const\s+)?\w+\s*\*?\s*(\w+)\s*\(", text, flags=re.M)


def _check(rc: int):
    if rc != PWD_OK:
        raise PwdError(rc, load_library().decoder_last_error().decode())


def geometry(d: int, W: int, max_windows: int) -> Geometry:
    return Geometry(d, W, max_windows)


TOKENS_STABILIZERS, TOKENS_GRID = 0, 1


EMBED_LINEAR, EMBED_RESNET = 0, 1


def dims(D: int, L: int, H: int, mlp_ratio: int, dtype: int, token_set: int = TOKENS_STABILIZERS,
         embedder: int = EMBED_LINEAR, dilations=(0, 0, 0)) -> ModelDims:
    return ModelDims(D, L, H, mlp_ratio, dtype, token_set, embedder, (ctypes.c_int32 * 3)(*dilations))


def pack_dilations(dil) -> int:
    """Blob header word 13: byte j = dilation of the j-th dilated convolution (0: none)."""
    dil = list(dil) if dil else [0, 0, 0]
    return dil[0] | (dil[1] << 8) | (dil[2] << 16)


def make_blob(d: int, W: int, D: int, L: int, H: int, F: int, dtype: int, weights: dict,
              token_set: int = TOKENS_STABILIZERS, rotary: RotaryDims | None = None) -> bytes:
    """Serializes a weight dict into the library's blob format (header + fp32 tensors). A rotary network's
    layers hold the norm gains "gq" and "gk" where it norms its queries and keys."""
    kappa = np.float32(weights["kappa"])
    eps = np.float32(weights["eps"])
    hdr = [BLOB_MAGIC, BLOB_VERSION, d, W, D, L, H, F, dtype,
           struct.unpack("<I", struct.pack("<f", kappa))[0],
           struct.unpack("<I", struct.pack("<f", eps))[0], token_set,
           EMBED_RESNET if "res" in weights else EMBED_LINEAR, pack_dilations(weights.get("dilations")), 0, 0]
    if rotary is not None:
        hdr[14] = rotary.qk_norm | rotary.pairs[0] << 8 | rotary.pairs[1] << 16
        hdr[15] = struct.unpack("<I", struct.pack("<f", rotary.theta))[0]
    parts = [weights["w_e"], weights["b_e"]]
    for lw in weights["layers"]:
        parts += [lw[k] for k in ("Wq", "bq", "Wk", "bk", "Wv", "bv", "Wo", "bo", "g1", "be1",
                                  "W1", "b1", "W2", "b2", "g2", "be2")]
    parts += [weights["Wc"], weights["bc"], weights["w_o"], weights["b_o"], weights["beta"]]
    if "res" in weights:
        parts += [weights["res"][k] for k in ("W1", "b1", "W2", "b2")]
    if weights.get("dilations"):
        for lw in weights["layers"]:
            parts += [lw["Wd"], lw["bd"]]
    if rotary is not None and rotary.qk_norm:
        for lw in weights["layers"]:
            parts += [lw["gq"], lw["gk"]]
    body = np.concatenate([np.asarray(p, dtype=np.float64).ravel() for p in parts]).astype("<f4")
    return struct.pack("<16I", *hdr) + body.tobytes()


def _dtype_names(t) -> str:
    return str(t.dtype).replace("torch.", "")


def require(t, name: str, dtypes: tuple, device: int, shape: tuple | None = None, min_numel: int | None = None):
    """Checks a device buffer before its pointer crosses the ABI: a CUDA tensor on the decoder's
    device, of one of `dtypes` (names such as "int32"), contiguous, and of exactly `shape` or at
    least `min_numel` elements. The kernels index these buffers with the decoder's geometry, so
    a mismatch would be an out-of-bounds device access; it raises ValueError instead."""
    if t is None:
        raise ValueError(f"{name}: a tensor is required")
    if not getattr(t, "is_cuda", False):
        raise ValueError(f"{name}: must be a CUDA tensor (got device {getattr(t, 'device', '?')})")
    if t.device.index is not None and t.device.index != device:
        raise ValueError(f"{name}: on cuda:{t.device.index}, the decoder is on cuda:{device}")
    if _dtype_names(t) not in dtypes:
        raise ValueError(f"{name}: dtype {_dtype_names(t)}, need one of {', '.join(dtypes)}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, need {tuple(shape)}")
    if min_numel is not None and t.numel() < min_numel:
        raise ValueError(f"{name}: {t.numel()} elements, need at least {min_numel}")


WORDS = ("int32", "uint32")


def _stream_ptr(stream) -> ctypes.c_void_p:
    if stream is None:
        import torch
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


class Decoder:
    """Owns one pwd_decoder handle."""

    def __init__(self, d: int, W: int, max_windows: int, D: int, L: int, H: int, mlp_ratio: int,
                 dtype: int, blob: bytes, token_set: int = TOKENS_STABILIZERS, embedder: int = EMBED_LINEAR,
                 dilations=(0, 0, 0), rotary: RotaryDims | None = None):
        import torch
        # torch's HIP runtime starts first: created the other way round (the library's HIP calls
        # before torch initialises its device), torch then finds no GPU in this process
        self.device = torch.cuda.current_device()   # decoder_create uses the current HIP device
        lib = load_library()
        self._lib = lib
        self.d, self.W, self.max_windows = d, W, max_windows
        self.N = d * d - 1
        self.words = (self.N + 31) // 32
        g, m = geometry(d, W, max_windows), dims(D, L, H, mlp_ratio, dtype, token_set, embedder, dilations)
        h = ctypes.c_void_p()
        buf = ctypes.create_string_buffer(blob, len(blob))
        if rotary is None:
            _check(lib.decoder_create(ctypes.byref(g), ctypes.byref(m), buf, len(blob), ctypes.byref(h)))
        else:
            _check(lib.decoder_create_rotary(ctypes.byref(g), ctypes.byref(m), ctypes.byref(rotary), buf, len(blob),
                                             ctypes.byref(h)))
        self._h = h

    @classmethod
    def from_workload(cls, wl, weights: dict, max_windows: int | None = None,
                      rotary: RotaryDims | None = None) -> "Decoder":
        ts = TOKENS_GRID if getattr(wl, "grid", False) else TOKENS_STABILIZERS
        emb = EMBED_RESNET if "res" in weights else EMBED_LINEAR
        blob = make_blob(wl.d, wl.W, wl.D, wl.L, wl.H, wl.F, wl.dtype, weights, ts, rotary)
        dil = tuple(weights["dilations"]) if weights.get("dilations") else (0, 0, 0)
        return cls(wl.d, wl.W, max_windows or wl.B, wl.D, wl.L, wl.H, wl.mlp_ratio, wl.dtype, blob, ts, emb, dil,
                   rotary)

    def _windows_in(self, meas, types) -> int:
        require(types, "types", ("uint8",), self.device)
        if types.dim() != 1:
            raise ValueError(f"types: shape {tuple(types.shape)}, need (n,)")
        n = types.shape[0]
        if n > self.max_windows:
            raise ValueError(f"{n} windows, the decoder was created for at most {self.max_windows}")
        require(meas, "meas", WORDS, self.device, shape=(n, self.W + 1, self.words))
        return n

    def decode(self, meas, types, logits, bits, stream=None):
        """meas: int32/uint32 [n][W+1][words] cuda tensor; types: uint8 [n]; outputs float32/uint8 [n]."""
        n = self._windows_in(meas, types)
        require(logits, "logits", ("float32",), self.device, min_numel=n)
        require(bits, "bits", ("uint8",), self.device, min_numel=n)
        _check(self._lib.decode_windows(self._h, ctypes.c_void_p(meas.data_ptr()),
                                        ctypes.c_void_p(types.data_ptr()), n,
                                        ctypes.c_void_p(logits.data_ptr()), ctypes.c_void_p(bits.data_ptr()),
                                        _stream_ptr(stream)))

    def decode_noalloc(self, meas, types, logits, bits, stream=None):
        """As decode, on the library's fixed per-GPU scratch instead of the handle's (no
        allocation; calls on one GPU must not overlap)."""
        n = self._windows_in(meas, types)
        require(logits, "logits", ("float32",), self.device, min_numel=n)
        require(bits, "bits", ("uint8",), self.device, min_numel=n)
        _check(self._lib.decode_windows_noalloc(self._h, ctypes.c_void_p(meas.data_ptr()),
                                                ctypes.c_void_p(types.data_ptr()), n,
                                                ctypes.c_void_p(logits.data_ptr()), ctypes.c_void_p(bits.data_ptr()),
                                                _stream_ptr(stream)))

    def decode_recurrent(self, meas, types, logits, bits, stream=None):
        """As decode, with outputs float32 / uint8 [n][distance]: a readout after each of the
        last `distance` rounds (the recurrent branch of Algorithm 1)."""
        n = self._windows_in(meas, types)
        require(logits, "logits", ("float32",), self.device, min_numel=n * self.d)
        require(bits, "bits", ("uint8",), self.device, min_numel=n * self.d)
        _check(self._lib.decode_windows_recurrent(self._h, ctypes.c_void_p(meas.data_ptr()),
                                                  ctypes.c_void_p(types.data_ptr()), n,
                                                  ctypes.c_void_p(logits.data_ptr()),
                                                  ctypes.c_void_p(bits.data_ptr()), _stream_ptr(stream)))

    def decode_stream(self, rounds, bit, prob=None, window_logits=None, window_bits=None, stream=None,
                      window_probs=None):
        """rounds: int32/uint32 [T][words] cuda tensor of packed measurement rounds; bit: uint8 [1]
        out; prob: float32 [1] out or None; window_logits / window_bits / window_probs: float32 /
        uint8 / float32 [ceil(T/d)] out or None (window_probs: sigmoid of each logit)."""
        ptr = lambda t: ctypes.c_void_p(t.data_ptr()) if t is not None else ctypes.c_void_p(0)
        require(rounds, "rounds", WORDS, self.device)
        if rounds.dim() != 2 or rounds.shape[1] != self.words:
            raise ValueError(f"rounds: shape {tuple(rounds.shape)}, need (T, {self.words})")
        m = -(-rounds.shape[0] // self.d)
        require(bit, "bit", ("uint8",), self.device, min_numel=1)
        if prob is not None:
            require(prob, "prob", ("float32",), self.device, min_numel=1)
        if window_logits is not None:
            require(window_logits, "window_logits", ("float32",), self.device, min_numel=m)
        if window_bits is not None:
            require(window_bits, "window_bits", ("uint8",), self.device, min_numel=m)
        if window_probs is not None:
            require(window_probs, "window_probs", ("float32",), self.device, min_numel=m)
        _check(self._lib.decode_stream(self._h, ptr(rounds), rounds.shape[0], ptr(window_logits),
                                       ptr(window_bits), ptr(window_probs), ptr(bit), ptr(prob),
                                       _stream_ptr(stream)))

    def detection_events(self, meas, types, events, stream=None):
        """events: int32/uint32 [n][W][words] out."""
        n = self._windows_in(meas, types)
        require(events, "events", WORDS, self.device, shape=(n, self.W, self.words))
        _check(self._lib.decoder_detection_events(self._h, ctypes.c_void_p(meas.data_ptr()),
                                                  ctypes.c_void_p(types.data_ptr()), n,
                                                  ctypes.c_void_p(events.data_ptr()), _stream_ptr(stream)))

    def sync_status(self, stream=None) -> int:
        return self._lib.decoder_sync_status(self._h, _stream_ptr(stream))

    def schedule(self, which: int):
        """SCHEDULE_AUTO, SCHEDULE_LAYERS or SCHEDULE_RESIDENT for the following decodes."""
        _check(self._lib.decoder_schedule(self._h, which))

    def profile(self, enable: bool):
        """Per-stage kernel timing with HIP events on the decode stream (on/off)."""
        _check(self._lib.decoder_profile(self._h, 1 if enable else 0))

    def profile_read(self) -> dict:
        """{stage: (total ms, launches)} of the launches recorded since the last read."""
        st = StageTimes()
        _check(self._lib.decoder_profile_read(self._h, ctypes.byref(st)))
        return {STAGE_NAMES[i]: (st.ms[i], st.launches[i]) for i in range(NUM_STAGES) if st.launches[i]}

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            self._lib.decoder_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---- transformer operators (pwd_linear, pwd_rope, pwd_qk_norm_rope, pwd_attention)

ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}
ROPE_LAYOUTS = {"half": 0, "adjacent": 1}
ROPE_FREQUENCIES = {"axis": 0, "shared": 1}
_OP_DTYPES = {"torch.float32": DTYPE_F32, "torch.bfloat16": DTYPE_BF16}
_dtype_codes = {}   # torch.dtype -> PWD_DTYPE_* of those in _OP_DTYPES


def _choice(value, table: dict, name: str) -> int:
    if value not in table:
        raise ValueError(f"{name}: {value!r}, need one of {', '.join(table)}")
    return table[value]


def _operand(t, name: str, dims: int) -> tuple[int, int]:
    """(device, dtype code) of an operator's first operand: a CUDA tensor of `dims` axes, the last contiguous,
    bfloat16 or float32. Raises ValueError. (Plain attribute reads: these checks are most of what a small
    call costs on the host.)"""
    if t is None or not getattr(t, "is_cuda", False):
        raise ValueError(f"{name}: must be a CUDA tensor (got {getattr(t, 'device', t)})")
    code = _dtype_codes.get(t.dtype)
    if code is None:
        if str(t.dtype) not in _OP_DTYPES:
            raise ValueError(f"{name}: dtype {_dtype_names(t)}, need bfloat16 or float32")
        code = _dtype_codes[t.dtype] = _OP_DTYPES[str(t.dtype)]
    if t.dim() != dims:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, need {dims} axes")
    if t.stride(-1) != 1 and t.size(-1) > 1:
        raise ValueError(f"{name}: its last axis must be contiguous (strides {tuple(t.stride())})")
    return t.get_device(), code


def _same(t, name: str, dev: int, dtype, shape: tuple):
    """Checks a further operand: on device `dev`, of torch dtype `dtype` (or a dtype's name), of `shape`, its
    last axis contiguous. Raises ValueError."""
    if t is None or not getattr(t, "is_cuda", False):
        raise ValueError(f"{name}: must be a CUDA tensor (got {getattr(t, 'device', t)})")
    if t.get_device() != dev:
        raise ValueError(f"{name}: on cuda:{t.get_device()}, need cuda:{dev}")
    if t.dtype != dtype and str(t.dtype) != dtype:
        raise ValueError(f"{name}: dtype {_dtype_names(t)}, need {str(dtype).replace('torch.', '')}")
    if t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, need {tuple(shape)}")
    if t.stride(-1) != 1 and t.size(-1) > 1:
        raise ValueError(f"{name}: its last axis must be contiguous (strides {tuple(t.stride())})")


def _ptr(t):
    return t.data_ptr() if t is not None else None


def _stride(t, axis: int, row: int) -> int:
    """Stride of an axis, that of packed rows where it has one element (torch leaves it arbitrary)."""
    return t.stride(axis) if t.size(axis) != 1 else row


def _call(fn, dev: int, stream, *args):
    """Runs a library call that ends with a stream argument on device `dev`: on the given stream (which must be
    of that device) or on that device's current one. Raises PwdError."""
    import torch
    if stream is None:
        raw = torch._C._cuda_getCurrentRawStream(dev)
    else:
        if stream.device.index != dev:
            raise ValueError(f"stream: of cuda:{stream.device.index}, the tensors are on cuda:{dev}")
        raw = stream.cuda_stream
    if torch.cuda.current_device() == dev:
        rc = fn(*args, raw)
    else:
        with torch.cuda.device(dev):
            rc = fn(*args, raw)
    if rc != PWD_OK:
        _check(rc)


def _set_workspace(a, need: int, given, dev: int, stream):
    """Puts the caller's workspace (uint8, at least `need` bytes) into the arguments, or one from torch's
    allocator, which reuses it in the order of the call's stream. Returns the tensor."""
    if given is not None:
        require(given, "workspace", ("uint8",), dev, min_numel=need)
    elif need:
        import torch
        if stream is None:
            given = torch.empty(need, dtype=torch.uint8, device=f"cuda:{dev}")
        else:
            with torch.cuda.stream(stream):
                given = torch.empty(need, dtype=torch.uint8, device=f"cuda:{dev}")
    if given is not None:
        a.d_workspace, a.workspace_bytes = given.data_ptr(), given.numel()
    return given


def linear(x, w, y, bias=None, activation: str = "none", residual=None, workspace=None, stream=None):
    """y = activation(x w^T + bias) + residual. x: bfloat16 or float32 [m][k], w: the same type [n][k]
    (one row per output feature); bias: float32 [n]; y: bfloat16 or float32 [m][n], residual of y's
    type and shape (y itself allowed). Rows may be strided. activation: none, relu, gelu, gelu_tanh,
    silu. workspace: uint8 cuda tensor of linear_workspace(...) bytes (None: taken from torch)."""
    a, dev = _linear_args(x, w, y, bias, activation, residual)
    lib = _lib or load_library()
    r = ctypes.byref(a)
    need = lib.pwd_linear_workspace(r)
    held = _set_workspace(a, need, workspace, dev, stream) if need or workspace is not None else None
    _call(lib.pwd_linear, dev, stream, r)
    del held   # not before the call


def _linear_args(x, w, y, bias, activation, residual) -> tuple[LinearArgs, int]:
    dev, code = _operand(x, "x", 2)
    m, k = x.shape
    n = w.size(0) if getattr(w, "is_cuda", False) and w.dim() == 2 else 0
    _same(w, "w", dev, x.dtype, (n, k))
    _, out = _operand(y, "y", 2)
    _same(y, "y", dev, y.dtype, (m, n))
    if bias is not None:
        _same(bias, "bias", dev, "torch.float32", (n,))
    ld_r = n
    if residual is not None:
        _same(residual, "residual", dev, y.dtype, (m, n))
        ld_r = _stride(residual, 0, n)
    return LinearArgs(m, n, k, x.data_ptr(), _stride(x, 0, k), w.data_ptr(), _stride(w, 0, k), _ptr(bias), _ptr(residual), ld_r,
                      y.data_ptr(), _stride(y, 0, n), code, out, _choice(activation, ACTIVATIONS, "activation")), dev


def linear_workspace(x, w, y) -> int:
    """Bytes of workspace that linear takes for these operands."""
    return load_library().pwd_linear_workspace(ctypes.byref(_linear_args(x, w, y, None, "none", None)[0]))


def _rope_args(q, k, positions, pairs, theta, layout, frequencies, inverse, q_out, k_out) -> tuple[RopeArgs, int]:
    ref = q if q is not None else k
    if ref is None:
        raise ValueError("rope: q or k is required")
    dev, code = _operand(ref, "q" if q is not None else "k", 3)
    tokens, heads, dh = ref.shape
    dt = ref.dtype
    if (q_out is not None and q is None) or (k_out is not None and k is None):
        raise ValueError("rope: an output without its input")
    hq, hk = (heads, 0) if q is not None else (0, heads)
    if k is not None and q is not None:
        hk = k.size(1) if getattr(k, "is_cuda", False) and k.dim() == 3 else 0
        _same(k, "k", dev, dt, (tokens, hk, dh))
    fields = []
    for t, n, name in ((q, hq, "q"), (k, hk, "k"), (q_out, hq, "q_out"), (k_out, hk, "k_out")):
        if t is None and name.endswith("_out"):
            fields += fields[-6:-3]          # in place
        elif t is None:
            fields += [None, 0, 0]
        else:
            if name.endswith("_out"):
                _same(t, name, dev, dt, (tokens, n, dh))
            fields += [t.data_ptr(), _stride(t, 0, dh * n), _stride(t, 1, dh)]
    pairs = tuple(pairs)
    axes = len(pairs)
    if axes > 3:
        raise ValueError(f"pairs: {axes} axes, need at most 3")
    if axes:
        one = axes == 1 and positions is not None and positions.dim() == 1
        _same(positions, "positions", dev, "torch.int32", (tokens,) if one else (tokens, axes))
        if not positions.is_contiguous():
            raise ValueError("positions: must be contiguous")
    elif positions is not None:
        raise ValueError("positions: given without pairs")
    return RopeArgs(tokens, hq, hk, dh, code, *fields, _ptr(positions), axes, pairs + (0,) * (3 - axes),
                    _choice(layout, ROPE_LAYOUTS, "layout"), _choice(frequencies, ROPE_FREQUENCIES, "frequencies"),
                    1 if inverse else 0, theta), dev


def rope(q, k, positions, pairs, theta: float = 10000.0, layout: str = "half", frequencies: str = "axis",
         inverse: bool = False, q_out=None, k_out=None, stream=None):
    """Rotates the heads of q [tokens][q_heads][dh] and k [tokens][k_heads][dh] (either may be None;
    bfloat16 or float32) by their tokens' positions, int32 [tokens][axes] (or [tokens]), in place or into
    q_out / k_out. pairs: feature pairs of each axis. layout: half (pair j is features j and j + P) or
    adjacent (2 j and 2 j + 1); frequencies: axis (theta^(-i / pairs of the axis)) or shared
    (theta^(-j / P)); inverse: undo the rotation."""
    a, dev = _rope_args(q, k, positions, pairs, theta, layout, frequencies, inverse, q_out, k_out)
    _call((_lib or load_library()).pwd_rope, dev, stream, ctypes.byref(a))


def qk_norm_rope(q, k, gain_q, gain_k, positions, pairs, theta: float = 10000.0, layout: str = "half",
                 frequencies: str = "axis", eps: float = 1e-6, q_out=None, k_out=None, stream=None):
    """RMS norm of every head of q and k (gains float32 [dh], or None), then the rotation of rope, in
    one pass. pairs = () and positions = None: the norm alone."""
    a, dev = _rope_args(q, k, positions, pairs, theta, layout, frequencies, False, q_out, k_out)
    for gain, name in ((gain_q, "gain_q"), (gain_k, "gain_k")):
        if gain is not None:
            _same(gain, name, dev, "torch.float32", (a.head_dim,))
    _call((_lib or load_library()).pwd_qk_norm_rope, dev, stream, ctypes.byref(a), _ptr(gain_q), _ptr(gain_k), eps)


_I64x3 = ctypes.c_int64 * 3


def _attention_args(q, k, v, out, window, sinks, scale, q_lengths, k_lengths) -> tuple[AttentionArgs, int]:
    dev, code = _operand(q, "q", 4)
    b, sq, hq, dh = q.shape
    dt = q.dtype
    sk, hk = (k.size(1), k.size(2)) if getattr(k, "is_cuda", False) and k.dim() == 4 else (0, 0)
    _same(k, "k", dev, dt, (b, sk, hk, dh))
    _same(v, "v", dev, dt, (b, sk, hk, dh))
    _same(out, "out", dev, dt, (b, sq, hq, dh))
    for t, name in ((q_lengths, "q_lengths"), (k_lengths, "k_lengths")):
        if t is not None:
            _same(t, name, dev, "torch.int32", (b,))
    fields = []
    for t, n, h in ((q, sq, hq), (k, sk, hk), (v, sk, hk), (out, sq, hq)):
        fields += [t.data_ptr(), _I64x3(_stride(t, 0, dh * h * n), _stride(t, 1, dh * h), _stride(t, 2, dh))]
    left, right = window
    return AttentionArgs(b, sq, sk, hq, hk, dh, code, *fields, _ptr(q_lengths), _ptr(k_lengths), left, right, sinks,
                         dh ** -0.5 if scale is None and dh else scale or 0.0), dev


def attention(q, k, v, out, window=(-1, -1), sinks: int = 0, scale: float | None = None, q_lengths=None,
              k_lengths=None, workspace=None, stream=None):
    """out = softmax(scale q k^T) v. q, out: bfloat16 or float32 [batch][q_len][q_heads][dh]; k, v:
    [batch][k_len][k_heads][dh], q_heads a multiple of k_heads; rows may be strided. window = (left,
    right): keys before and after a query's own position that it sees (-1: all; right = 0: causal), besides
    the first `sinks` keys. q_lengths / k_lengths: int32 [batch], the queries and keys of each sequence; the
    queries are its last tokens, and output rows past them are left as they are. A query that sees no
    key gives zeros. scale: dh^-0.5 by default. workspace: uint8 cuda tensor of
    attention_workspace(...) bytes (None: taken from torch)."""
    a, dev = _attention_args(q, k, v, out, window, sinks, scale, q_lengths, k_lengths)
    lib = _lib or load_library()
    r = ctypes.byref(a)
    need = lib.pwd_attention_workspace(r)
    held = _set_workspace(a, need, workspace, dev, stream) if need or workspace is not None else None
    _call(lib.pwd_attention, dev, stream, r)
    del held   # not before the call


def attention_workspace(q, k, v, out, window=(-1, -1), sinks: int = 0) -> int:
    """Bytes of workspace that attention takes for these operands."""
    return load_library().pwd_attention_workspace(
        ctypes.byref(_attention_args(q, k, v, out, window, sinks, None, None, None)[0]))
