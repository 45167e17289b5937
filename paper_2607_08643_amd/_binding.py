"""ctypes binding of libbsq.so (include/bsq.h). Argument marshalling only:
torch provides device memory and the current stream; every step of the codec
and of the products runs in the library's HIP kernels.

The functions carry the C names. Where the C call writes into caller buffers,
the Python function allocates them with torch unless `out=` / `ws=` are given
(pre-allocated buffers are what a HIP-graph capture needs).
"""
from __future__ import annotations

import ctypes as ct
import functools
import math
import os
from dataclasses import dataclass, field

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libbsq.so")

MAX_STAGES = 4
PITCH_ALIGN = 16
MAX_LORA_RANK = 16
MAX_GROUP = 8
MAX_ADAPTERS = 1024
MAX_ADAPTER_RANK = 128
GEMV_NOALLOC_SCRATCH_BYTES = 8 << 20

BSQ_OK, BSQ_ERR_ARG, BSQ_ERR_SHAPE, BSQ_ERR_DTYPE, BSQ_ERR_ALIGN = 0, 1, 2, 3, 4
BSQ_ERR_BUFFER_TOO_SMALL, BSQ_ERR_NONFINITE, BSQ_ERR_DEVICE, BSQ_ERR_UNSUPPORTED = 5, 6, 7, 8
BSQ_F32, BSQ_BF16 = 0, 1
DEC_IDENTITY, DEC_LINEAR, DEC_MLP, DEC_MLP_RES1 = 0, 1, 2, 3
PROT_INT8, PROT_E4M3, PROT_E5M2 = 0, 1, 2
ENC_IDENTITY, ENC_LINEAR = 0, 1
OP_ENCODE, OP_GEMV, OP_GEMM, OP_SELECT = 0, 1, 2, 3
DEVERR_NONFINITE, DEVERR_BAD_SET, DEVERR_TIMEOUT, DEVERR_POISONED = 1, 2, 4, 8


class BsqError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: {status_str(status)} (status {status})")
        self.status = status


# ---------------------------------------------------------------- C structs
class bsq_config(ct.Structure):
    _fields_ = [("d", ct.c_int32), ("b", ct.c_int32), ("stages", ct.c_int32), ("dec_kind", ct.c_int32),
                ("hidden", ct.c_int32), ("protect_num", ct.c_int32), ("protect_den", ct.c_int32),
                ("protect_axis", ct.c_int32), ("protect_format", ct.c_int32), ("encoder", ct.c_int32)]


class bsq_decoder(ct.Structure):
    _fields_ = [("W1", ct.c_void_p), ("b1", ct.c_void_p), ("W2", ct.c_void_p), ("b2", ct.c_void_p),
                ("R", ct.c_void_p), ("c", ct.c_void_p), ("E", ct.c_void_p)]


class bsq_layer(ct.Structure):
    _fields_ = [("codes", ct.c_void_p * MAX_STAGES), ("gains", ct.c_void_p * MAX_STAGES),
                ("prot_idx", ct.c_void_p), ("prot_q8", ct.c_void_p), ("prot_scale", ct.c_void_p),
                ("prot_bits", ct.c_void_p),
                ("d_out", ct.c_int64), ("d_in", ct.c_int64), ("pitch", ct.c_int64), ("k", ct.c_int64),
                ("n_mats", ct.c_int64)]


class bsq_lora(ct.Structure):
    _fields_ = [("A", ct.c_void_p), ("B", ct.c_void_p), ("rank", ct.c_int32)]


class bsq_sizes(ct.Structure):
    _fields_ = [("pitch", ct.c_int64), ("k", ct.c_int64), ("chunks", ct.c_int64),
                ("code_plane_bytes", ct.c_int64), ("gain_plane_bytes", ct.c_int64),
                ("idx_bytes", ct.c_int64), ("q8_bytes", ct.c_int64), ("scale_bytes", ct.c_int64),
                ("bits_bytes", ct.c_int64),
                ("S_code", ct.c_double), ("S_dec", ct.c_double), ("S_8bit", ct.c_double),
                ("S_LoRA", ct.c_double), ("S_meta", ct.c_double), ("S_tot", ct.c_double),
                ("bpw_nominal", ct.c_double), ("bpw_real", ct.c_double)]


EXPORTS = ("bsq_version", "bsq_status_str", "bsq_config_check", "bsq_layer_sizes", "bsq_workspace_bytes",
           "bsq_codec_bytes", "bsq_codec_prepare", "bsq_encode", "bsq_decode", "bsq_gemv", "bsq_gemv_prepare",
           "bsq_gemv_run", "bsq_gemm", "bsq_encode_with_set", "bsq_coupled_select",
           "bsq_debug_set_wait_limit", "bsq_decode_stage", "bsq_gemv_noalloc", "bsq_train_param_count",
           "bsq_train_workspace_bytes", "bsq_train_grad", "bsq_train_adam", "bsq_adapters_plan_bytes",
           "bsq_adapters_plan", "bsq_adapters_workspace_bytes", "bsq_adapters_apply", "bsq_adapters_grad",
           "bsq_xent_workspace_bytes", "bsq_xent_loss", "bsq_xent_grad", "bsq_clip_table_bytes", "bsq_clip_prepare",
           "bsq_grad_norm", "bsq_grad_clip")

# struct layouts above follow this version of include/bsq.h
ABI_VERSION = 8

_lib = None


def lib():
    """Load libbsq.so; raise if it has not been built (there is no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -c 'import __graft_entry__ as g; "
                          f"g.build()'` (the HIP library is the only implementation)")
    L = ct.CDLL(LIB_PATH)
    P, I32, I64, SZ = ct.c_void_p, ct.c_int32, ct.c_int64, ct.c_size_t
    L.bsq_version.restype = I32
    L.bsq_status_str.argtypes = [I32]
    L.bsq_status_str.restype = ct.c_char_p
    L.bsq_config_check.argtypes = [P]
    L.bsq_layer_sizes.argtypes = [P, I64, I64, I32, P]
    L.bsq_workspace_bytes.argtypes = [P, I32, I64, I64, I64, I64, ct.POINTER(SZ)]
    L.bsq_codec_bytes.argtypes = [P, ct.POINTER(SZ)]
    L.bsq_codec_prepare.argtypes = [P, P, P, SZ, P]
    L.bsq_encode.argtypes = [P, P, P, I32, I64, I64, I64, P, P, P, P, SZ, P]
    L.bsq_decode.argtypes = [P, P, P, P, I32, P]
    L.bsq_gemv.argtypes = [P, I32, P, P, P, P, I32, P, I32, P, SZ, P, P]
    L.bsq_gemv_prepare.argtypes = [P, I32, P, P, P, P, I32, P, SZ, P]
    L.bsq_gemv_run.argtypes = [P, I32, P, P, P, P, I32, P, I32, P, SZ, P, P]
    L.bsq_gemm.argtypes = [P, P, P, P, P, I32, I64, I64, P, I32, I64, P, SZ, P, P]
    L.bsq_debug_set_wait_limit.argtypes = [I32]
    L.bsq_decode_stage.argtypes = [P, P, P, I32, I32, P, P]
    L.bsq_gemv_noalloc.argtypes = [P, I32, P, P, P, P, I32, P, I32, I32, P, P]
    L.bsq_encode_with_set.argtypes = [P, P, P, I32, I64, I64, I64, P, P, P, P, SZ, P]
    L.bsq_coupled_select.argtypes = [P, P, P, P, I32, I64, I64, P, P, P, P, P, P, P, SZ, P]
    L.bsq_train_param_count.argtypes = [P, ct.POINTER(I64)]
    L.bsq_train_workspace_bytes.argtypes = [P, I64, ct.POINTER(SZ)]
    L.bsq_train_grad.argtypes = [P, P, P, I32, I64, P, I64, P, P, P, P, P, SZ, P]
    L.bsq_train_adam.argtypes = [P, P, I32, P, P, P, P, P]
    L.bsq_adapters_plan_bytes.argtypes = [I64, I32, ct.POINTER(SZ)]
    L.bsq_adapters_plan.argtypes = [P, SZ, P, P]
    L.bsq_adapters_workspace_bytes.argtypes = [I32, I64, I32, I32, I32, I64, P, ct.POINTER(SZ)]
    L.bsq_adapters_apply.argtypes = [P, I32, P, I32, I64, P, I64, P, P, P, P, I32, P, P, SZ, P]
    L.bsq_adapters_grad.argtypes = [P, I32, P, I32, I64, P, I64, P, P, P, P, I64, P, I64, I32, P, P, I32, P, SZ, P]
    L.bsq_xent_workspace_bytes.argtypes = [I32, I64, I64, I64, ct.POINTER(SZ)]
    L.bsq_xent_loss.argtypes = [P, I64, P, I64, I64, I64, I64, P, P, P, P, P, SZ, P]
    L.bsq_xent_grad.argtypes = [P, I64, P, I64, I64, I64, I64, P, P, P, P, I64, P, I64, I32, I32, P, P, SZ, P]
    L.bsq_clip_table_bytes.argtypes = [I64, P, ct.POINTER(SZ)]
    L.bsq_clip_prepare.argtypes = [P, SZ, P, P, P, P, P]
    L.bsq_grad_norm.argtypes = [P, ct.c_float, P, P, P]
    L.bsq_grad_clip.argtypes = [P, ct.c_float, P, P, P]
    for f in EXPORTS[2:]:
        getattr(L, f).restype = I32
    if L.bsq_version() != ABI_VERSION:
        raise ImportError(f"{LIB_PATH} implements ABI version {L.bsq_version()}, these bindings expect "
                          f"{ABI_VERSION}: rebuild the library")
    _lib = L
    return L


def status_str(status: int) -> str:
    return lib().bsq_status_str(int(status)).decode()


def _check(status: int, what: str):
    if status != BSQ_OK:
        raise BsqError(status, what)


def _ptr(t):
    if t is None:
        return None
    return ct.c_void_p(t.data_ptr())


def _stream(stream=None):
    if stream is None:
        stream = torch.cuda.current_stream()
    return ct.c_void_p(stream.cuda_stream)


def _dtype_code(dt) -> int:
    if dt == torch.float32:
        return BSQ_F32
    if dt == torch.bfloat16:
        return BSQ_BF16
    raise TypeError(f"unsupported dtype {dt}")


# ---------------------------------------------------------------- config
@dataclass(frozen=True)
class Config:
    d: int = 8
    stages: int = 2
    kind: int = DEC_MLP
    hidden: int = 8
    protect_num: int = 1
    protect_den: int = 100
    protect_axis: int = 0   # 0: protected input columns, 1: protected output rows
    protect_format: int = PROT_INT8   # payload of the protected slices: int8, FP8-E4M3 or FP8-E5M2
    encoder: int = ENC_IDENTITY       # ENC_LINEAR: each stage codec carries E [b, d]
    codebook_bits: int = 0            # b; 0 means b = d

    @property
    def b(self) -> int:
        return self.codebook_bits or self.d

    def c(self) -> bsq_config:
        return bsq_config(self.d, self.b, self.stages, self.kind, self.hidden, self.protect_num,
                          self.protect_den, self.protect_axis, self.protect_format, self.encoder)

    def k(self, n: int) -> int:
        """ceil(rho * n): protected channels among n."""
        if self.protect_num == 0:
            return 0
        return (n * self.protect_num + self.protect_den - 1) // self.protect_den

    def k_for(self, d_out: int, d_in: int) -> int:
        """Protected slices of a d_out x d_in matrix on this config's axis."""
        return self.k(d_out if self.protect_axis == 1 else d_in)

    def pitch(self, d_in: int) -> int:
        C = d_in // self.d
        return (C + PITCH_ALIGN - 1) // PITCH_ALIGN * PITCH_ALIGN


def bsq_version() -> int:
    return lib().bsq_version()


def bsq_config_check(cfg: Config) -> int:
    c = cfg.c()
    return lib().bsq_config_check(ct.byref(c))


def bsq_layer_sizes(cfg: Config, d_out: int, d_in: int, lora_rank: int = 0) -> dict:
    c, s = cfg.c(), bsq_sizes()
    _check(lib().bsq_layer_sizes(ct.byref(c), d_out, d_in, lora_rank, ct.byref(s)), "bsq_layer_sizes")
    return {name: getattr(s, name) for name, _ in bsq_sizes._fields_}


def bsq_workspace_bytes(cfg: Config, op: int, n_mats: int, d_out: int, d_in: int, M: int = 0) -> int:
    c, out = cfg.c(), ct.c_size_t(0)
    _check(lib().bsq_workspace_bytes(ct.byref(c), op, n_mats, d_out, d_in, M, ct.byref(out)),
           "bsq_workspace_bytes")
    return out.value


def bsq_codec_bytes(cfg: Config) -> int:
    c, out = cfg.c(), ct.c_size_t(0)
    _check(lib().bsq_codec_bytes(ct.byref(c), ct.byref(out)), "bsq_codec_bytes")
    return out.value


# ---------------------------------------------------------------- codec
@dataclass
class Codec:
    """Prepared decoder tables of one category (device buffer) plus the
    device copies of the decoder parameters they were built from."""
    cfg: Config
    buf: torch.Tensor
    params: list = field(default_factory=list)

    def ptr(self):
        return self.buf.data_ptr()


def _empty_aligned(nbytes: int, device, align: int = 256, zero: bool = False) -> torch.Tensor:
    """A uint8 device buffer whose data pointer is `align`-byte aligned."""
    t = (torch.zeros if zero else torch.empty)(nbytes + align, dtype=torch.uint8, device=device)
    off = (-t.data_ptr()) % align
    return t[off:off + nbytes]


def bsq_codec_prepare(cfg: Config, decoders, device="cuda", stream=None) -> Codec:
    """decoders: per stage an object with W1/b1/W2/b2 and, for the residual-block
    decoder, R/c (numpy or torch, fp32; None or absent where unused)."""
    dev = torch.device(device)
    params = []
    arr = (bsq_decoder * MAX_STAGES)()
    for s in range(cfg.stages):
        dec = decoders[s] if decoders is not None else None
        ts = []
        for name in ("W1", "b1", "W2", "b2", "R", "c", "E"):
            v = getattr(dec, name, None) if dec is not None else None
            if v is None:
                ts.append(None)
                continue
            t = torch.as_tensor(v, dtype=torch.float32).contiguous().to(dev)
            ts.append(t)
        params.append(ts)
        arr[s] = bsq_decoder(*[None if t is None else t.data_ptr() for t in ts])
    buf = _empty_aligned(bsq_codec_bytes(cfg), dev)
    c = cfg.c()
    _check(lib().bsq_codec_prepare(ct.byref(c), arr, _ptr(buf), buf.numel(), _stream(stream)),
           "bsq_codec_prepare")
    return Codec(cfg, buf, params)


# ---------------------------------------------------------------- layers
@dataclass
class Layer:
    """Encoded matrix (or stack of n_mats): torch tensors holding the planes."""
    cfg: Config
    codes: list
    gains: list
    idx: torch.Tensor | None
    q8: torch.Tensor | None
    scale: torch.Tensor | None
    d_out: int
    d_in: int
    n_mats: int = 1
    bits: torch.Tensor | None = None  # protected-column bitmap, int32 [.., pitch * d / 32]

    @property
    def pitch(self) -> int:
        return self.cfg.pitch(self.d_in)

    @property
    def k(self) -> int:
        return self.cfg.k_for(self.d_out, self.d_in)

    def c(self) -> bsq_layer:
        L = bsq_layer()
        for s in range(self.cfg.stages):
            L.codes[s] = self.codes[s].data_ptr()
            L.gains[s] = self.gains[s].data_ptr()
        if self.k > 0:
            L.prot_idx = self.idx.data_ptr()
            L.prot_q8 = self.q8.data_ptr()
            L.prot_scale = self.scale.data_ptr()
            if self.bits is not None:
                L.prot_bits = self.bits.data_ptr()
        L.d_out, L.d_in, L.pitch, L.k, L.n_mats = self.d_out, self.d_in, self.pitch, self.k, self.n_mats
        return L

    @property
    def row_groups(self) -> int:
        return (self.d_out + 63) // 64

    def rowmajor(self, plane):
        """A tiled plane [.., RG, pitch/16, 64, 16] as row-major [.., d_out, pitch]
        (a view change for comparisons and host tools; no arithmetic)."""
        lead = plane.shape[:-4]
        t = plane.transpose(-3, -2).reshape(*lead, self.row_groups * 64, self.pitch)
        return t[..., :self.d_out, :]

    def mat(self, m: int) -> "Layer":
        """Matrix m of a stack, as a single-matrix layer (views, no copy)."""
        if self.n_mats == 1:
            return self
        k = self.k
        return Layer(self.cfg, [c[m] for c in self.codes], [g[m] for g in self.gains],
                     None if k == 0 else self.idx[m], None if k == 0 else self.q8[m],
                     None if k == 0 else self.scale[m], self.d_out, self.d_in, 1,
                     None if (k == 0 or self.bits is None) else self.bits[m])

    def nbytes_streamed(self) -> int:
        """Bytes a product reads from this layer: the code and gain planes of
        the d_out real rows, the protected payload, scales, indices and bitmap."""
        per_row = self.pitch * (self.codes[0].element_size() + 2) * self.cfg.stages
        n = per_row * self.d_out
        if self.k and self.cfg.protect_axis == 1:
            n += self.q8.numel() + self.scale.numel() * 4 + self.idx.numel() * 4
        elif self.k:
            n += self.d_out * self.k + self.scale.numel() * 4 + self.idx.numel() * 4
            if self.bits is not None:
                n += self.bits.numel() * 4
        return n


def layer_empty(cfg: Config, d_out: int, d_in: int, n_mats: int = 1, device="cuda") -> Layer:
    """Planes in the tiled layout [n_mats][ceil(d_out/64)][pitch/16][64][16];
    the protected payload (one byte per element) as [n_mats][d_out][roundup(k, 16)] (protected rows:
    [n_mats][k][roundup(d_in, 16)], and no bitmap)."""
    P, k = cfg.pitch(d_in), cfg.k_for(d_out, d_in)
    ct_ = torch.uint8 if cfg.b <= 8 else torch.int16
    tiles = ((d_out + 63) // 64, P // 16, 64, 16)
    shape = ((n_mats,) + tiles) if n_mats > 1 else tiles
    codes = [torch.empty(shape, dtype=ct_, device=device) for _ in range(cfg.stages)]
    gains = [torch.empty(shape, dtype=torch.float16, device=device) for _ in range(cfg.stages)]
    idx = q8 = scale = bits = None
    if k > 0:
        lead = (n_mats,) if n_mats > 1 else ()
        idx = torch.empty(lead + (k,), dtype=torch.int32, device=device)
        scale = torch.empty(lead + (k,), dtype=torch.float32, device=device)
        if cfg.protect_axis == 1:
            q8 = torch.empty(lead + (k, (d_in + 15) // 16 * 16), dtype=torch.int8, device=device)
        else:
            q8 = torch.empty(lead + (d_out, (k + 15) // 16 * 16), dtype=torch.int8, device=device)
            bits = torch.empty(lead + (P * cfg.d // 32,), dtype=torch.int32, device=device)
    return Layer(cfg, codes, gains, idx, q8, scale, d_out, d_in, n_mats, bits)


def bsq_encode(cfg: Config, codec: Codec, W: torch.Tensor, g: torch.Tensor | None = None,
               out: Layer | None = None, ws: torch.Tensor | None = None, err: torch.Tensor | None = None,
               check: bool = True, stream=None) -> Layer:
    """Encode W [d_out, d_in] or a stack [n_mats, d_out, d_in] (bf16 or fp32, on the GPU)."""
    if W.dim() == 2:
        n_mats, (d_out, d_in) = 1, W.shape
    elif W.dim() == 3:
        n_mats, d_out, d_in = W.shape
    else:
        raise ValueError("W must be 2-D or 3-D")
    W = W.contiguous()
    dev = W.device
    out = out or layer_empty(cfg, d_out, d_in, n_mats, dev)
    need = bsq_workspace_bytes(cfg, OP_ENCODE, n_mats, d_out, d_in)
    ws = ws if ws is not None else _empty_aligned(need, dev)
    own_err = err is None
    err = err if err is not None else torch.zeros(1, dtype=torch.int32, device=dev)
    c, L = cfg.c(), out.c()
    gp = None if g is None else _ptr(g.contiguous().to(torch.float32))
    _check(lib().bsq_encode(ct.byref(c), ct.c_void_p(codec.ptr()), _ptr(W), _dtype_code(W.dtype), n_mats, d_out,
                            d_in, gp, ct.byref(L), _ptr(err), _ptr(ws), ws.numel(), _stream(stream)),
           "bsq_encode")
    if check and own_err:
        if int(err.item()) & 1:
            raise BsqError(BSQ_ERR_NONFINITE, "bsq_encode")
    return out


def bsq_encode_with_set(cfg: Config, codec: Codec, W: torch.Tensor, idx: torch.Tensor, out: Layer | None = None,
                        ws: torch.Tensor | None = None, err: torch.Tensor | None = None, check: bool = True,
                        stream=None) -> Layer:
    """Encode W with a given protected set idx (int32 [k] or [n_mats, k], ascending)
    on cfg.protect_axis: columns (axis 0) or rows (axis 1)."""
    if W.dim() == 2:
        n_mats, (d_out, d_in) = 1, W.shape
    elif W.dim() == 3:
        n_mats, d_out, d_in = W.shape
    else:
        raise ValueError("W must be 2-D or 3-D")
    W = W.contiguous()
    dev = W.device
    out = out or layer_empty(cfg, d_out, d_in, n_mats, dev)
    need = bsq_workspace_bytes(cfg, OP_ENCODE, n_mats, d_out, d_in)
    ws = ws if ws is not None else _empty_aligned(need, dev)
    own_err = err is None
    err = err if err is not None else torch.zeros(1, dtype=torch.int32, device=dev)
    idx = idx.to(device=dev, dtype=torch.int32).contiguous()
    if idx.numel() != n_mats * out.k:
        raise ValueError(f"idx holds {idx.numel()} entries, the layout needs {n_mats} x {out.k}")
    c, L = cfg.c(), out.c()
    _check(lib().bsq_encode_with_set(ct.byref(c), ct.c_void_p(codec.ptr()), _ptr(W), _dtype_code(W.dtype), n_mats,
                                     d_out, d_in, _ptr(idx) if idx.numel() else None, ct.byref(L), _ptr(err),
                                     _ptr(ws), ws.numel(), _stream(stream)), "bsq_encode_with_set")
    if check and own_err:
        e = int(err.item())
        if e & 1:
            raise BsqError(BSQ_ERR_NONFINITE, "bsq_encode_with_set")
        if e & 2:
            raise BsqError(BSQ_ERR_ARG, "bsq_encode_with_set (protected set not ascending or out of range)")
    return out


def bsq_coupled_select(cfg: Config, W_gate: torch.Tensor, W_up: torch.Tensor, W_down: torch.Tensor,
                       g_gate=None, g_up=None, g_down=None, with_scores: bool = False, check: bool = True,
                       stream=None):
    """Coupled MLP intermediate-channel set (eq. mlp_coupled_protection): int32
    [ceil(rho d_ffn)] ascending, and with_scores the fp64 scores [d_ffn]."""
    d_ffn, d_model = W_gate.shape
    if tuple(W_up.shape) != (d_ffn, d_model) or tuple(W_down.shape) != (d_model, d_ffn):
        raise ValueError("W_gate, W_up must be [d_ffn, d_model] and W_down [d_model, d_ffn]")
    if not (W_gate.dtype == W_up.dtype == W_down.dtype):
        raise TypeError("the three matrices must share one dtype")
    dev = W_gate.device
    Wg, Wu, Wd = (t.contiguous() for t in (W_gate, W_up, W_down))
    k = cfg.k(d_ffn)
    idx = torch.empty(max(k, 1), dtype=torch.int32, device=dev)
    scores = torch.empty(d_ffn, dtype=torch.float64, device=dev) if with_scores else None
    err = torch.zeros(1, dtype=torch.int32, device=dev)
    ws = _empty_aligned(bsq_workspace_bytes(cfg, OP_SELECT, 1, d_ffn, d_model), dev)
    gs = [None if g is None else g.to(device=dev, dtype=torch.float32).contiguous() for g in (g_gate, g_up, g_down)]
    c = cfg.c()
    _check(lib().bsq_coupled_select(ct.byref(c), _ptr(Wg), _ptr(Wu), _ptr(Wd), _dtype_code(Wg.dtype), d_model,
                                    d_ffn, *[_ptr(g) for g in gs], _ptr(idx), _ptr(scores), _ptr(err), _ptr(ws),
                                    ws.numel(), _stream(stream)), "bsq_coupled_select")
    if check and int(err.item()) & 1:
        raise BsqError(BSQ_ERR_NONFINITE, "bsq_coupled_select")
    idx = idx[:k]
    return (idx, scores) if with_scores else idx


def bsq_decode(cfg: Config, codec: Codec, layer: Layer, dtype=torch.float32, out: torch.Tensor | None = None,
               stream=None) -> torch.Tensor:
    dev = layer.codes[0].device
    shape = (layer.n_mats, layer.d_out, layer.d_in) if layer.n_mats > 1 else (layer.d_out, layer.d_in)
    out = out if out is not None else torch.empty(shape, dtype=dtype, device=dev)
    c, L = cfg.c(), layer.c()
    _check(lib().bsq_decode(ct.byref(c), ct.c_void_p(codec.ptr()), ct.byref(L), _ptr(out), _dtype_code(out.dtype),
                            _stream(stream)), "bsq_decode")
    return out


def bsq_decode_stage(cfg: Config, codec: Codec, layer: Layer, stage: int, accumulate: bool, out: torch.Tensor,
                     stream=None) -> torch.Tensor:
    """One residual stage of a sequential decode into the fp32 `out`
    (bsq_decode_stage); stages 0 .. S-1, accumulating from stage 1, give the
    bits of bsq_decode."""
    c, L = cfg.c(), layer.c()
    _check(lib().bsq_decode_stage(ct.byref(c), ct.c_void_p(codec.ptr()), ct.byref(L), int(stage), int(accumulate),
                                  _ptr(out), _stream(stream)), "bsq_decode_stage")
    return out


def _lora_struct(lora) -> bsq_lora:
    if lora is None:
        return bsq_lora(None, None, 0)
    A, B = lora
    return bsq_lora(A.data_ptr(), B.data_ptr(), int(A.shape[0]))


class GemvPlan:
    """Marshalled arguments of one grouped bsq_gemv call, reusable across
    calls (and inside a HIP-graph capture) with the same buffers."""

    def __init__(self, cfg: Config, codecs, layers, x: torch.Tensor, loras=None, y_dtype=torch.bfloat16,
                 out=None, ws=None, err=None):
        n = len(layers)
        if not (1 <= n <= MAX_GROUP) or len(codecs) != n:
            raise ValueError("group size must be 1..8 with one codec per layer")
        dev = x.device
        self.cfg, self.n, self.x = cfg, n, x
        self.layers, self.codecs, self.loras = layers, codecs, loras
        self.out = out if out is not None else [torch.empty(L.d_out, dtype=y_dtype, device=dev) for L in layers]
        need = bsq_workspace_bytes(cfg, OP_GEMV, n, max(L.d_out for L in layers), layers[0].d_in)
        # zero-filled once: the kernels leave their flagged slots at zero
        self.ws = ws if ws is not None else _empty_aligned(need, dev, zero=True)
        self.err = err  # device int32 error word (TIMEOUT / POISONED bits), or None
        self._c = cfg.c()
        self._codecs = (ct.c_void_p * n)(*[cd.ptr() for cd in codecs])
        self._layers = (bsq_layer * n)(*[L.c() for L in layers])
        self._loras = None if loras is None else (bsq_lora * n)(*[_lora_struct(l) for l in loras])
        self._y = (ct.c_void_p * n)(*[t.data_ptr() for t in self.out])
        self._xd = _dtype_code(x.dtype)
        self._yd = _dtype_code(self.out[0].dtype)

    def __call__(self, stream=None):
        _check(lib().bsq_gemv(ct.byref(self._c), self.n, self._codecs, self._layers, self._loras, _ptr(self.x),
                              self._xd, self._y, self._yd, _ptr(self.ws), self.ws.numel(), _ptr(self.err),
                              _stream(stream)), "bsq_gemv")
        return self.out

    def prepare(self, stream=None):
        """bsq_gemv_prepare: the LoRA vectors A x and, for the d = 16 symmetric
        decoder, the folded activations (no launch when neither applies)."""
        _check(lib().bsq_gemv_prepare(ct.byref(self._c), self.n, self._codecs, self._layers, self._loras,
                                      _ptr(self.x), self._xd, _ptr(self.ws), self.ws.numel(), _stream(stream)),
               "bsq_gemv_prepare")

    def run(self, stream=None):
        """bsq_gemv_run: the streaming product over the prepared workspace."""
        _check(lib().bsq_gemv_run(ct.byref(self._c), self.n, self._codecs, self._layers, self._loras,
                                  _ptr(self.x), self._xd, self._y, self._yd, _ptr(self.ws), self.ws.numel(),
                                  _ptr(self.err), _stream(stream)), "bsq_gemv_run")
        return self.out


def bsq_gemv(cfg: Config, codecs, layers, x: torch.Tensor, loras=None, y_dtype=torch.bfloat16, out=None,
             ws=None, stream=None, err=None):
    """Grouped fused decode-GEMV: returns [W_hat_g x + B_g A_g x for each layer g]."""
    if isinstance(layers, Layer):
        layers, codecs = [layers], [codecs]
        loras = None if loras is None else [loras]
        single = True
    else:
        single = False
    plan = GemvPlan(cfg, codecs, layers, x.contiguous(), loras, y_dtype, out, ws, err)
    ys = plan(stream)
    return ys[0] if single else ys


def bsq_gemv_noalloc(cfg: Config, codecs, layers, x: torch.Tensor, loras=None, y_dtype=torch.bfloat16, out=None,
                     clear_scratch=False, err=None, stream=None):
    """bsq_gemv on the library's own scratch array (bsq_gemv_noalloc): no
    workspace argument, nothing allocated by the call (outputs are allocated
    here unless `out` is given)."""
    single = isinstance(layers, Layer)
    if single:
        layers, codecs = [layers], [codecs]
        loras = None if loras is None else [loras]
    n = len(layers)
    dev = x.device
    outs = out if out is not None else [torch.empty(L.d_out, dtype=y_dtype, device=dev) for L in layers]
    c = cfg.c()
    cds = (ct.c_void_p * n)(*[cd.ptr() for cd in codecs])
    lys = (bsq_layer * n)(*[L.c() for L in layers])
    los = None if loras is None else (bsq_lora * n)(*[_lora_struct(l) for l in loras])
    ys = (ct.c_void_p * n)(*[t.data_ptr() for t in outs])
    _check(lib().bsq_gemv_noalloc(ct.byref(c), n, cds, lys, los, _ptr(x), _dtype_code(x.dtype), ys,
                                  _dtype_code(outs[0].dtype), int(bool(clear_scratch)), _ptr(err), _stream(stream)),
           "bsq_gemv_noalloc")
    return outs[0] if single else outs


def bsq_gemm(cfg: Config, codec: Codec, layer: Layer, X: torch.Tensor, lora=None, y_dtype=torch.bfloat16,
             out=None, ws=None, stream=None, err=None) -> torch.Tensor:
    """Fused decode-GEMM: Y = X W_hat^T + (X A^T) B^T for X [M, d_in] bf16."""
    M, d_in = X.shape
    dev = X.device
    out = out if out is not None else torch.empty((M, layer.d_out), dtype=y_dtype, device=dev)
    need = bsq_workspace_bytes(cfg, OP_GEMM, 1, layer.d_out, d_in, M)
    ws = ws if ws is not None else _empty_aligned(need, dev)
    c, L = cfg.c(), layer.c()
    lo = _lora_struct(lora)
    _check(lib().bsq_gemm(ct.byref(c), ct.c_void_p(codec.ptr()), ct.byref(L), ct.byref(lo), _ptr(X),
                          _dtype_code(X.dtype), M, X.stride(0), _ptr(out), _dtype_code(out.dtype), out.stride(0),
                          _ptr(ws), ws.numel(), _ptr(err), _stream(stream)), "bsq_gemm")
    return out


def bsq_debug_set_wait_limit(polls: int) -> int:
    """Testing aid (bsq_debug_set_wait_limit): polls before a product's
    finishing workgroup gives up waiting; 0 forces every such wait to give
    up, a negative value restores the default. Returns the previous value."""
    return int(lib().bsq_debug_set_wait_limit(int(polls)))


# ---------------------------------------------------------------- codec training
class bsq_train_hparams(ct.Structure):
    _fields_ = [(n, ct.c_float) for n in ("lambda_c", "lambda_e", "gamma", "tau", "lr", "beta1", "beta2", "eps")]


@dataclass(frozen=True)
class TrainHyper:
    """Codec-training hyperparameters (bsq_train_hparams)."""
    lambda_c: float = 0.25
    lambda_e: float = 0.1
    gamma: float = 1.0
    tau: float = 1.0
    lr: float = 1e-3
    beta1: float = 0.9
    beta2: float = 0.999
    eps: float = 1e-8

    def c(self) -> bsq_train_hparams:
        return bsq_train_hparams(self.lambda_c, self.lambda_e, self.gamma, self.tau, self.lr, self.beta1,
                                 self.beta2, self.eps)


def bsq_train_param_count(cfg: Config) -> int:
    out = ct.c_int64()
    c = cfg.c()
    _check(lib().bsq_train_param_count(ct.byref(c), ct.byref(out)), "bsq_train_param_count")
    return out.value


def bsq_train_workspace_bytes(cfg: Config, n: int) -> int:
    out = ct.c_size_t()
    c = cfg.c()
    _check(lib().bsq_train_workspace_bytes(ct.byref(c), n, ct.byref(out)), "bsq_train_workspace_bytes")
    return out.value


def bsq_train_grad(cfg: Config, hp: TrainHyper, chunks, theta, idx=None, n=None, grad=None, loss=None, err=None,
                   ws=None, stream=None):
    """Loss [4] (L, L_rec, L_com, L_ent) and gradient [P] of one mini-batch.
    chunks: a device tensor (fp32 or bf16) whose elements are the category's
    chunks back to back (any shape with numel a multiple of d); idx: device
    int64 chunk indices or None for the first n chunks."""
    dev = chunks.device
    x_dtype = BSQ_BF16 if chunks.dtype == torch.bfloat16 else BSQ_F32
    n_total = chunks.numel() // cfg.d
    if n is None:
        n = idx.numel() if idx is not None else n_total
    P = bsq_train_param_count(cfg)
    grad = torch.empty(P, dtype=torch.float32, device=dev) if grad is None else grad
    loss = torch.empty(4, dtype=torch.float32, device=dev) if loss is None else loss
    if ws is None:
        ws = _empty_aligned(bsq_train_workspace_bytes(cfg, n), dev)
    c, h = cfg.c(), hp.c()
    _check(lib().bsq_train_grad(ct.byref(c), ct.byref(h), _ptr(chunks), x_dtype, n_total, _ptr(idx), n, _ptr(theta),
                                _ptr(grad), _ptr(loss), _ptr(err), _ptr(ws), ws.numel(), _stream(stream)),
           "bsq_train_grad")
    return loss, grad


def bsq_train_adam(cfg: Config, hp: TrainHyper, step: int, theta, grad, m, v, stream=None):
    c, h = cfg.c(), hp.c()
    _check(lib().bsq_train_adam(ct.byref(c), ct.byref(h), step, _ptr(theta), _ptr(grad), _ptr(m), _ptr(v),
                                _stream(stream)), "bsq_train_adam")


# ---------------------------------------------------------------- shared by the operators below
def _device_of(tensors, what):
    """The one GPU that all tensors (None skipped) lie on."""
    dev = None
    for t in tensors:
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError(f"{what}: tensors must be on the GPU")
        if dev is None:
            dev = t.device
        elif t.device != dev:
            raise ValueError(f"{what}: tensors on {dev} and {t.device}")
    return dev


def _need(t, dtype, shape, what):
    """t has this dtype and shape and is contiguous."""
    if t.dtype != dtype:
        raise TypeError(f"{what}: {dtype} expected, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{what}: shape {tuple(shape)} expected, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{what}: must be contiguous")
    return t


def _matrix(t, dtype, shape, what):
    """A matrix of this dtype and shape whose rows are contiguous; the elements
    from one row to the next."""
    if t.dtype != dtype:
        raise TypeError(f"{what}: {dtype} expected, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{what}: shape {tuple(shape)} expected, got {tuple(t.shape)}")
    rows, cols = shape
    ld, one = t.stride()
    if cols > 1 and one != 1:
        raise ValueError(f"{what}: rows must be contiguous")
    if rows < 2:
        return cols
    if ld < cols:
        raise ValueError(f"{what}: rows overlap")
    return ld


def _workspace(need, dev):
    """A device buffer of `need` bytes, 256-byte aligned."""
    t = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    return t if t.data_ptr() % 256 == 0 else _empty_aligned(need, dev)


# the current stream of a device as a hipStream_t (without a Stream object
# around it, which takes longer than a launch, where torch offers that)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


class _Launch:
    """The device and stream of a call: what it allocates belongs to that
    stream (so that a buffer it frees is reused in that stream's order)."""

    def __init__(self, dev, stream):
        self.dev, self.stream = dev, stream

    def __enter__(self):
        self.ctx = None
        if self.stream is not None:
            self.ctx = torch.cuda.stream(self.stream)
        elif self.dev.index is not None and self.dev.index != torch.cuda.current_device():
            self.ctx = torch.cuda.device(self.dev)
        if self.ctx is not None:
            self.ctx.__enter__()
        return ct.c_void_p(_raw_stream(self.dev.index) if self.stream is None else self.stream.cuda_stream)

    def __exit__(self, *exc):
        if self.ctx is not None:
            self.ctx.__exit__(*exc)
        return False


# ---------------------------------------------------------------- adapters of many requests
class bsq_adapter_pool(ct.Structure):
    _fields_ = [("A", ct.c_void_p), ("B", ct.c_void_p), ("scale", ct.c_void_p), ("ranks", ct.c_void_p),
                ("d_out", ct.c_int64)]


class bsq_adapter_plan(ct.Structure):
    _fields_ = [("ids", ct.c_void_p), ("buf", ct.c_void_p), ("M", ct.c_int64), ("n", ct.c_int32)]


class AdapterPool:
    """The adapters of one projection: A [n, rank, d_in] and B [n, d_out, rank]
    (bf16), scale fp32 [n] (None: ones), ranks int32 [n] (None: all full)."""

    def __init__(self, A: torch.Tensor, B: torch.Tensor, scale: torch.Tensor | None = None,
                 ranks: torch.Tensor | None = None):
        if A.dim() != 3 or B.dim() != 3:
            raise ValueError("A must be [n, rank, d_in] and B [n, d_out, rank]")
        n, rank, d_in = A.shape
        nb, d_out, rb = B.shape
        if not (A.dtype is B.dtype is torch.bfloat16 and nb == n and rb == rank and A.is_contiguous()
                and B.is_contiguous()):
            _need(A, torch.bfloat16, (n, rank, d_in), "A")
            _need(B, torch.bfloat16, (n, d_out, rank), "B")
        if scale is not None:
            _need(scale, torch.float32, (n,), "scale")
        if ranks is not None:
            _need(ranks, torch.int32, (n,), "ranks")
        self.device = _device_of((A, B, scale, ranks), "AdapterPool")
        self.A, self.B, self.scale, self.ranks = A, B, scale, ranks
        self.n, self.rank, self.d_in, self.d_out = n, rank, d_in, d_out

    def c(self) -> bsq_adapter_pool:
        return bsq_adapter_pool(self.A.data_ptr(), self.B.data_ptr(),
                                None if self.scale is None else self.scale.data_ptr(),
                                None if self.ranks is None else self.ranks.data_ptr(), self.d_out)


class AdapterPlan:
    """A batch's tokens sorted by adapter (bsq_adapters_plan), for every
    layer's calls on that batch. buf: None for batches that need none."""

    def __init__(self, ids: torch.Tensor, n: int, buf: torch.Tensor | None):
        self.ids, self.n, self.buf, self.M = ids, n, buf, ids.shape[0]
        self._c = bsq_adapter_plan(ids.data_ptr(), None if buf is None else buf.data_ptr(), self.M, n)

    def c(self) -> bsq_adapter_plan:
        return self._c


@functools.lru_cache(maxsize=1024)
def bsq_adapters_plan_bytes(M: int, n: int) -> int:
    out = ct.c_size_t(0)
    _check(lib().bsq_adapters_plan_bytes(M, n, ct.byref(out)), "bsq_adapters_plan_bytes")
    return out.value


def bsq_adapters_plan(ids: torch.Tensor, n: int, buf: torch.Tensor | None = None, err: torch.Tensor | None = None,
                      stream=None) -> AdapterPlan:
    """The plan of a batch whose token m has adapter ids[m] of n (int32 [M];
    negative: none). ids must keep its values while the plan is used."""
    dev = _device_of((ids, buf, err), "bsq_adapters_plan")
    _need(ids, torch.int32, (ids.numel(),), "ids")
    need = bsq_adapters_plan_bytes(ids.shape[0], n)
    if not need and err is None:
        return AdapterPlan(ids, n, buf)
    with _Launch(dev, stream) as st:
        if buf is None and need:
            buf = torch.empty(need, dtype=torch.uint8, device=dev)
        plan = AdapterPlan(ids, n, buf)
        _check(lib().bsq_adapters_plan(ct.byref(plan._c), 0 if buf is None else buf.numel() * buf.element_size(), _ptr(err),
                                       st), "bsq_adapters_plan")
    return plan


def bsq_adapters_workspace_bytes(back: bool, M: int, n: int, rank: int, d_in: int, d_out) -> int:
    return _adapters_workspace(bool(back), M, n, rank, d_in, tuple(d_out))


@functools.lru_cache(maxsize=1024)
def _adapters_workspace(back, M, n, rank, d_in, d_out):
    out = ct.c_size_t(0)
    dims = (ct.c_int64 * len(d_out))(*d_out)
    _check(lib().bsq_adapters_workspace_bytes(int(back), M, n, len(d_out), rank, d_in, dims, ct.byref(out)),
           "bsq_adapters_workspace_bytes")
    return out.value


def _adapter_group(plan, pools, X, what):
    if not 1 <= len(pools) <= MAX_GROUP:
        raise ValueError(f"{what}: 1..{MAX_GROUP} projections")
    n, rank, d_in = pools[0].n, pools[0].rank, pools[0].d_in
    if any((p.n, p.rank, p.d_in) != (n, rank, d_in) for p in pools):
        raise ValueError(f"{what}: the pools of a group share n, rank and d_in")
    if plan.n != n:
        raise ValueError(f"{what}: the plan is for {plan.n} adapters, the pools hold {n}")
    ldx = _matrix(X, torch.bfloat16, (plan.M, d_in), "X")
    dims = [p.d_out for p in pools]
    return rank, d_in, ldx, (bsq_adapter_pool * len(pools))(*[p.c() for p in pools]), dims


def _pointers(tensors):
    return (ct.c_void_p * len(tensors))(*[None if t is None else t.data_ptr() for t in tensors])


def _strides(values):
    return (ct.c_int64 * len(values))(*values)


def bsq_adapters_apply(plan: AdapterPlan, pools, X: torch.Tensor, base, out=None, keep: bool = False,
                       y_dtype=torch.bfloat16, ws: torch.Tensor | None = None, stream=None):
    """y = base + s B (A x) of every token for each projection of a group
    (bsq_adapters_apply). base: a list of [M, d_out] (bf16 or fp32, which y
    takes too), or None for zero (y of y_dtype); out: where y goes, e.g. base
    itself (in place). Returns (list of y, list of t or None): keep asks for t =
    A x (fp32 [M, rank]), which the gradients take. One AdapterPool instead of a
    list: single tensors instead of lists."""
    what = "bsq_adapters_apply"
    single = isinstance(pools, AdapterPool)
    if single:
        pools, base, out = [pools], None if base is None else [base], None if out is None else [out]
    rank, d_in, ldx, arr, dims = _adapter_group(plan, pools, X, what)
    M, np_ = plan.M, len(pools)
    if base is not None:
        if len(base) != np_:
            raise ValueError(f"{what}: one base per projection")
        y_dtype = base[0].dtype
        ldb = [_matrix(b, y_dtype, (M, d), "base") for b, d in zip(base, dims)]
    dev = _device_of([plan.ids, X, ws] + [p.A for p in pools] + list(base or []) + list(out or []), what)
    code = _dtype_code(y_dtype)
    need = bsq_adapters_workspace_bytes(False, M, plan.n, rank, d_in, dims)
    with _Launch(dev, stream) as st:
        if out is None:
            out = [torch.empty((M, d), dtype=y_dtype, device=dev) for d in dims]
        ldy = [_matrix(y, y_dtype, (M, d), "out") for y, d in zip(out, dims)]
        if len(out) != np_:
            raise ValueError(f"{what}: one output per projection")
        t = [torch.empty((M, rank), dtype=torch.float32, device=dev) for _ in dims] if keep else None
        ws = ws if ws is not None else _workspace(need, dev)
        _check(lib().bsq_adapters_apply(ct.byref(plan._c), np_, arr, rank, d_in, _ptr(X), ldx,
                                        None if base is None else _pointers(base),
                                        None if base is None else _strides(ldb), _pointers(out), _strides(ldy), code,
                                        None if t is None else _pointers(t), _ptr(ws), ws.numel(), st), what)
    if single:
        return out[0], None if t is None else t[0]
    return out, t


def bsq_adapters_grad(plan: AdapterPlan, pools, X: torch.Tensor, t, dy, base: torch.Tensor | None = None,
                      want_dx: bool = True, dx: torch.Tensor | None = None, dx_dtype=torch.bfloat16, grads=None,
                      accumulate: bool = False, ws: torch.Tensor | None = None, stream=None):
    """The gradients of bsq_adapters_apply: (dx or None, list of dA, list of
    dB). t: as kept by the forward call; dy: list of [M, d_out] (bf16); base:
    what else reaches x (bf16 [M, d_in], or None for zero); dx: where that goes,
    e.g. base itself. grads: (list of dA, list of dB) to write, or with
    accumulate to add to (fp32, shaped as A and B)."""
    what = "bsq_adapters_grad"
    single = isinstance(pools, AdapterPool)
    if single:
        pools, t, dy = [pools], [t], [dy]
        grads = None if grads is None else ([grads[0]], [grads[1]])
    rank, d_in, ldx, arr, dims = _adapter_group(plan, pools, X, what)
    M, n, np_ = plan.M, plan.n, len(pools)
    if len(t) != np_ or len(dy) != np_:
        raise ValueError(f"{what}: one t and one dy per projection")
    for q in t:
        _need(q, torch.float32, (M, rank), "t")
    lddy = [_matrix(q, torch.bfloat16, (M, d), "dy") for q, d in zip(dy, dims)]
    if accumulate and grads is None:
        raise ValueError(f"{what}: accumulate needs grads")
    ldb = 0 if base is None else _matrix(base, torch.bfloat16, (M, d_in), "base")
    more = [] if grads is None else list(grads[0]) + list(grads[1])
    dev = _device_of([plan.ids, X, base, dx, ws] + [p.A for p in pools] + list(t) + list(dy) + more, what)
    need = bsq_adapters_workspace_bytes(True, M, n, rank, d_in, dims)
    with _Launch(dev, stream) as st:
        if grads is None:
            grads = ([torch.empty((n, rank, d_in), dtype=torch.float32, device=dev) for _ in dims],
                     [torch.empty((n, d, rank), dtype=torch.float32, device=dev) for d in dims])
        dA, dB = list(grads[0]), list(grads[1])
        if len(dA) != np_ or len(dB) != np_:
            raise ValueError(f"{what}: one dA and one dB per projection")
        for q, w, d in zip(dA, dB, dims):
            _need(q, torch.float32, (n, rank, d_in), "dA")
            _need(w, torch.float32, (n, d, rank), "dB")
        if want_dx and dx is None:
            dx = torch.empty((M, d_in), dtype=dx_dtype, device=dev)
        if not want_dx:
            dx = None
        lddx = 0 if dx is None else _matrix(dx, dx.dtype, (M, d_in), "dx")
        ws = ws if ws is not None else _workspace(need, dev)
        _check(lib().bsq_adapters_grad(ct.byref(plan._c), np_, arr, rank, d_in, _ptr(X), ldx, _pointers(t), _pointers(dy),
                                       _strides(lddy), _ptr(base), ldb, _ptr(dx), lddx,
                                       BSQ_BF16 if dx is None else _dtype_code(dx.dtype), _pointers(dA), _pointers(dB),
                                       int(accumulate), _ptr(ws), ws.numel(), st), what)
    return (dx, dA[0], dB[0]) if single else (dx, dA, dB)


# ---------------------------------------------------------------- cross entropy
@functools.lru_cache(maxsize=1024)
def bsq_xent_workspace_bytes(grad: bool, T: int, N: int, D: int) -> int:
    out = ct.c_size_t(0)
    _check(lib().bsq_xent_workspace_bytes(int(grad), T, N, D, ct.byref(out)), "bsq_xent_workspace_bytes")
    return out.value


def _xent_shapes(H, V, target):
    T, D = H.shape
    ldh = _matrix(H, torch.bfloat16, (T, D), "H")
    ldv = _matrix(V, torch.bfloat16, (V.shape[0], D), "V")
    _need(target, torch.int64, (T,), "target")
    return T, V.shape[0], D, ldh, ldv


def bsq_xent_loss(H: torch.Tensor, V: torch.Tensor, target: torch.Tensor, loss=None, lse=None, err=None,
                  ws: torch.Tensor | None = None, stream=None):
    """Per-token softmax cross entropy of hidden states H [T, D] under the head
    V [N, D] (bf16) and targets int64 [T] (negative: no loss), without keeping
    the logits: (loss, lse), fp32 [T]."""
    T, N, D, ldh, ldv = _xent_shapes(H, V, target)
    dev = _device_of((H, V, target, loss, lse, err, ws), "bsq_xent_loss")
    need = bsq_xent_workspace_bytes(False, T, N, D)
    with _Launch(dev, stream) as st:
        loss = torch.empty(T, dtype=torch.float32, device=dev) if loss is None else _need(loss, torch.float32, (T,), "loss")
        lse = torch.empty(T, dtype=torch.float32, device=dev) if lse is None else _need(lse, torch.float32, (T,), "lse")
        ws = ws if ws is not None else _workspace(need, dev)
        _check(lib().bsq_xent_loss(_ptr(H), ldh, _ptr(V), ldv, T, N, D, _ptr(target), _ptr(loss), _ptr(lse), _ptr(err),
                                   _ptr(ws), ws.numel(), st), "bsq_xent_loss")
    return loss, lse


def bsq_xent_grad(H: torch.Tensor, V: torch.Tensor, target: torch.Tensor, lse: torch.Tensor, g: torch.Tensor,
                  head: bool = True, dH=None, dV=None, accumulate: bool = False, err=None,
                  ws: torch.Tensor | None = None, stream=None):
    """Gradients of sum(g * loss): (dH [T, D] bf16, dV [N, D] or None where head
    is False). lse: as returned by bsq_xent_loss; g: fp32 [T]. dV: where the
    head's gradient goes (bf16 or fp32; by default a new bf16 tensor), or with
    accumulate what it is added to."""
    T, N, D, ldh, ldv = _xent_shapes(H, V, target)
    _need(lse, torch.float32, (T,), "lse")
    _need(g, torch.float32, (T,), "g")
    if accumulate and (dV is None or not head):
        raise ValueError("bsq_xent_grad: accumulate needs dV")
    dev = _device_of((H, V, target, lse, g, dH, dV, err, ws), "bsq_xent_grad")
    need = bsq_xent_workspace_bytes(True, T, N, D)
    with _Launch(dev, stream) as st:
        if dH is None:
            dH = torch.empty((T, D), dtype=torch.bfloat16, device=dev)
        lddh = _matrix(dH, torch.bfloat16, (T, D), "dH")
        if not head:
            dV = None
        elif dV is None:
            dV = torch.empty((N, D), dtype=torch.bfloat16, device=dev)
        lddv = 0 if dV is None else _matrix(dV, dV.dtype, (N, D), "dV")
        ws = ws if ws is not None else _workspace(need, dev)
        _check(lib().bsq_xent_grad(_ptr(H), ldh, _ptr(V), ldv, T, N, D, _ptr(target), _ptr(lse), _ptr(g), _ptr(dH), lddh,
                                   _ptr(dV), lddv, BSQ_BF16 if dV is None else _dtype_code(dV.dtype), int(accumulate),
                                   _ptr(err), _ptr(ws), ws.numel(), st), "bsq_xent_grad")
    return dH, dV


# ---------------------------------------------------------------- gradient norm and clipping
class bsq_clip_plan(ct.Structure):
    _fields_ = [("table", ct.c_void_p), ("count", ct.c_int64), ("chunks", ct.c_int64)]


class GradPlan:
    """The gradients of a training program (fp32 or bf16 tensors, contiguous, none
    overlapping another), prepared once for bsq_grad_norm and bsq_grad_clip; outs:
    where the clipped ones go (None: in place). The plan is of the memory that the
    tensors have now, and keeps it: gradients have to stay there from step to step,
    zeroed in place (zero_grad(set_to_none=False)). One that becomes another tensor,
    as zero_grad() makes of it by default, needs a new plan; this one would go on
    with the old values. (Preparing 504 tensors takes the host 0.3 ms, with outputs
    of their own 0.6 ms; clipping them takes 0.1 ms.)"""

    def __init__(self, tensors, outs=None, stream=None):
        tensors = list(tensors)
        outs = None if outs is None else list(outs)
        if not tensors:
            raise ValueError("GradPlan: no tensors")
        if outs is not None and len(outs) != len(tensors):
            raise ValueError("GradPlan: one output per tensor")
        for i, t in enumerate(tensors):
            if not t.is_contiguous():
                raise ValueError("GradPlan: tensors must be contiguous")
            if outs is not None:
                _need(outs[i], t.dtype, t.shape, "output")
        dev = _device_of(tensors + (outs or []), "GradPlan")
        count = len(tensors)
        sizes = _strides([t.numel() for t in tensors])
        dtypes = (ct.c_int32 * count)(*[_dtype_code(t.dtype) for t in tensors])
        need = ct.c_size_t(0)
        _check(lib().bsq_clip_table_bytes(count, sizes, ct.byref(need)), "bsq_clip_table_bytes")
        self.tensors, self.outs, self.device = tensors, outs, dev
        # (a tensor object may be given other memory; the table's pointers stay good)
        self._memory = [t.untyped_storage() for t in tensors + (outs or [])]
        with _Launch(dev, stream) as st:
            self.table = _workspace(need.value, dev)
            self._c = bsq_clip_plan(self.table.data_ptr(), count, 0)
            _check(lib().bsq_clip_prepare(ct.byref(self._c), self.table.numel(), _pointers(tensors),
                                          None if outs is None else _pointers(outs), sizes, dtypes, st),
                   "bsq_clip_prepare")


def _grad_call(fn, name, plan, max_norm, stats, err, stream):
    _device_of((plan.table, stats, err), name)
    with _Launch(plan.device, stream) as st:
        stats = torch.empty(2, dtype=torch.float32, device=plan.device) if stats is None else _need(
            stats, torch.float32, (2,), "stats")
        _check(fn(ct.byref(plan._c), max_norm, _ptr(stats), _ptr(err), st), name)
    return stats


def bsq_grad_norm(plan: GradPlan, max_norm: float, stats=None, err=None, stream=None) -> torch.Tensor:
    """fp32 [2] on the GPU: the global norm of the plan's tensors and the
    coefficient min(1, max_norm / (norm + 1e-6))."""
    return _grad_call(lib().bsq_grad_norm, "bsq_grad_norm", plan, max_norm, stats, err, stream)


def bsq_grad_clip(plan: GradPlan, max_norm: float, stats=None, err=None, stream=None) -> torch.Tensor:
    """bsq_grad_norm, and the tensors times the coefficient (in place, or in the
    plan's outputs)."""
    return _grad_call(lib().bsq_grad_clip, "bsq_grad_clip", plan, max_norm, stats, err, stream)
