"""ctypes binding of libattn_abft.so (include/attn_abft.h).

Argument marshalling only: every step of the protected layer runs in the
HIP library. torch tensors provide device memory and the current stream;
their data pointers are passed through the C ABI unchanged. If the built
library is missing, importing this module raises.
"""
from __future__ import annotations

import array
import ctypes
import dataclasses
import os
import weakref

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libattn_abft.so")

OPS = ("Q", "K", "V", "AS", "CL", "O", "dCL", "dWO", "dAP", "dV", "dQ", "dK",
       "dWQ", "dWK", "dWV", "dX")
OP_ID = {n: i for i, n in enumerate(OPS)}
KINDS = ("NUMERIC", "NEAR_INF", "INF", "NAN", "-")
ACTIONS = ("RECOMPUTE", "DELTA", "RECONSTRUCT", "UNCORRECTABLE")

ABFT_OK = 0
BF16, FP32 = 0, 1
SEC_AS, SEC_CL, SEC_O, SEC_BWD, SEC_ALL = 1, 2, 4, 8, 15
FLAG_ROOT_CHECK, FLAG_REPORT_APPEND, FLAG_UNPROTECTED, FLAG_FUSED = 1, 2, 4, 8

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is not built; run __graft_entry__.build() "
                      f"(or python -m paper_2410_11720_amd._build)")
_lib = ctypes.CDLL(LIB_PATH)


class Config(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("seq", ctypes.c_int32),
                ("hidden", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("causal", ctypes.c_int32),
                ("block_rows", ctypes.c_int32), ("scale", ctypes.c_float),
                ("t_near_inf", ctypes.c_float), ("t_correct", ctypes.c_float),
                ("e_rel", ctypes.c_float), ("sections", ctypes.c_uint32),
                ("flags", ctypes.c_uint32)]


FAULT_SET, FAULT_FLIP = 0, 1


class Fault(ctypes.Structure):
    _fields_ = [("op", ctypes.c_int32), ("b", ctypes.c_int32), ("h", ctypes.c_int32),
                ("row", ctypes.c_int32), ("col", ctypes.c_int32), ("value", ctypes.c_float),
                ("mode", ctypes.c_int32)]


class Event(ctypes.Structure):
    _fields_ = [("op", ctypes.c_int32), ("b", ctypes.c_int32), ("h", ctypes.c_int32),
                ("row", ctypes.c_int32), ("col", ctypes.c_int32), ("kind", ctypes.c_int32),
                ("action", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("observed", ctypes.c_float), ("reserved2", ctypes.c_float)]


class FreqOp(ctypes.Structure):
    _fields_ = [("flops", ctypes.c_double), ("p", ctypes.c_double * 3)]


class FreqSection(ctypes.Structure):
    _fields_ = [("n_ops", ctypes.c_int32), ("first_op", ctypes.c_int32),
                ("cost", ctypes.c_double)]


class CrossConfigC(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("q_len", ctypes.c_int32), ("k_len", ctypes.c_int32),
                ("heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("causal", ctypes.c_int32), ("scale", ctypes.c_float),
                ("buckets", ctypes.c_int32), ("max_distance", ctypes.c_int32),
                ("bidirectional", ctypes.c_int32)]


class CrossTensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("batch_stride", ctypes.c_int64),
                ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class Grad(ctypes.Structure):
    _fields_ = [("grad", ctypes.c_void_p), ("out", ctypes.c_void_p), ("numel", ctypes.c_int64),
                ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class NormConfigC(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("tokens", ctypes.c_int32), ("cols", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("weight_dtype", ctypes.c_int32),
                ("site", ctypes.c_uint32), ("dropout", ctypes.c_double), ("eps", ctypes.c_double)]


class DropoutConfigC(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("tokens", ctypes.c_int32), ("cols", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("dropout", ctypes.c_double), ("site", ctypes.c_uint32),
                ("reserved", ctypes.c_int32)]


class RotaryConfigC(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("tokens", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("rotary_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("magnitude", ctypes.c_float)]


class Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("batch_stride", ctypes.c_int64),
                ("token_stride", ctypes.c_int64)]


REPORT_HEADER = 32  # bytes before the event array
assert ctypes.sizeof(Event) == 40 and ctypes.sizeof(Fault) == 28

_vp, _sz, _i32, _i64, _f32, _u32 = (ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32,
                                   ctypes.c_int64, ctypes.c_float, ctypes.c_uint32)
_P = ctypes.POINTER(Config)
_CP = ctypes.POINTER(CrossConfigC)
_NP, _DP, _RP = map(ctypes.POINTER, (NormConfigC, DropoutConfigC, RotaryConfigC))
_u64, _f64 = ctypes.c_uint64, ctypes.c_double
_sig = {
    "attn_abft_workspace_bytes": (_sz, [_P]),
    "attn_abft_report_bytes": (_sz, [_i32]),
    "attn_abft_report_init": (ctypes.c_int, [_vp, _i32, _vp]),
    "attn_abft_forward": (ctypes.c_int, [_P, _vp, _vp, _vp, _vp, _vp, _sz, _vp, _i32, _vp, _vp]),
    "attn_abft_backward": (ctypes.c_int, [_P, _vp, _vp, _vp, _vp, _vp, _sz, _vp, _vp, _vp,
                                          _vp, _i32, _vp, _vp]),
    "attn_abft_forward_stages": (ctypes.c_int, [_P, _vp, _vp, _vp, _vp, _vp, _sz, _vp, _i32, _vp,
                                                _u32, _vp]),
    "attn_abft_backward_stages": (ctypes.c_int, [_P, _vp, _vp, _vp, _vp, _vp, _sz, _vp, _vp, _vp,
                                                 _vp, _i32, _vp, _u32, _vp]),
    "encode_checksums": (ctypes.c_int, [_vp, _i32, _i64, _i64, _i64, _i64, _i64, _i32, _i32,
                                        _vp, _vp, _vp]),
    "verify_and_correct": (ctypes.c_int, [_vp, _i32, _i64, _i64, _i64, _i64, _i64, _i32, _i32,
                                          _vp, _vp, _f32, _f32, _f32, _i32, _vp, _vp]),
    "attn_abft_workspace_offsets": (ctypes.c_int, [_P, ctypes.POINTER(_sz),
                                                   ctypes.POINTER(_sz), ctypes.POINTER(_sz)]),
    "attn_abft_strerror": (ctypes.c_char_p, [ctypes.c_int]),
    "attn_abft_workspace_tensor": (ctypes.c_int, [_P, _i32, ctypes.POINTER(_sz)]),
    "attn_abft_unsafe_probability": (ctypes.c_int, [ctypes.POINTER(FreqOp),
                                                    ctypes.POINTER(FreqSection), _i32, _vp,
                                                    _vp, _vp]),
    "attn_abft_optimize_frequencies": (ctypes.c_int, [ctypes.POINTER(FreqOp),
                                                      ctypes.POINTER(FreqSection), _i32, _vp,
                                                      ctypes.c_double, _vp]),
    "attn_abft_sections_for_step": (_u32, [_vp, _i64]),
    "attn_rel_bucket": (ctypes.c_int, [_i64, _i32, _i32, _i32]),
    "attn_cross_workspace_bytes": (_sz, [_CP]),
    "attn_cross_forward": (ctypes.c_int, [_CP, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                          _sz, _vp]),
    "attn_cross_backward": (ctypes.c_int, [_CP, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                           _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "clip_gradients_workspace_bytes": (_sz, [_i32]),
    "global_grad_norm": (ctypes.c_int, [_vp, _i32, _vp, _vp, _sz, _vp]),
    "clip_gradients": (ctypes.c_int, [_vp, _i32, ctypes.c_double, _vp, _vp, _sz, _vp]),
    "attn_abft_forward_noalloc": (ctypes.c_int, [_P, _vp, _vp, _vp, _vp, _vp, _i32, _vp, _vp]),
    "attn_dropout_draw": (ctypes.c_int, [_u64, _u64, _u32, _u32, _u32]),
    "attn_dropout": (ctypes.c_int, [_DP, _vp, _vp, _vp, _vp, _vp]),
    "attn_norm_workspace_bytes": (_sz, [_NP]),
    "attn_norm_forward": (ctypes.c_int, [_NP, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "attn_norm_backward": (ctypes.c_int, [_NP, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                          _vp, _vp, _sz, _vp]),
    "attn_rotary_frequencies": (ctypes.c_int, [_i32, _f64, _i32, _f64, _f64, _f64, _f64, _vp]),
    "attn_rotary": (ctypes.c_int, [_RP, _i32, _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "attn_rotary_append": (ctypes.c_int, [_RP, _vp, _vp, _vp, _vp, _vp, _i32, _vp, _vp, _vp, _vp]),
}
for _name, (_res, _args) in _sig.items():
    _f = getattr(_lib, _name)
    _f.restype = _res
    _f.argtypes = _args


class AbftError(RuntimeError):
    pass


def strerror(status: int) -> str:
    return _lib.attn_abft_strerror(status).decode()


def _check(status: int, what: str):
    if status != ABFT_OK:
        raise AbftError(f"{what}: {strerror(status)} ({status})")


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


@dataclasses.dataclass
class LayerConfig:
    batch: int
    seq: int
    hidden: int
    heads: int
    dtype: str = "bf16"          # "bf16" | "f32"
    causal: bool = False
    block_rows: int = 128
    scale: float = 0.0
    t_near_inf: float = 1e10
    t_correct: float = 1e5
    e_rel: float = 0.0
    sections: int = SEC_ALL
    root_check: bool = True
    protect: bool = True
    fused: bool = False          # forward attention core in one kernel (no AS/AP)

    def to_c(self, append=False) -> Config:
        flags = (FLAG_ROOT_CHECK if self.root_check else 0)
        flags |= (FLAG_REPORT_APPEND if append else 0)
        flags |= (0 if self.protect else FLAG_UNPROTECTED)
        flags |= (FLAG_FUSED if self.fused else 0)
        return Config(self.batch, self.seq, self.hidden, self.heads,
                      FP32 if self.dtype == "f32" else BF16, int(self.causal), self.block_rows,
                      self.scale, self.t_near_inf, self.t_correct, self.e_rel, self.sections,
                      flags)

    @property
    def torch_dtype(self):
        return torch.float32 if self.dtype == "f32" else torch.bfloat16


def attn_abft_workspace_bytes(cfg: LayerConfig) -> int:
    c = cfg.to_c()
    n = _lib.attn_abft_workspace_bytes(ctypes.byref(c))
    if n == 0:
        raise AbftError("invalid configuration")
    return n


def attn_abft_report_bytes(capacity: int) -> int:
    return _lib.attn_abft_report_bytes(capacity)


def attn_abft_report_init(report, capacity, stream=None):
    _check(_lib.attn_abft_report_init(_ptr(report), capacity, _stream(stream)), "report_init")


def attn_abft_workspace_offsets(cfg: LayerConfig):
    c = cfg.to_c()
    q, a, l = _sz(), _sz(), _sz()
    _check(_lib.attn_abft_workspace_offsets(ctypes.byref(c), ctypes.byref(q), ctypes.byref(a),
                                            ctypes.byref(l)), "workspace_offsets")
    return q.value, a.value, l.value


def attn_abft_forward(cfg: LayerConfig, X, Wqkv, Wo, O, workspace, faults, n_faults, report,
                      stream=None, append=False):
    c = cfg.to_c(append)
    _check(_lib.attn_abft_forward(ctypes.byref(c), _ptr(X), _ptr(Wqkv), _ptr(Wo), _ptr(O),
                                  _ptr(workspace), workspace.numel() * workspace.element_size(),
                                  _ptr(faults), n_faults, _ptr(report), _stream(stream)),
           "attn_abft_forward")


def attn_abft_forward_noalloc(cfg: LayerConfig, X, Wqkv, Wo, O, faults, n_faults, report,
                              stream=None, append=False):
    c = cfg.to_c(append)
    _check(_lib.attn_abft_forward_noalloc(ctypes.byref(c), _ptr(X), _ptr(Wqkv), _ptr(Wo), _ptr(O),
                                          _ptr(faults), n_faults, _ptr(report), _stream(stream)),
           "attn_abft_forward_noalloc")


def attn_abft_backward(cfg: LayerConfig, dO, X, Wqkv, Wo, workspace, dX, dWqkv, dWo, faults,
                       n_faults, report, stream=None, append=False):
    c = cfg.to_c(append)
    _check(_lib.attn_abft_backward(ctypes.byref(c), _ptr(dO), _ptr(X), _ptr(Wqkv), _ptr(Wo),
                                   _ptr(workspace), workspace.numel() * workspace.element_size(),
                                   _ptr(dX), _ptr(dWqkv), _ptr(dWo), _ptr(faults), n_faults,
                                   _ptr(report), _stream(stream)), "attn_abft_backward")


STAGE_ALL = 0x7FF
FWD_STAGES = {"encode": 0x001, "qkv": 0x002, "score": 0x004, "softmax": 0x008,
              "context": 0x010, "out": 0x020}
BWD_STAGES = {"encode": 0x001, "dCL": 0x002, "dWo": 0x004, "dAP": 0x008, "dV": 0x010,
              "softmax_bwd": 0x020, "dQ": 0x040, "dK": 0x080, "dWqkv": 0x100, "dX": 0x200}


def attn_abft_forward_stages(cfg: LayerConfig, X, Wqkv, Wo, O, workspace, faults, n_faults,
                             report, stages, stream=None, append=False):
    c = cfg.to_c(append)
    _check(_lib.attn_abft_forward_stages(ctypes.byref(c), _ptr(X), _ptr(Wqkv), _ptr(Wo), _ptr(O),
                                         _ptr(workspace),
                                         workspace.numel() * workspace.element_size(),
                                         _ptr(faults), n_faults, _ptr(report), stages,
                                         _stream(stream)), "attn_abft_forward_stages")


def attn_abft_backward_stages(cfg: LayerConfig, dO, X, Wqkv, Wo, workspace, dX, dWqkv, dWo,
                              faults, n_faults, report, stages, stream=None, append=False):
    c = cfg.to_c(append)
    _check(_lib.attn_abft_backward_stages(ctypes.byref(c), _ptr(dO), _ptr(X), _ptr(Wqkv),
                                          _ptr(Wo), _ptr(workspace),
                                          workspace.numel() * workspace.element_size(),
                                          _ptr(dX), _ptr(dWqkv), _ptr(dWo), _ptr(faults),
                                          n_faults, _ptr(report), stages, _stream(stream)),
           "attn_abft_backward_stages")


def encode_checksums(A, dtype, batch, rows, cols, ld, batch_stride, block_rows, block_cols,
                     col_chk, row_chk, stream=None):
    _check(_lib.encode_checksums(_ptr(A), dtype, batch, rows, cols, ld, batch_stride,
                                 block_rows, block_cols, _ptr(col_chk), _ptr(row_chk),
                                 _stream(stream)), "encode_checksums")


def verify_and_correct(C, dtype, batch, rows, cols, ld, batch_stride, block_rows, block_cols,
                       col_chk, row_chk, t_near_inf, t_correct, e_rel, op_tag, report,
                       stream=None):
    _check(_lib.verify_and_correct(_ptr(C), dtype, batch, rows, cols, ld, batch_stride,
                                   block_rows, block_cols, _ptr(col_chk), _ptr(row_chk),
                                   t_near_inf, t_correct, e_rel, op_tag, _ptr(report),
                                   _stream(stream)), "verify_and_correct")


# ---- conveniences for callers holding torch tensors -----------------------

def _freq_args(sections):
    """sections: [(cost, [(flops, (p_inf, p_nan, p_ninf)), ...]), ...]"""
    ops, secs = [], []
    for cost, sec_ops in sections:
        secs.append(FreqSection(len(sec_ops), len(ops), float(cost)))
        for flops, p in sec_ops:
            ops.append(FreqOp(float(flops), (ctypes.c_double * 3)(*[float(x) for x in p])))
    oa = (FreqOp * max(1, len(ops)))(*ops)
    sa = (FreqSection * len(secs))(*secs)
    return oa, sa, len(secs)


def _doubles(xs):
    return (ctypes.c_double * len(xs))(*[float(x) for x in xs])


def attn_abft_unsafe_probability(sections, lam, freqs) -> float:
    oa, sa, n = _freq_args(sections)
    out = ctypes.c_double()
    _check(_lib.attn_abft_unsafe_probability(oa, sa, n, _doubles(lam), _doubles(freqs),
                                             ctypes.byref(out)), "unsafe_probability")
    return out.value


def attn_abft_optimize_frequencies(sections, lam, fail_target) -> list:
    oa, sa, n = _freq_args(sections)
    out = (ctypes.c_double * n)()
    _check(_lib.attn_abft_optimize_frequencies(oa, sa, n, _doubles(lam), float(fail_target),
                                               out), "optimize_frequencies")
    return list(out)


def attn_abft_sections_for_step(freqs4, step: int) -> int:
    return int(_lib.attn_abft_sections_for_step(_doubles(freqs4), int(step)))


def faults_to_device(faults, device="cuda"):
    """Pack (op, b, h, row, col, value[, mode]) tuples into a device array
    of abft_fault records; mode "set" (default) or "flip". Returns (tensor
    or None, count)."""
    faults = [f.as_tuple() if hasattr(f, "as_tuple") else tuple(f) for f in faults]
    if not faults:
        return None, 0

    def rec(t):
        o, b, h, r, c, v = t[:6]
        mode = FAULT_FLIP if len(t) > 6 and t[6] == "flip" else FAULT_SET
        return Fault(OP_ID[o] if isinstance(o, str) else int(o), b, h, r, c, float(v), mode)
    arr = (Fault * len(faults))(*[rec(t) for t in faults])
    host = torch.frombuffer(bytearray(bytes(arr)), dtype=torch.uint8)
    return host.to(device), len(faults)


def new_report(capacity=4096, device="cuda", stream=None):
    rep = torch.empty(attn_abft_report_bytes(capacity), dtype=torch.uint8, device=device)
    attn_abft_report_init(rep, capacity, stream)
    return rep


def read_report(report) -> dict:
    """Copy a report to the host: counters and the event list as tuples
    (op, b, h, row, col, kind, action)."""
    raw = bytes(report.cpu().numpy().tobytes())
    n_events, n_corr, n_unc, cap, overflow = (int.from_bytes(raw[4 * i:4 * i + 4], "little",
                                                             signed=True) for i in range(5))
    evs = []
    for k in range(min(n_events, cap)):
        e = Event.from_buffer_copy(raw, REPORT_HEADER + k * ctypes.sizeof(Event))
        evs.append((OPS[e.op], e.b, e.h, e.row, e.col, KINDS[e.kind], ACTIONS[e.action]))
    return dict(n_events=n_events, n_corrected=n_corr, n_uncorrectable=n_unc,
                capacity=cap, overflow=overflow, events=evs)


class ProtectedAttention:
    """Owns the workspace and report of one layer shape and runs the
    protected forward and backward through the C ABI."""

    def __init__(self, cfg: LayerConfig, device="cuda", capacity=4096):
        self.cfg = cfg
        self.device = device
        self.workspace = torch.empty(attn_abft_workspace_bytes(cfg), dtype=torch.uint8,
                                     device=device)
        self.report = new_report(capacity, device)
        self.report_bwd = new_report(capacity, device)

    def forward(self, X, Wqkv, Wo, faults=None, O=None):
        c = self.cfg
        if O is None:
            O = torch.empty((c.batch, c.seq, c.hidden), dtype=c.torch_dtype, device=self.device)
        f, n = faults if faults is not None else (None, 0)
        attn_abft_forward(c, X, Wqkv, Wo, O, self.workspace, f, n, self.report)
        return O

    def backward(self, dO, X, Wqkv, Wo, faults=None, dX=None, dWqkv=None, dWo=None):
        c = self.cfg
        if dX is None:
            dX = torch.empty((c.batch, c.seq, c.hidden), dtype=c.torch_dtype, device=self.device)
        if dWqkv is None:
            dWqkv = torch.empty((c.hidden, 3 * c.hidden), dtype=torch.float32, device=self.device)
        if dWo is None:
            dWo = torch.empty((c.hidden, c.hidden), dtype=torch.float32, device=self.device)
        f, n = faults if faults is not None else (None, 0)
        attn_abft_backward(c, dO, X, Wqkv, Wo, self.workspace, dX, dWqkv, dWo, f, n,
                           self.report_bwd)
        return dX, dWqkv, dWo

    TENSORS = ("QKV", "AS", "AP", "CL", "dQKV", "dCL", "APc", "APr", "dAS")

    def tensor(self, which):
        """View of a tensor the forward or backward leaves in the workspace:
        "QKV", "AS" (until the next backward), "AP", "CL", "dQKV", "dCL",
        "dAS" (storage dtype), "APc", "APr" (fp32 checksums of AP)."""
        c = self.cfg
        k = self.TENSORS.index(which)
        off = ctypes.c_size_t()
        _check(_lib.attn_abft_workspace_tensor(ctypes.byref(c.to_c()), k, ctypes.byref(off)),
               "workspace_tensor")
        B, S, H, nh = c.batch, c.seq, c.hidden, c.heads
        nq = S // c.block_rows
        shape = {"QKV": (B, S, 3 * H), "AS": (B, nh, S, S), "AP": (B, nh, S, S),
                 "CL": (B, S, H), "dQKV": (B, S, 3 * H), "dCL": (B, S, H),
                 "dAS": (B, nh, S, S), "APc": (B, nh, nq, 2, S),
                 "APr": (B, nh, S, nq, 2)}[which]
        dt = torch.float32 if which in ("APc", "APr") else c.torch_dtype
        es = 4 if dt == torch.float32 else 2
        n = 1
        for x in shape:
            n *= x
        o = off.value
        return self.workspace[o:o + n * es].view(dt).view(*shape)

    def saved(self):
        """Views of the saved QKV, AP and CL inside the workspace."""
        c = self.cfg
        q, a, l = attn_abft_workspace_offsets(c)
        es = 4 if c.dtype == "f32" else 2
        T, H, S = c.batch * c.seq, c.hidden, c.seq

        def view(off, n, shape):
            return self.workspace[off:off + n * es].view(c.torch_dtype).view(*shape)
        return (view(q, T * 3 * H, (c.batch, S, 3 * H)),
                view(a, c.batch * c.heads * S * S, (c.batch, c.heads, S, S)),
                view(l, T * H, (c.batch, S, H)))


# ---- attention over keys of another length ---------------------------------

def attn_rel_bucket(relative: int, buckets: int, max_distance: int = 128,
                    bidirectional: bool = True) -> int:
    """Bucket of the relative position key - query (host only)."""
    k = _lib.attn_rel_bucket(int(relative), buckets, max_distance, int(bidirectional))
    if k < 0:
        raise AbftError(f"attn_rel_bucket: {strerror(k)} ({k})")
    return k


@dataclasses.dataclass
class CrossConfig:
    batch: int
    q_len: int
    k_len: int
    heads: int
    head_dim: int
    kv_heads: int = 0            # 0: one key head per query head
    dtype: str = "bf16"          # "bf16" | "f32"
    causal: bool = False
    scale: float = 0.0
    buckets: int = 0             # rows of the relative position bias table; 0: none
    max_distance: int = 128
    bidirectional: bool = True

    def to_c(self) -> CrossConfigC:
        return CrossConfigC(self.batch, self.q_len, self.k_len, self.heads,
                            self.kv_heads or self.heads, self.head_dim,
                            FP32 if self.dtype == "f32" else BF16, int(self.causal), self.scale,
                            self.buckets, self.max_distance, int(self.bidirectional))

    @property
    def torch_dtype(self):
        return torch.float32 if self.dtype == "f32" else torch.bfloat16


def attn_cross_workspace_bytes(cfg: CrossConfig) -> int:
    c = cfg.to_c()
    n = _lib.attn_cross_workspace_bytes(ctypes.byref(c))
    if n == 0:
        raise AbftError("invalid configuration")
    return n


def _data(t):
    return None if t is None else t.data_ptr()


# (a stream object costs 2.7 us, a quarter of a small call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream",
                      lambda index: torch.cuda.current_stream(index).cuda_stream)


_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _call(fn, device, *args):
    """fn(*args, current stream of the device) with that device current."""
    index = device.index
    if index == _current_device():
        return fn(*args, _raw_stream(index))
    with torch.cuda.device(index):
        return fn(*args, _raw_stream(index))


class CrossSaved:
    """What a forward leaves for its backward: the row statistics `lse`, and
    `rest`, what rounding took off O (None in fp32)."""

    def __init__(self, cfg: CrossConfig, device):
        rows = (cfg.batch, cfg.heads, cfg.q_len)
        self.lse = torch.empty(rows, dtype=torch.float32, device=device)
        self.rest = None
        if cfg.dtype != "f32":
            self.rest = torch.empty((*rows, cfg.head_dim), dtype=torch.bfloat16, device=device)
        self._of = None              # where the O that they belong to was written


class CrossAttention:
    """Attention of q_len queries over k_len keys a sequence: owns the
    workspace of one shape and one record of what a forward leaves for its
    backward (`lse`, `rest`), as ProtectedAttention does for its layer; with
    training=False it has no record. A forward replaces the record: backward
    raises if its O is not the last forward's. Where other forwards come in
    between (layers that share the object, micro-batches), or O has moved since,
    pass a record of `new_saved` to both calls as `saved`; which O belongs to it
    is then the caller's to know. Calls run on the current stream of the tensors'
    device.

    Q, O, dO, dQ [batch, q_len, heads, head_dim]; K, V, dK, dV [batch, k_len,
    kv_heads, head_dim]; any strides with whole rows at multiples of 16 bytes
    (views of packed projections, of a cache); results not given are laid out as
    torch.empty_like of Q, K or V. bias, dbias [buckets, heads]
    fp32; k_lens, q_start [batch] int32."""

    def __init__(self, cfg: CrossConfig, device="cuda", training=True):
        self.cfg = cfg
        self.device = torch.empty(0, device=device).device
        self._c = cfg.to_c()
        self.workspace = torch.empty(attn_cross_workspace_bytes(cfg), dtype=torch.uint8,
                                     device=self.device)
        self._saved = self.new_saved() if training else None
        kvh = cfg.kv_heads or cfg.heads
        self._q_shape = (cfg.batch, cfg.q_len, cfg.heads, cfg.head_dim)
        self._k_shape = (cfg.batch, cfg.k_len, kvh, cfg.head_dim)

    @property
    def lse(self):
        return self._saved and self._saved.lse

    @property
    def rest(self):
        return self._saved and self._saved.rest

    def new_saved(self):
        """Another record for a forward and its backward."""
        return CrossSaved(self.cfg, self.device)

    def _record(self, saved):
        c = self.cfg
        if (saved.lse.shape != (c.batch, c.heads, c.q_len) or saved.lse.device != self.device
                or (saved.rest is None) != (c.dtype == "f32")
                or saved.rest is not None and saved.rest.shape[3] != c.head_dim):
            raise AbftError("saved: made for another shape, type or device")
        return saved

    def _tensors(self, names, tensors, shapes):
        """The tensors' attn_cross_tensor records, one after the other; returns
        them and the address of each."""
        fields, dtype, index = [], self.cfg.torch_dtype, self.device.index
        for name, t, shape in zip(names, tensors, shapes):
            st = t.stride()
            if t.get_device() != index or t.dtype != dtype or t.shape != shape or st[3] != 1:
                raise AbftError(f"{name}: expected {shape} {dtype} on {self.device} with a "
                                f"contiguous last dimension, got {tuple(t.shape)} {t.dtype} on "
                                f"{t.device}, strides {st}")
            fields += (t.data_ptr(), st[0], st[1], st[2])
        records = array.array("q", fields)
        at = records.buffer_info()[0]
        return records, range(at, at + 32 * len(names), 32)

    def _vector(self, t, name, shape, dtype):
        if t is None:
            return None
        if t.device != self.device or t.dtype != dtype or t.shape != shape or not t.is_contiguous():
            raise AbftError(f"{name}: expected contiguous {shape} {dtype} on {self.device}, got "
                            f"{tuple(t.shape)} {t.dtype} on {t.device}")
        return t.data_ptr()

    def _keys(self, bias, k_lens, q_start):
        c = self.cfg
        return (self._vector(bias, "bias", (c.buckets, c.heads), torch.float32),
                self._vector(k_lens, "k_lens", (c.batch,), torch.int32),
                self._vector(q_start, "q_start", (c.batch,), torch.int32))

    def forward(self, Q, K, V, bias=None, k_lens=None, q_start=None, O=None, saved=None):
        if O is None:
            O = torch.empty_like(Q)
        qs, ks = self._q_shape, self._k_shape
        held, (q, k, v, o) = self._tensors("QKVO", (Q, K, V, O), (qs, ks, ks, qs))
        bias, k_lens, q_start = self._keys(bias, k_lens, q_start)
        saved = self._saved if saved is None else self._record(saved)
        lse = rest = None
        if saved is not None:
            lse, rest, saved._of = _data(saved.lse), _data(saved.rest), None
        _check(_call(_lib.attn_cross_forward, self.device, self._c, q, k, v, bias, k_lens, q_start,
                     o, lse, rest, self.workspace.data_ptr(), self.workspace.numel()),
               "attn_cross_forward")
        if saved is not None:
            saved._of = O.data_ptr()
        return O

    def backward(self, dO, Q, K, V, O, bias=None, k_lens=None, q_start=None, dQ=None, dK=None,
                 dV=None, dbias=None, saved=None):
        c = self.cfg
        own = saved is None
        saved = self._saved if own else self._record(saved)
        if saved is None:
            raise AbftError("backward: made with training=False")
        if saved._of is None or own and saved._of != O.data_ptr():
            raise AbftError("backward: O is not what the last forward left" if saved._of is not None
                            else "backward: no forward has left its statistics")
        dQ = torch.empty_like(Q) if dQ is None else dQ
        dK = torch.empty_like(K) if dK is None else dK
        dV = torch.empty_like(V) if dV is None else dV
        if dbias is None and c.buckets:
            dbias = torch.empty((c.buckets, c.heads), dtype=torch.float32, device=self.device)
        qs, ks = self._q_shape, self._k_shape
        held, (do, q, k, v, o, dq, dk, dv) = self._tensors(
            ("dO", "Q", "K", "V", "O", "dQ", "dK", "dV"), (dO, Q, K, V, O, dQ, dK, dV),
            (qs, qs, ks, ks, qs, qs, ks, ks))
        bias, k_lens, q_start = self._keys(bias, k_lens, q_start)
        db = self._vector(dbias, "dbias", (c.buckets, c.heads), torch.float32)
        _check(_call(_lib.attn_cross_backward, self.device, self._c, do, q, k, v, o,
                     _data(saved.lse), _data(saved.rest), bias, k_lens, q_start, dq, dk, dv, db,
                     self.workspace.data_ptr(), self.workspace.numel()), "attn_cross_backward")
        return dQ, dK, dV, dbias


# ---- norm and clipping of gradients -------------------------------------------

_GRAD_DTYPES = {torch.float32: FP32, torch.bfloat16: BF16}


class GradStats:
    """Views of the device statistics that global_grad_norm and clip_gradients
    leave: `norm` and `coef` (fp32) and `nonfinite` (int64), of no dimension."""

    def __init__(self, device):
        self.raw = torch.zeros(2, dtype=torch.int64, device=device)
        f = self.raw[:1].view(torch.float32)
        self.norm, self.coef, self.nonfinite = f[0], f[1], self.raw[1]


class GradientClip:
    """Global norm of gradient tensors, and clipping by it: owns the
    workspace for as many tensors as `grads` holds, and the statistics of the
    last call (`stats`). Tensors are contiguous, bf16 or fp32, on one device."""

    def __init__(self, grads):
        grads = list(grads)
        self.device = grads[0].device if grads else torch.empty(0, device="cuda").device
        self._n = len(grads)
        self.workspace = torch.empty(_lib.clip_gradients_workspace_bytes(self._n),
                                     dtype=torch.uint8, device=self.device)
        self.stats = GradStats(self.device)

    def _list(self, grads, out):
        n = len(grads)
        if n > self._n:
            raise AbftError(f"{n} gradients, made for {self._n}")
        if len(out) != n:
            raise AbftError(f"{n} gradients, {len(out)} outputs")
        # checked and read a field at a time (a tensor at a time takes twice as
        # long, more than clipping 28 M elements does)
        dtypes = [_GRAD_DTYPES.get(g.dtype) for g in grads]
        numel = self._plain(grads, "gradient")
        if None in dtypes:
            i = dtypes.index(None)
            raise AbftError(f"gradient {i}: {grads[i].dtype}")
        grad_ptrs = out_ptrs = list(map(torch.Tensor.data_ptr, grads))
        if out is not grads:
            if (self._plain(out, "output") != numel
                    or [_GRAD_DTYPES.get(o.dtype) for o in out] != dtypes):
                raise AbftError("outputs: expected the gradients' types and sizes")
            out_ptrs = list(map(torch.Tensor.data_ptr, out))
        fields = [0] * (4 * n)   # abft_grad, dtype and reserved as one
        fields[0::4], fields[1::4], fields[2::4], fields[3::4] = grad_ptrs, out_ptrs, numel, dtypes
        return array.array("q", fields), n

    def _plain(self, tensors, name):
        """Sizes of contiguous tensors on the device (else raises)."""
        index = self.device.index
        if (not all(map(torch.Tensor.is_contiguous, tensors))
                or any(d != index for d in map(torch.Tensor.get_device, tensors))):
            raise AbftError(f"{name}s: expected contiguous tensors on {self.device}")
        return list(map(torch.Tensor.numel, tensors))

    def norm(self, grads):
        """Leaves the norm in `stats`, which it returns."""
        arr, n = self._list(grads, grads)
        _check(_call(_lib.global_grad_norm, self.device, arr.buffer_info()[0], n,
                     self.stats.raw.data_ptr(), self.workspace.data_ptr(),
                     self.workspace.numel()), "global_grad_norm")
        return self.stats

    def clip(self, grads, max_norm, out=None):
        """Scales the gradients to a global norm of at most max_norm, in place
        or into `out`; leaves norm, coef and nonfinite in `stats`."""
        arr, n = self._list(grads, grads if out is None else out)
        _check(_call(_lib.clip_gradients, self.device, arr.buffer_info()[0], n, float(max_norm),
                     self.stats.raw.data_ptr(), self.workspace.data_ptr(),
                     self.workspace.numel()), "clip_gradients")
        return self.stats


# ---- layer norm, dropout, rotary positions ----------------------------------------

_DTYPES = {"bf16": (BF16, torch.bfloat16), "f32": (FP32, torch.float32)}


def _dtype_of(name, what):
    if name not in _DTYPES:
        raise AbftError(f"{what}: {name!r} is neither \"bf16\" nor \"f32\"")
    return _DTYPES[name]


def _fits(lo, hi, **sizes):
    """Raises for a size that its field of the C structures would cut."""
    for name, n in sizes.items():
        if not lo <= n < hi:
            raise AbftError(f"{name}: {n} is not in [{lo}, {hi})")


_I32, _U32 = (-2 ** 31, 2 ** 31), (0, 2 ** 32)


def _columns(t):
    """A new tensor, laid out with contiguous columns if it is not (torch.empty_like of rows
    that move on by one element is not)."""
    if t.stride()[-1] != 1 and t.shape[-1] > 1:
        t.as_strided_(t.shape, torch.empty(t.shape, device="meta").stride())
    return t


class _Op:
    """Marshalling that the classes below share: tensors of one type and device
    as records of address and strides."""

    def _records(self, names, tensors, shapes, fresh=()):
        """Records (address, all strides but the last) one after the other, None
        for an absent tensor; `fresh` ones, which a call has just made like one of
        the others, are not looked over. Returns the records and the address of each."""
        fields, at, dtype, index = [], [], self._dtype, self.device.index
        for name, t, shape in zip(names, tensors, shapes):
            if t is None:
                at.append(None)
                continue
            st = t.stride()
            if t.get_device() != index or t.dtype is not dtype or t.shape != shape or (
                    st[-1] != 1 and shape[-1] > 1):
                raise AbftError(f"{name}: expected {tuple(shape)} {dtype} on {self.device} with a "
                                f"contiguous last dimension, got {tuple(t.shape)} {t.dtype} on "
                                f"{t.device}, strides {st}")
            at.append(8 * len(fields))
            fields.append(t.data_ptr())
            fields += st[:-1]
        for t in fresh:
            st = t.stride()
            if st[-1] != 1:
                st = _columns(t).stride()
            at.append(8 * len(fields))
            fields.append(t.data_ptr())
            fields += st[:-1]
        held = array.array("q", fields)
        base = held.buffer_info()[0]
        return held, [None if a is None else base + a for a in at]

    def _vector(self, t, name, shape, dtype):
        if t is None:
            return None
        if (t.get_device() != self.device.index or t.dtype != dtype or t.shape != shape
                or not t.is_contiguous()):
            raise AbftError(f"{name}: expected contiguous {shape} {dtype} on {self.device}, got "
                            f"{tuple(t.shape)} {t.dtype} on {t.device}")
        return t.data_ptr()

    def _state(self, rng, used):
        if rng is None:
            if used:
                raise AbftError("rng: dropout needs its seed and offset")
            return None
        return self._vector(rng, "rng", (2,), torch.int64)


def attn_dropout_draw(seed: int, offset: int, site: int, row: int, col: int) -> int:
    """The 16-bit draw of an element (host only): it stays if the draw is at least
    floor(65536 p + 1/2)."""
    _fits(*_U32, site=site, row=row, col=col)
    k = _lib.attn_dropout_draw(seed % 2 ** 64, offset % 2 ** 64, site, row, col)
    if k < 0:
        raise AbftError(f"attn_dropout_draw: {strerror(k)} ({k})")
    return k


@dataclasses.dataclass
class DropoutConfig:
    batch: int
    tokens: int
    cols: int
    dtype: str = "bf16"          # "bf16" | "f32"
    p: float = 0.1
    site: int = 0                # tells calls that share seed and offset apart

    def to_c(self) -> DropoutConfigC:
        _fits(*_I32, batch=self.batch, tokens=self.tokens, cols=self.cols)
        _fits(*_U32, site=self.site)
        return DropoutConfigC(self.batch, self.tokens, self.cols, _dtype_of(self.dtype, "dtype")[0],
                              self.p, self.site, 0)


class Dropout(_Op):
    """Dropout of rows [batch, tokens, cols], with an optional residual. No mask is
    stored: which elements stay follows from their position, `site` and `rng`, an
    int64 tensor (seed, offset) on the device, whose owner advances the offset from
    step to step; a backward takes the values that its forward had. Any strides with
    contiguous columns; results not given are laid out as torch.empty_like of x or
    dy (with contiguous columns), and may be an input (in place). Calls run on the
    current stream of the tensors' device."""

    def __init__(self, cfg: DropoutConfig, device="cuda"):
        self.cfg = cfg
        self.device = torch.empty(0, device=device).device
        self._c = cfg.to_c()
        self._dtype = _DTYPES[cfg.dtype][1]
        self._shapes = ((cfg.batch, cfg.tokens, cfg.cols),) * 3
        self._drops = cfg.p >= 2.0 ** -17

    def _run(self, names, x, residual, rng, y):
        if y is None:
            y = torch.empty_like(x)
            held, (x, r, o) = self._records(names, (x, residual), self._shapes, (y,))
        else:
            held, (x, r, o) = self._records(names, (x, residual, y), self._shapes)
        rng = self._state(rng, self._drops)
        _check(_call(_lib.attn_dropout, self.device, self._c, x, r, rng, o), "attn_dropout")
        return y

    def forward(self, x, rng=None, residual=None, y=None):
        """residual + dropout(x)."""
        return self._run(("x", "residual", "y"), x, residual, rng, y)

    def backward(self, dy, rng=None, dx=None):
        """dropout(dy), the gradient of x; that of the residual is dy itself."""
        return self._run(("dy", "", "dx"), dy, None, rng, dx)


@dataclasses.dataclass
class NormConfig:
    batch: int
    tokens: int
    cols: int
    dtype: str = "bf16"          # of the rows: "bf16" | "f32"
    weight_dtype: str = "f32"    # of gain and offset; their gradients are fp32
    eps: float = 1e-5
    dropout: float = 0.0         # ResidualNorm only
    site: int = 0

    def to_c(self) -> NormConfigC:
        _fits(*_I32, batch=self.batch, tokens=self.tokens, cols=self.cols)
        _fits(*_U32, site=self.site)
        return NormConfigC(self.batch, self.tokens, self.cols, _dtype_of(self.dtype, "dtype")[0],
                           _dtype_of(self.weight_dtype, "weight_dtype")[0], self.site, self.dropout,
                           self.eps)


def attn_norm_workspace_bytes(cfg: NormConfig) -> int:
    c = cfg.to_c()
    n = _lib.attn_norm_workspace_bytes(ctypes.byref(c))
    if n == 0:
        raise AbftError("invalid configuration")
    return n


class NormSaved:
    """What a forward leaves for its backward: mean and 1 / deviation of each row."""

    def __init__(self, cfg: NormConfig, device):
        self.stats = torch.empty((cfg.batch, cfg.tokens, 2), dtype=torch.float32, device=device)
        self._of = None              # the rows that they belong to

    def _keep(self, rows, held, at):
        # (tensor and storage weakly: the address alone may be another tensor's by the
        # backward; the storage for views that come and go; address and strides: held
        # from `at` on)
        self._of = weakref.ref(rows), weakref.ref(rows.untyped_storage()), held, at

    def _is_of(self, rows):
        tensor, storage, held, at = self._of
        if held[at] != rows.data_ptr():
            return False
        return tensor() is rows or storage() is rows.untyped_storage() and all(
            a == b for a, b, n in zip(held[at + 1:], rows.stride(), rows.shape[:2]) if n > 1)

    def _address(self):
        return None if self._of is None else self._of[2][self._of[3]]


class _Norm(_Op):
    def __init__(self, cfg: NormConfig, device="cuda", training=True):
        self.cfg = cfg
        self.device = torch.empty(0, device=device).device
        self._c = cfg.to_c()
        n = attn_norm_workspace_bytes(cfg)
        self.workspace = None
        if training:
            self.workspace = torch.empty(n, dtype=torch.uint8, device=self.device)
        self._saved = self.new_saved() if training else None
        self._dtype, self._wdtype = _DTYPES[cfg.dtype][1], _DTYPES[cfg.weight_dtype][1]
        self._shape, self._cols = (cfg.batch, cfg.tokens, cfg.cols), (cfg.cols,)
        self._shapes = (self._shape,) * 5
        self._any = 0 not in self._shape     # (without rows all addresses are 0)
        self._drops = cfg.dropout >= 2.0 ** -17
        if training:
            self._sums = torch.empty(cfg.cols, dtype=torch.float32, device=self.device)

    @property
    def stats(self):
        return self._saved and self._saved.stats

    def new_saved(self):
        """Another record for a forward and its backward."""
        return NormSaved(self.cfg, self.device)

    def _record(self, saved):
        if saved.stats.shape != (*self._shape[:2], 2) or saved.stats.device != self.device:
            raise AbftError("saved: made for another shape or device")
        return saved

    def _forward(self, rows, weight, bias, lens, rng, saved, of, written):
        """rows: of x, residual, h, y; of: what holds the norm's rows, and their place in
        the records (None: y does not leave them); written: the caller's h and y."""
        x, r, h, y = rows
        if lens is not None:
            lens = self._vector(lens, "lens", self._shape[:1], torch.int32)
        saved = self._saved if saved is None else self._record(saved)
        stats = None
        if saved is not None:
            stats, saved._of = saved.stats.data_ptr(), None
            if written is not None and saved is not self._saved:
                self._gone(written)
        _check(_call(_lib.attn_norm_forward, self.device, self._c, x, r,
                     self._vector(weight, "weight", self._cols, self._wdtype),
                     self._vector(bias, "bias", self._cols, self._wdtype),
                     lens, rng, h, y, stats),
               "attn_norm_forward")
        if saved is not None and of is not None:
            saved._keep(*of)

    def _of(self, saved, h):
        """The record of the rows h."""
        own = saved is None
        saved = self._saved if own else self._record(saved)
        if saved is None or self.workspace is None:
            raise AbftError("backward: made with training=False")
        if saved._of is None or own and self._any and not saved._is_of(h):
            raise AbftError("backward: the rows are not those of the last forward"
                            if saved._of is not None
                            else "backward: no forward has left its statistics")
        return saved

    def _backward(self, rows, weight, lens, rng, dweight, dbias, saved, of, written):
        """rows: of dy, dh, h, dx, dresidual; of: h itself; written: the caller's dx and
        dresidual, which may be on it."""
        dy, dh, h, dx, dr = rows
        if lens is not None:
            lens = self._vector(lens, "lens", self._shape[:1], torch.int32)
        if dweight is None:
            dweight = torch.empty_like(self._sums)
            dw = dweight.data_ptr()
        else:
            dw = self._vector(dweight, "dweight", self._cols, torch.float32)
        if dbias is None:
            dbias = torch.empty_like(self._sums)
            db = dbias.data_ptr()
        else:
            db = self._vector(dbias, "dbias", self._cols, torch.float32)
        _check(_call(_lib.attn_norm_backward, self.device, self._c, dy, dh, h,
                     self._vector(weight, "weight", self._cols, self._wdtype), saved.stats.data_ptr(),
                     lens, rng, dx, dr, dw, db,
                     self.workspace.data_ptr(), self.workspace.numel()), "attn_norm_backward")
        if written is not None and self._gone(written, of):
            saved._of = None
        return dweight, dbias

    def _gone(self, written, rows=None):
        """The caller's results `written` end the object's record if they are on its rows.
        Returns whether they are on `rows`."""
        at = [t.data_ptr() for t in written if t is not None and self._any]
        own = self._saved
        if own is not None and own._address() in at:
            own._of = None
        return rows is not None and rows.data_ptr() in at


class LayerNorm(_Norm):
    """Layer norm of rows [batch, tokens, cols]: owns the workspace of one shape
    and one record of what a forward leaves for its backward (`stats`), as
    CrossAttention does; with training=False it has neither. A forward replaces the
    record: backward raises if x is not the last forward's (its memory and layout; what
    it holds must not have changed). Where other forwards come in between, or x has
    moved since, pass a record of `new_saved` to both calls as `saved`; which x belongs
    to it is then the caller's to know. Calls run on the current stream of the tensors'
    device. Those that share workspace or record, in graphs too, must not overlap.

    weight and bias [cols] may be None (1 and 0); lens [batch] int32: tokens of
    each sequence, behind them nothing is read and results are 0. Any strides with
    contiguous columns; results not given are laid out as torch.empty_like of x or
    dy (with contiguous columns), and may be an input (in place; y or dx on x leaves no
    record for a backward)."""

    def __init__(self, cfg: NormConfig, device="cuda", training=True):
        if cfg.dropout != 0.0:
            raise AbftError("dropout stands in front of a ResidualNorm")
        super().__init__(cfg, device, training)

    def forward(self, x, weight=None, bias=None, lens=None, y=None, saved=None):
        written = None
        if y is None:
            y = torch.empty_like(x)
            held, (x_, y_) = self._records(("x",), (x,), self._shapes, (y,))
            kept = x, held, 0
        else:
            written = (y,)
            held, (x_, y_) = self._records(("x", "y"), (x, y), self._shapes)
            kept = (x, held, 0) if not self._any or held[0] != held[3] else None
        self._forward((x_, None, None, y_), weight, bias, lens, None, saved, kept, written)
        return y

    def backward(self, dy, x, weight=None, lens=None, dx=None, dweight=None, dbias=None, saved=None):
        """dx, dweight, dbias."""
        saved, written = self._of(saved, x), None
        if dx is None:
            dx = torch.empty_like(dy)
            held, (dy_, x_, o) = self._records(("dy", "x"), (dy, x), self._shapes, (dx,))
        else:
            written = (dx,)
            held, (dy_, x_, o) = self._records(("dy", "x", "dx"), (dy, x, dx), self._shapes)
        dweight, dbias = self._backward((dy_, None, x_, o, None), weight, lens, None, dweight, dbias,
                                        saved, x, written)
        return dx, dweight, dbias


class ResidualNorm(_Norm):
    """h = residual + dropout(x) as it is stored, and its layer norm y, in one pass
    each way: the same bits as Dropout and LayerNorm one after the other. Records and
    tensors as of LayerNorm (backward takes h, and raises if it is not the last
    forward's), rng as of Dropout. In place: h on x or on the residual; dx or dresidual on
    h leaves no record."""

    def forward(self, x, residual, weight=None, bias=None, rng=None, lens=None, h=None, y=None,
                saved=None):
        """h, y."""
        if residual is None:
            raise AbftError("residual: LayerNorm is the norm without one")
        written = None
        if h is None and y is None:
            h, y = torch.empty_like(x), torch.empty_like(x)
            held, rows = self._records(("x", "residual"), (x, residual), self._shapes, (h, y))
        else:
            written = (h, y)
            h = _columns(torch.empty_like(x)) if h is None else h
            y = _columns(torch.empty_like(x)) if y is None else y
            held, rows = self._records(("x", "residual", "h", "y"), (x, residual, h, y), self._shapes)
        self._forward(rows, weight, bias, lens, self._state(rng, self._drops), saved, (h, held, 6),
                      written)
        return h, y

    def backward(self, dy, h, weight=None, dh=None, rng=None, lens=None, dx=None, dresidual=None,
                 dweight=None, dbias=None, saved=None):
        """dx, dresidual, dweight, dbias. dh: what comes to h beside its norm's
        gradient. Without dropout dx and dresidual are alike: one tensor unless both
        are given."""
        saved = self._of(saved, h)
        drops, names, written = self._drops, ("dy", "dh", "h", "dx", "dresidual"), None
        if dx is None and dresidual is None:
            dx = dresidual = torch.empty_like(dy)
            fresh = (dx,)
            if drops:
                dresidual = torch.empty_like(dy)
                fresh = (dx, dresidual)
            held, rows = self._records(names, (dy, dh, h), self._shapes, fresh)
        else:
            written = (dx, dresidual)
            if dx is None:
                dx = _columns(torch.empty_like(dy)) if drops else dresidual
            if dresidual is None:
                dresidual = _columns(torch.empty_like(dy)) if drops else dx
            second = () if dresidual is dx and not drops else (dresidual,)
            held, rows = self._records(names, (dy, dh, h, dx, *second), self._shapes)
        if len(rows) == 4:
            rows.append(None)
        dweight, dbias = self._backward(rows, weight, lens, self._state(rng, drops), dweight, dbias,
                                        saved, h, written)
        return dx, dresidual, dweight, dbias


@dataclasses.dataclass
class RotaryConfig:
    batch: int
    tokens: int
    heads: int
    head_dim: int
    kv_heads: int = 0            # 0: one key head per query head
    rotary_dim: int = 0          # 0: the whole head
    interleaved: bool = False    # pairs of neighbours; else dims k and rotary_dim / 2 + k
    dtype: str = "bf16"          # "bf16" | "f32"
    base: float = 10000.0
    scaling: str = "none"        # "none" | "linear" | "parts" (attn_rotary_frequencies)
    factor: float = 1.0
    original_len: float = 2048
    low_turns: float = 1.0
    high_turns: float = 32.0
    magnitude: float = 1.0

    def to_c(self) -> RotaryConfigC:
        _fits(*_I32, batch=self.batch, tokens=self.tokens, heads=self.heads, kv_heads=self.kv_heads,
              head_dim=self.head_dim, rotary_dim=self.rotary_dim)
        return RotaryConfigC(self.batch, self.tokens, self.heads, self.kv_heads or self.heads,
                             self.head_dim, self.rotary_dim or self.head_dim, int(self.interleaved),
                             _dtype_of(self.dtype, "dtype")[0], self.magnitude)


def attn_rotary_frequencies(rotary_dim: int, base: float = 10000.0, scaling: str = "none",
                            factor: float = 1.0, original_len: float = 2048,
                            low_turns: float = 1.0, high_turns: float = 32.0) -> list:
    """Radians a position of each pair (host only)."""
    _fits(*_I32, rotary_dim=rotary_dim)
    kinds = {"none": 0, "linear": 1, "parts": 2}
    if scaling not in kinds:
        raise AbftError(f"scaling: {scaling!r} is none of {sorted(kinds)}")
    out = (ctypes.c_double * max(1, rotary_dim // 2))()
    _check(_lib.attn_rotary_frequencies(rotary_dim, base, kinds[scaling], factor, original_len,
                                        low_turns, high_turns, ctypes.addressof(out)),
           "attn_rotary_frequencies")
    return list(out)[:rotary_dim // 2]


class Rotary(_Op):
    """Rotary positions of queries and keys [batch, tokens, heads, head_dim]: holds
    the frequencies of one configuration on the device (`freqs`, fp64, which may be
    replaced by others). Token i of sequence b lies at position q_start[b] + i (q_start
    [batch] int32, None: 0), as CrossAttention has it. Any strides with contiguous
    dims; results not given are laid out as torch.empty_like of Q or K (with contiguous
    dims), and may be Q or K (in place). Calls run on the current stream of the tensors'
    device."""

    def __init__(self, cfg: RotaryConfig, device="cuda"):
        self.cfg = cfg
        self.device = torch.empty(0, device=device).device
        self._c = cfg.to_c()
        self._dtype = _DTYPES[cfg.dtype][1]
        freqs = attn_rotary_frequencies(self._c.rotary_dim, cfg.base, cfg.scaling, cfg.factor,
                                        cfg.original_len, cfg.low_turns, cfg.high_turns)
        self.freqs = torch.tensor(freqs, dtype=torch.float64, device=self.device)
        self._q_shape = (cfg.batch, cfg.tokens, cfg.heads, cfg.head_dim)
        self._k_shape = (cfg.batch, cfg.tokens, self._c.kv_heads, cfg.head_dim)

    def _at(self, q_start):
        return (self._vector(self.freqs, "freqs", (self._c.rotary_dim // 2,), torch.float64),
                self._vector(q_start, "q_start", (self.cfg.batch,), torch.int32))

    def _turn(self, backward, names, Q, K, q_start, Q_out, K_out):
        qs, ks = self._q_shape, self._k_shape
        if Q_out is None and K_out is None:
            Q_out, K_out = torch.empty_like(Q), torch.empty_like(K)
            held, (q, k, qo, ko) = self._records(names, (Q, K), (qs, ks), (Q_out, K_out))
        else:
            Q_out = _columns(torch.empty_like(Q)) if Q_out is None else Q_out
            K_out = _columns(torch.empty_like(K)) if K_out is None else K_out
            held, (q, k, qo, ko) = self._records(names, (Q, K, Q_out, K_out), (qs, ks, qs, ks))
        freqs, start = self._at(q_start)
        _check(_call(_lib.attn_rotary, self.device, self._c, backward, q, k, freqs, start, qo, ko),
               "attn_rotary")
        return Q_out, K_out

    def forward(self, Q, K, q_start=None, Q_out=None, K_out=None):
        """The turned queries and keys."""
        return self._turn(0, ("Q", "K", "Q_out", "K_out"), Q, K, q_start, Q_out, K_out)

    def backward(self, dQ, dK, q_start=None, dQ_out=None, dK_out=None):
        """Gradients of Q and K from those of the turned ones."""
        return self._turn(1, ("dQ", "dK", "dQ_out", "dK_out"), dQ, dK, q_start, dQ_out, dK_out)

    def append(self, Q, K, V, K_cache, V_cache, q_start=None, Q_out=None):
        """Returns the turned queries; turned keys and the values go to rows q_start +
        i of the caches [batch, capacity, kv_heads, head_dim] (left out where the
        caches have no such row)."""
        qs, ks = self._q_shape, self._k_shape
        capacity = K_cache.shape[1]
        if capacity >= 2 ** 31:
            raise AbftError(f"K_cache: {capacity} rows, at most 2^31 - 1 are supported")
        cs = (ks[0], capacity, ks[2], ks[3])
        names, tensors = ("Q", "K", "V", "K_cache", "V_cache", "Q_out"), (Q, K, V, K_cache, V_cache)
        if Q_out is None:
            Q_out = torch.empty_like(Q)
            held, at = self._records(names, tensors, (qs, ks, ks, cs, cs), (Q_out,))
        else:
            held, at = self._records(names, (*tensors, Q_out), (qs, ks, ks, cs, cs, qs))
        q, k, v, kc, vc, qo = at
        freqs, start = self._at(q_start)
        _check(_call(_lib.attn_rotary_append, self.device, self._c, q, k, v, freqs, start, capacity,
                     qo, kc, vc), "attn_rotary_append")
        return Q_out
