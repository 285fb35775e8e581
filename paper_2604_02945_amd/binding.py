"""Thin ctypes binding of libmsao.so (the C ABI in include/msao.h).

Argument marshalling only: torch provides device memory and the current
stream; every step of the analysis runs in the library's HIP kernels. The
library must be built in-tree (paper_2604_02945_amd/build.py); importing this
module never falls back to anything else.
"""
from __future__ import annotations

import contextlib
import ctypes
import dataclasses
import os
from typing import Dict, List, Optional, Sequence

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libmsao.so")

NMOD = 4
TEXT, IMAGE, VIDEO, AUDIO = 0, 1, 2, 3
F32, BF16 = 0, 1
FLAG_TEMPORAL_LITERAL = 1
FLAG_SELECT_PER_FRAME = 2
(KERNEL_SCORE, KERNEL_POST, KERNEL_GATHER, KERNEL_ENTROPY, KERNEL_HEAD, KERNEL_SIMHASH, KERNEL_HASH_POST,
 KERNEL_CLIP, KERNEL_READ, NUM_KERNELS) = 0, 1, 2, 3, 4, 5, 6, 7, 8, 9
MODAL_DESC = 8
DECIDE_HOLD, DECIDE_SEND, DECIDE_OFFLOAD = 0, 1, 2
MAX_AXES = 4
APPEND_NEIGHBOURS = 1
ATTEND_CAUSAL, ATTEND_WEIGHT = 1, 2
(CACHE_KERNEL_APPEND, CACHE_KERNEL_ATTEND, CACHE_KERNEL_COMBINE, CACHE_KERNEL_WEIGHT,
 CACHE_KERNEL_WEIGHT_JOIN, CACHE_KERNEL_SELECT, CACHE_KERNEL_MOVE, NUM_CACHE_KERNELS) = 0, 1, 2, 3, 4, 5, 6, 7

STATUS = {0: "MSAO_OK", 1: "MSAO_ERR_INVALID_ARG", 2: "MSAO_ERR_ALIGNMENT", 3: "MSAO_ERR_WORKSPACE",
          4: "MSAO_ERR_UNSUPPORTED", 5: "MSAO_ERR_HIP"}

_P = ctypes.c_void_p


class MsaoSegment(ctypes.Structure):
    _fields_ = [("data", _P), ("row_stride", ctypes.c_int64), ("request", ctypes.c_int32),
                ("modality", ctypes.c_int32), ("n_frames", ctypes.c_int32),
                ("tokens_per_frame", ctypes.c_int32), ("hidden", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("keep_ratio", ctypes.c_float)]


class MsaoParams(ctypes.Structure):
    _fields_ = [("tau", ctypes.c_float), ("tau_s", ctypes.c_float),
                ("lambda_s", ctypes.c_float * NMOD), ("lambda_t", ctypes.c_float * NMOD),
                ("flags", ctypes.c_uint32)]


class MsaoTokenOut(ctypes.Structure):
    _fields_ = [(n, _P) for n in ("z", "l1", "l2", "info", "d", "res")]


class MsaoFrameOut(ctypes.Structure):
    _fields_ = [(n, _P) for n in ("dframe", "sim", "gamma")]


class MsaoReqOut(ctypes.Structure):
    _fields_ = [(n, _P) for n in ("agg", "rho", "temporal", "beta", "mas", "present")]


class MsaoSelectOut(ctypes.Structure):
    _fields_ = [(n, _P) for n in ("keep", "kept_idx", "kept_count")]


class MsaoSpatialHead(ctypes.Structure):
    _fields_ = [("weight", _P), ("bias", ctypes.c_float), ("grid_w", ctypes.c_int32), ("pool", ctypes.c_int32)]


class MsaoModalMlp(ctypes.Structure):
    _fields_ = [("w1", _P), ("b1", _P), ("w2", _P), ("b2", ctypes.c_float), ("hidden", ctypes.c_int32),
                ("prompt_dim", ctypes.c_int32), ("prompt", _P)]


class MsaoSimHash(ctypes.Structure):
    _fields_ = [("planes", _P), ("bits", ctypes.c_int32)]


class MsaoEntropyOut(ctypes.Structure):
    _fields_ = [(n, _P) for n in ("entropy", "entropy_norm", "draft_token", "speculate")]


class MsaoSchedParams(ctypes.Structure):
    _fields_ = [("p_target", ctypes.c_double), ("n_max", ctypes.c_int32), ("quantile", ctypes.c_double),
                ("delta", ctypes.c_double), ("theta_min", ctypes.c_double), ("alpha", ctypes.c_double)]


class MsaoSchedState(ctypes.Structure):
    _fields_ = [("theta", ctypes.c_double), ("p_conf", ctypes.c_double), ("n_draft", ctypes.c_int32),
                ("cache", ctypes.c_int32), ("cache_h", ctypes.c_double), ("steps", ctypes.c_int64),
                ("held", ctypes.c_int64), ("sends", ctypes.c_int64), ("offloads", ctypes.c_int64),
                ("tokens_sent", ctypes.c_int64)]


class MsaoLatencyModel(ctypes.Structure):
    _fields_ = [("prefill_edge", ctypes.c_double), ("prefill_cloud", ctypes.c_double),
                ("comm_offloaded", ctypes.c_double), ("p_conf", ctypes.c_double), ("n_draft", ctypes.c_int32),
                ("t_draft", ctypes.c_double), ("t_verify", ctypes.c_double), ("t_offload", ctypes.c_double)]


class MsaoKvCache(ctypes.Structure):
    _fields_ = [("k", _P), ("v", _P), ("k_stride", ctypes.c_int64 * 3), ("v_stride", ctypes.c_int64 * 3),
                ("dtype", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("n_pages", ctypes.c_int32), ("n_seqs", ctypes.c_int32),
                ("pages_per_seq", ctypes.c_int32), ("table_stride", ctypes.c_int64), ("pages", _P), ("length", _P),
                ("weight", _P), ("weight_stride", ctypes.c_int64)]


class MsaoChunk(ctypes.Structure):
    _fields_ = [("start", _P), ("n_rows", ctypes.c_int32), ("max_new", ctypes.c_int32)]


class MsaoAppend(ctypes.Structure):
    _fields_ = [("q", _P), ("q_out", _P), ("k", _P), ("v", _P), ("q_stride", ctypes.c_int64),
                ("q_out_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64),
                ("q_norm", _P), ("k_norm", _P), ("eps", ctypes.c_float), ("heads", ctypes.c_int32),
                ("rot_dim", ctypes.c_int32), ("inv_freq", _P), ("positions", _P), ("position_stride", ctypes.c_int64),
                ("n_axes", ctypes.c_int32), ("sections", ctypes.c_int32 * MAX_AXES), ("flags", ctypes.c_uint32)]


class MsaoError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS.get(status, status)}: {message}")
        self.status = status


_lib = None

# (name, restype, argtypes) of every entry point in include/msao.h
SIGNATURES = [
    ("msao_create", ctypes.c_int, [ctypes.POINTER(_P), ctypes.c_int]),
    ("msao_destroy", None, [_P]),
    ("msao_last_error", ctypes.c_char_p, [_P]),
    ("msao_last_error_global", ctypes.c_char_p, []),
    ("msao_status_string", ctypes.c_char_p, [ctypes.c_int]),
    ("msao_default_params", MsaoParams, []),
    ("msao_validate", ctypes.c_int, [_P, ctypes.c_int, ctypes.c_int, _P]),
    ("msao_count", ctypes.c_int, [_P, ctypes.c_int, _P, _P]),
    ("msao_workspace_size", ctypes.c_int, [_P, ctypes.c_int, ctypes.c_int, _P]),
    ("msao_compact_layout", ctypes.c_int, [_P, ctypes.c_int, _P, _P]),
    ("msao_mas_score", ctypes.c_int, [_P, _P, ctypes.c_int, ctypes.c_int, _P, _P, _P, _P, _P, _P,
                                      ctypes.c_size_t, _P]),
    ("msao_temporal_redundancy", ctypes.c_int, [_P, _P, ctypes.c_int, ctypes.c_int, _P, _P, _P, _P, _P, _P,
                                                ctypes.c_size_t, _P]),
    ("msao_select_tokens", ctypes.c_int, [_P, _P, ctypes.c_int, ctypes.c_int, _P, _P, _P, _P, _P, _P,
                                          ctypes.c_size_t, _P]),
    ("msao_compact", ctypes.c_int, [_P, _P, ctypes.c_int, _P, _P, _P, _P, ctypes.c_int64, _P,
                                    ctypes.c_size_t, _P]),
    ("msao_run", ctypes.c_int, [_P, _P, ctypes.c_int, ctypes.c_int, _P, _P, _P, _P, _P, _P, _P, _P,
                                ctypes.c_int64, _P, ctypes.c_size_t, _P]),
    ("msao_run_noalloc", ctypes.c_int, [_P, _P, ctypes.c_int, ctypes.c_int, _P, _P, _P, _P, _P, _P, _P, _P,
                                        ctypes.c_int64, _P]),
    ("msao_plan_create", ctypes.c_int, [_P, _P, ctypes.c_int, ctypes.c_int, _P, _P, _P, _P, ctypes.c_size_t, _P,
                                        ctypes.POINTER(_P)]),
    ("msao_plan_run", ctypes.c_int, [_P, _P, _P, _P, _P, _P, ctypes.c_int64, _P]),
    ("msao_plan_destroy", None, [_P]),
    ("msao_set_profiling", ctypes.c_int, [_P, ctypes.c_int]),
    ("msao_kernel_times", ctypes.c_int, [_P, _P]),
    ("msao_mas_score_learned", ctypes.c_int, [_P, _P, ctypes.c_int, ctypes.c_int, _P, _P, _P, _P, _P, _P, _P, _P,
                                              _P, _P, _P, ctypes.c_size_t, _P]),
    ("msao_run_learned", ctypes.c_int, [_P, _P, ctypes.c_int, ctypes.c_int, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P,
                                        _P, _P, _P, ctypes.c_int64, _P, ctypes.c_size_t, _P]),
    ("msao_temporal_simhash", ctypes.c_int, [_P, _P, ctypes.c_int, ctypes.c_int, _P, _P, _P, _P, _P, _P, _P,
                                             ctypes.c_size_t, _P]),
    ("msao_run_simhash", ctypes.c_int, [_P, _P, ctypes.c_int, ctypes.c_int, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P,
                                        ctypes.c_int64, _P, ctypes.c_size_t, _P]),
    ("msao_draft_entropy", ctypes.c_int, [_P, _P, ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, ctypes.c_int,
                                          ctypes.c_float, _P, _P]),
    ("msao_cache_validate", ctypes.c_int, [_P, _P]),
    ("msao_cache_append", ctypes.c_int, [_P, _P, _P, _P, _P]),
    ("msao_cache_attention", ctypes.c_int, [_P, _P, _P, _P, ctypes.c_int64, ctypes.c_int, ctypes.c_float,
                                            ctypes.c_uint32, _P, ctypes.c_int64, _P, _P, ctypes.c_size_t, _P]),
    ("msao_cache_attention_workspace", ctypes.c_int, [_P, _P, ctypes.c_int, ctypes.c_uint32, _P]),
    ("msao_cache_evict", ctypes.c_int, [_P, _P, _P, _P, ctypes.c_int, ctypes.c_int, _P, ctypes.c_int64, _P,
                                        ctypes.c_size_t, _P]),
    ("msao_cache_evict_workspace", ctypes.c_int, [_P, _P]),
    ("msao_cache_kernel_times", ctypes.c_int, [_P, _P]),
    ("msao_stream_read", ctypes.c_int, [_P, _P, ctypes.c_int64, ctypes.c_int, _P, ctypes.c_int64, _P]),
    ("msao_sched_default_params", MsaoSchedParams, []),
    ("msao_sched_init", ctypes.c_int, [_P, ctypes.c_int64, _P, _P]),
    ("msao_sched_step", ctypes.c_int, [_P, _P, ctypes.c_float, _P]),
    ("msao_sched_run", ctypes.c_int, [_P, _P, _P, ctypes.c_int64, _P, _P]),
    ("msao_retention_floor", ctypes.c_int, [_P, ctypes.c_int, _P]),
    ("msao_comm_latency", ctypes.c_double, [ctypes.c_double, ctypes.c_double, ctypes.c_double]),
    ("msao_p_conf", ctypes.c_double, [_P, ctypes.c_int64, ctypes.c_double]),
    ("msao_expected_spec_tokens", ctypes.c_double, [ctypes.c_double]),
    ("msao_expected_e2e_latency", ctypes.c_double, [_P]),
]


def lib() -> ctypes.CDLL:
    """Load the in-tree libmsao.so; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with paper_2604_02945_amd/build.py "
                               "(or __graft_entry__.build()); there is no fallback path")
        L = ctypes.CDLL(LIB_PATH)
        for name, res, args in SIGNATURES:
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _addr(struct) -> ctypes.c_void_p:
    return ctypes.cast(ctypes.byref(struct), ctypes.c_void_p)


def default_params() -> dict:
    p = lib().msao_default_params()
    return {"tau": p.tau, "tau_s": p.tau_s, "lambda_s": list(p.lambda_s), "lambda_t": list(p.lambda_t),
            "flags": p.flags}


def params_struct(p: Optional[dict]) -> MsaoParams:
    if p is None:
        return lib().msao_default_params()
    q = MsaoParams()
    q.tau, q.tau_s = p["tau"], p["tau_s"]
    for m in range(NMOD):
        q.lambda_s[m] = p["lambda_s"][m]
        q.lambda_t[m] = p["lambda_t"][m]
    q.flags = p.get("flags", 0)
    return q


@dataclasses.dataclass
class DeviceSegment:
    """A modality-tagged activation tensor on the device.

    `data` is [rows, hidden] (row stride may exceed hidden) with rows = n_frames
    * tokens_per_frame, float32 or bfloat16.
    """
    data: torch.Tensor
    request: int
    modality: int
    keep_ratio: float
    n_frames: int = 1

    @property
    def rows(self) -> int:
        return int(self.data.shape[0])


def segment_table(segments: Sequence[DeviceSegment]):
    arr = (MsaoSegment * max(1, len(segments)))()
    for i, s in enumerate(segments):
        t = s.data
        if t.dim() != 2:
            raise ValueError("segment data must be a 2-D [rows, hidden] tensor")
        if t.dtype not in (torch.float32, torch.bfloat16):
            raise ValueError("segment data must be float32 or bfloat16")
        if t.numel() and t.stride(1) != 1:
            raise ValueError("rows must be contiguous")
        if s.rows % s.n_frames:
            raise ValueError("rows must be a multiple of n_frames")
        arr[i].data = t.data_ptr() if t.numel() else None
        arr[i].row_stride = t.stride(0) if t.shape[0] > 1 else t.shape[1]
        arr[i].request = s.request
        arr[i].modality = s.modality
        arr[i].n_frames = s.n_frames
        arr[i].tokens_per_frame = s.rows // s.n_frames
        arr[i].hidden = t.shape[1]
        arr[i].dtype = F32 if t.dtype == torch.float32 else BF16
        arr[i].keep_ratio = s.keep_ratio
    return arr


def _check(status: int, ctx: Optional["Context"] = None):
    if status != 0:
        msg = (lib().msao_last_error(ctx.handle) if ctx is not None else lib().msao_last_error_global()) or b""
        raise MsaoError(status, msg.decode())


class Context:
    """An msao_ctx bound to one device; one per concurrently used stream."""

    def __init__(self, device: int = 0):
        h = ctypes.c_void_p()
        _check(lib().msao_create(ctypes.byref(h), device))
        self.handle = h
        self.device = device

    def close(self):
        if getattr(self, "handle", None):
            lib().msao_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_profiling(self, enable: bool):
        _check(lib().msao_set_profiling(self.handle, 1 if enable else 0), self)

    def kernel_times(self) -> List[float]:
        ms = (ctypes.c_float * NUM_KERNELS)()
        _check(lib().msao_kernel_times(self.handle, ms), self)
        return list(ms)

    def cache_kernel_times(self) -> List[float]:
        ms = (ctypes.c_float * NUM_CACHE_KERNELS)()
        _check(lib().msao_cache_kernel_times(self.handle, ms), self)
        return list(ms)


_default_ctx: Dict[int, Context] = {}


def default_context(device: int) -> Context:
    if device not in _default_ctx:
        _default_ctx[device] = Context(device)
    return _default_ctx[device]


def sizes(segments: Sequence[DeviceSegment], n_requests: int):
    """(total tokens, total temporal frames, workspace bytes) of a segment table."""
    segt = segment_table(segments)
    nt, nf = ctypes.c_int64(), ctypes.c_int64()
    _check(lib().msao_count(segt, len(segments), ctypes.byref(nt), ctypes.byref(nf)))
    ws = ctypes.c_size_t()
    _check(lib().msao_workspace_size(segt, len(segments), n_requests, ctypes.byref(ws)))
    return nt.value, nf.value, ws.value


def compact_layout(segments: Sequence[DeviceSegment]):
    segt = segment_table(segments)
    off = (ctypes.c_int64 * max(1, len(segments)))()
    total = ctypes.c_int64()
    _check(lib().msao_compact_layout(segt, len(segments), off, ctypes.byref(total)))
    return [off[i] for i in range(len(segments))], total.value


def _workspace(nbytes: int, device) -> torch.Tensor:
    buf = torch.empty(max(nbytes, 1) + 256, dtype=torch.uint8, device=device)
    shift = (-buf.data_ptr()) % 256
    return buf[shift:shift + max(nbytes, 1)]


def _device_of(segments) -> torch.device:
    for s in segments:
        return s.data.device
    return torch.device("cuda", torch.cuda.current_device())


class Outputs:
    """Device buffers of every output of the analysis for one segment table."""

    def __init__(self, segments: Sequence[DeviceSegment], n_requests: int, device=None,
                 token_fields=("z", "l1", "l2", "info", "d", "res"), compact: bool = True,
                 workspace: bool = True):
        device = device or _device_of(segments)
        ntok, nfr, ws = sizes(segments, n_requests)
        self.ntok, self.nframes, self.ws_bytes = ntok, nfr, ws
        R, n = n_requests, len(segments)
        e = lambda k, dt: torch.empty(max(k, 1), dtype=dt, device=device)  # noqa: E731
        tk = {"z": torch.int32, "l1": torch.float32, "l2": torch.float32, "info": torch.float32,
              "d": torch.int32, "res": torch.float32}
        self.tok = {f: e(ntok, tk[f]) for f in token_fields}
        self.frm = {"dframe": e(nfr, torch.int64), "sim": e(nfr, torch.float32), "gamma": e(nfr, torch.float32)}
        self.req = {"agg": e(R * NMOD * 4, torch.int64), "rho": e(R * NMOD, torch.float32),
                    "temporal": e(R * NMOD, torch.float32), "beta": e(R * NMOD, torch.float32),
                    "mas": e(R * NMOD, torch.float32), "present": e(R * NMOD, torch.uint8)}
        self.sel = {"keep": e(ntok, torch.uint8), "kept_idx": e(ntok, torch.int32),
                    "kept_count": e(n, torch.int32)}
        # msao_run_noalloc takes no workspace (workspace=False leaves it out)
        self.workspace = _workspace(ws, device) if workspace else None
        self.out = None
        self.out_off = None
        if compact:
            offs, total = compact_layout(segments)
            self.out = e(total, torch.uint8)
            self.out_off = (ctypes.c_int64 * max(1, n))(*offs)
            self.out_bytes = total
        self._structs()

    def _structs(self):
        g = lambda d, k: _ptr(d.get(k))  # noqa: E731
        self.c_tok = MsaoTokenOut(*[g(self.tok, k) for k in ("z", "l1", "l2", "info", "d", "res")])
        self.c_frm = MsaoFrameOut(*[g(self.frm, k) for k in ("dframe", "sim", "gamma")])
        self.c_req = MsaoReqOut(*[g(self.req, k) for k in ("agg", "rho", "temporal", "beta", "mas", "present")])
        self.c_sel = MsaoSelectOut(*[g(self.sel, k) for k in ("keep", "kept_idx", "kept_count")])

    def results(self, n_requests: int, n_segments: int) -> dict:
        """Outputs trimmed to their logical sizes (still on the device)."""
        R, n, nt, nf = n_requests, n_segments, self.ntok, self.nframes
        r = {k: v[:nt] for k, v in self.tok.items()}
        r.update({k: v[:nf] for k, v in self.frm.items()})
        r.update({k: v[: (R * NMOD * 4 if k == "agg" else R * NMOD)] for k, v in self.req.items()})
        r["keep"] = self.sel["keep"][:nt]
        r["kept_idx"] = self.sel["kept_idx"][:nt]
        r["kept_count"] = self.sel["kept_count"][:n]
        return r


def _stream_ptr(stream, device: Optional[torch.device] = None) -> ctypes.c_void_p:
    """The handle of `stream`, or of the current stream of `device` (of the
    current device when None). The handle is read without building a
    torch.cuda.Stream, which takes 3 us, a fifth of a small call."""
    if stream is not None:
        return ctypes.c_void_p(stream.cuda_stream)
    if device is not None and device.type != "cuda":
        raise ValueError(f"expected a cuda device, got {device}")
    torch.cuda.init()
    index = device.index if device is not None and device.index is not None else torch.cuda.current_device()
    return ctypes.c_void_p(torch._C._cuda_getCurrentRawStream(index))


class Call:
    """Prepared arguments of one entry point, reusable across launches (the
    segment table and output pointers are marshalled once)."""

    def __init__(self, fn_name: str, args: list, ctx: Context, keep_alive: list):
        self.fn = getattr(lib(), fn_name)
        self.args = args
        self.ctx = ctx
        self.keep_alive = keep_alive

    def __call__(self, stream=None):
        _check(self.fn(*self.args[:-1], _stream_ptr(stream)), self.ctx)


def prepare(entry: str, segments: Sequence[DeviceSegment], n_requests: int, outputs: Outputs,
            params: Optional[dict] = None, alpha: Optional[Sequence[float]] = None,
            ctx: Optional[Context] = None, mas: Optional[torch.Tensor] = None,
            z: Optional[torch.Tensor] = None, d: Optional[torch.Tensor] = None,
            compact: bool = True) -> Call:
    """Marshal the arguments of entry point `entry` (msao_run, msao_mas_score, ...)."""
    device = _device_of(segments)
    ctx = ctx or default_context(device.index if device.index is not None else torch.cuda.current_device())
    segt = segment_table(segments)
    prm = params_struct(params)
    n, R = len(segments), n_requests
    al = None
    if alpha is not None:
        vals = list(alpha)
        if len(vals) != R * NMOD:
            raise ValueError("alpha needs n_requests * 4 logits")
        al = (ctypes.c_float * len(vals))(*vals)
    o = outputs
    ws = _ptr(o.workspace)
    wsb = ctypes.c_size_t(o.ws_bytes)
    keep = [segt, prm, al, o, mas, z, d]
    if entry == "msao_run":
        out = _ptr(o.out) if (compact and o.out is not None) else None
        off = o.out_off if (compact and o.out is not None) else None
        ob = ctypes.c_int64(o.out_bytes if out is not None else 0)
        args = [ctx.handle, segt, n, R, _addr(prm), al, _addr(o.c_tok), _addr(o.c_frm), _addr(o.c_req),
                _addr(o.c_sel), out, off, ob, ws, wsb, None]
    elif entry == "msao_run_noalloc":
        out = _ptr(o.out) if (compact and o.out is not None) else None
        off = o.out_off if (compact and o.out is not None) else None
        ob = ctypes.c_int64(o.out_bytes if out is not None else 0)
        args = [ctx.handle, segt, n, R, _addr(prm), al, _addr(o.c_tok), _addr(o.c_frm), _addr(o.c_req),
                _addr(o.c_sel), out, off, ob, None]
    elif entry == "msao_mas_score":
        args = [ctx.handle, segt, n, R, _addr(prm), al, _addr(o.c_tok), _addr(o.c_frm), _addr(o.c_req),
                ws, wsb, None]
    elif entry == "msao_temporal_redundancy":
        args = [ctx.handle, segt, n, R, _addr(prm), _ptr(o.tok.get("d")), _ptr(o.tok.get("res")),
                _addr(o.c_frm), _ptr(o.req["temporal"]), ws, wsb, None]
    elif entry == "msao_select_tokens":
        zz = z if z is not None else o.tok["z"]
        dd = d if d is not None else o.tok.get("d")
        args = [ctx.handle, segt, n, R, _addr(prm), _ptr(zz), _ptr(dd), _ptr(mas), _addr(o.c_sel),
                ws, wsb, None]
    elif entry == "msao_compact":
        args = [ctx.handle, segt, n, _ptr(o.sel["kept_idx"]), _ptr(o.sel["kept_count"]), _ptr(o.out),
                o.out_off, ctypes.c_int64(o.out_bytes), ws, wsb, None]
    else:
        raise ValueError(f"unknown entry point {entry}")
    return Call(entry, args, ctx, keep)


class Plan:
    """msao_plan: the tables of one segment table uploaded once into the
    workspace of `outputs`; each call enqueues the three launches of msao_run
    with no host-to-device copy. The segments' input buffers and `outputs`
    must outlive the plan. The upload is enqueued on `stream` (the current
    stream when None) and waited for before the constructor returns, so runs
    may then be launched on any stream."""

    def __init__(self, segments: Sequence[DeviceSegment], n_requests: int, outputs: Outputs,
                 params: Optional[dict] = None, alpha: Optional[Sequence[float]] = None,
                 ctx: Optional[Context] = None, compact: bool = True, stream=None):
        device = _device_of(segments)
        self.ctx = ctx or default_context(device.index if device.index is not None else torch.cuda.current_device())
        self.segt = segment_table(segments)
        self.prm = params_struct(params)
        n, R = len(segments), n_requests
        self.al = None
        if alpha is not None:
            vals = list(alpha)
            if len(vals) != R * NMOD:
                raise ValueError("alpha needs n_requests * 4 logits")
            self.al = (ctypes.c_float * len(vals))(*vals)
        o = self.outputs = outputs
        self.compact = compact and o.out is not None
        h = ctypes.c_void_p()
        up = stream if stream is not None else torch.cuda.current_stream(device)
        _check(lib().msao_plan_create(self.ctx.handle, self.segt, n, R, _addr(self.prm), self.al,
                                      o.out_off if self.compact else None, _ptr(o.workspace),
                                      ctypes.c_size_t(o.ws_bytes), _stream_ptr(up), ctypes.byref(h)), self.ctx)
        self.handle = h
        # the tables must be in the workspace before a run on another stream reads them
        up.synchronize()
        self.segments = list(segments)
        self._args = [h, _addr(o.c_tok), _addr(o.c_frm), _addr(o.c_req), _addr(o.c_sel),
                      _ptr(o.out) if self.compact else None,
                      ctypes.c_int64(o.out_bytes if self.compact else 0)]

    def __call__(self, stream=None):
        _check(lib().msao_plan_run(*self._args, _stream_ptr(stream)), self.ctx)

    def close(self):
        if getattr(self, "handle", None):
            lib().msao_plan_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _one_shot(entry, segments, n_requests, params=None, alpha=None, ctx=None, outputs=None, stream=None,
              compact=True, **kw):
    o = outputs or Outputs(segments, n_requests, compact=compact)
    prepare(entry, segments, n_requests, o, params, alpha, ctx, compact=compact, **kw)(stream)
    return o


def msao_mas_score(segments, n_requests, params=None, alpha=None, ctx=None, outputs=None, stream=None):
    """Per-token statistics, per-frame terms and per-modality MAS (Sec. 4.1)."""
    return _one_shot("msao_mas_score", segments, n_requests, params, alpha, ctx, outputs, stream, compact=False)


def msao_temporal_redundancy(segments, n_requests, params=None, ctx=None, outputs=None, stream=None):
    """Eq. 5 terms only: d, res, per-frame D/sim/gamma, temporal term per (request, modality)."""
    return _one_shot("msao_temporal_redundancy", segments, n_requests, params, None, ctx, outputs, stream,
                     compact=False)


def msao_temporal_simhash(segments, n_requests, hashes, params=None, ctx=None, outputs=None, stream=None, sig=None):
    """Eq. 5 with SimHash: hashes[s] = dict(planes=[bits, hidden] device
    tensor in the segment's dtype, bits) for temporal segments (None
    elsewhere). Fills outputs.tok["d"], outputs.frm and outputs.req["temporal"];
    returns (outputs, sig) with sig the [total tokens] int64 signatures."""
    device = _device_of(segments)
    ctx = ctx or default_context(device.index if device.index is not None else torch.cuda.current_device())
    o = outputs or Outputs(segments, n_requests, compact=False)
    segt = segment_table(segments)
    prm = params_struct(params)
    n = len(segments)
    harr, keep = _hash_array(hashes, n)
    if sig is None:
        sig = torch.empty(max(o.ntok, 1), dtype=torch.int64, device=device)[:o.ntok]
    st = _stream_ptr(stream, device)
    _check(lib().msao_temporal_simhash(ctx.handle, segt, n, n_requests, _addr(prm), ctypes.cast(harr, _P),
                                       _ptr(sig) if o.ntok else None, _ptr(o.tok["d"]) if o.ntok else None,
                                       _addr(o.c_frm), _ptr(o.req["temporal"]), _ptr(o.workspace),
                                       ctypes.c_size_t(o.ws_bytes), st), ctx)
    return o, sig


def _hash_array(hashes, n):
    harr = (MsaoSimHash * max(1, n))()
    keep = [harr]
    for i, h in enumerate(hashes):
        if h is None:
            continue
        keep.append(h["planes"])
        harr[i] = MsaoSimHash(h["planes"].data_ptr(), int(h["bits"]))
    return harr, keep


def msao_run_simhash(segments, n_requests, hashes, params=None, alpha=None, ctx=None, outputs=None, stream=None,
                     compact=True, sig=None):
    """msao_run with SimHash as Eq. 5's hash (hashes as for
    msao_temporal_simhash): returns (outputs, sig)."""
    device = _device_of(segments)
    ctx = ctx or default_context(device.index if device.index is not None else torch.cuda.current_device())
    o = outputs or Outputs(segments, n_requests, compact=compact)
    segt = segment_table(segments)
    prm = params_struct(params)
    n, R = len(segments), n_requests
    harr, keep = _hash_array(hashes, n)
    al = None
    if alpha is not None:
        vals = list(alpha)
        if len(vals) != R * NMOD:
            raise ValueError("alpha needs n_requests * 4 logits")
        al = (ctypes.c_float * len(vals))(*vals)
    if sig is None:
        sig = torch.empty(max(o.ntok, 1), dtype=torch.int64, device=device)[:o.ntok]
    use_out = compact and o.out is not None
    st = _stream_ptr(stream, device)
    _check(lib().msao_run_simhash(ctx.handle, segt, n, R, _addr(prm), ctypes.cast(harr, _P), al, _addr(o.c_tok),
                                  _ptr(sig) if o.ntok else None, _addr(o.c_frm), _addr(o.c_req), _addr(o.c_sel),
                                  _ptr(o.out) if use_out else None, o.out_off if use_out else None,
                                  ctypes.c_int64(o.out_bytes if use_out else 0), _ptr(o.workspace),
                                  ctypes.c_size_t(o.ws_bytes), st), ctx)
    del keep
    return o, sig


def prepare_simhash(entry, segments, n_requests, hashes, outputs, sig, params=None, alpha=None, ctx=None,
                    compact=True) -> Call:
    """msao_run_simhash's or msao_temporal_simhash's arguments (entry) marshalled
    once, as prepare() does for the other entry points; sig is the caller's
    [total tokens] int64 signature tensor."""
    device = _device_of(segments)
    ctx = ctx or default_context(device.index if device.index is not None else torch.cuda.current_device())
    o = outputs
    segt = segment_table(segments)
    prm = params_struct(params)
    n, R = len(segments), n_requests
    harr, keep = _hash_array(hashes, n)
    al = None
    if alpha is not None:
        vals = list(alpha)
        if len(vals) != R * NMOD:
            raise ValueError("alpha needs n_requests * 4 logits")
        al = (ctypes.c_float * len(vals))(*vals)
    keep += [segt, prm, al, o, sig]
    if entry == "msao_run_simhash":
        use_out = compact and o.out is not None
        args = [ctx.handle, segt, n, R, _addr(prm), ctypes.cast(harr, _P), al, _addr(o.c_tok),
                _ptr(sig) if o.ntok else None, _addr(o.c_frm), _addr(o.c_req), _addr(o.c_sel),
                _ptr(o.out) if use_out else None, o.out_off if use_out else None,
                ctypes.c_int64(o.out_bytes if use_out else 0), _ptr(o.workspace), ctypes.c_size_t(o.ws_bytes), None]
    elif entry == "msao_temporal_simhash":
        args = [ctx.handle, segt, n, R, _addr(prm), ctypes.cast(harr, _P), _ptr(sig) if o.ntok else None,
                _ptr(o.tok["d"]) if o.ntok else None, _addr(o.c_frm), _ptr(o.req["temporal"]), _ptr(o.workspace),
                ctypes.c_size_t(o.ws_bytes), None]
    else:
        raise ValueError(f"unknown SimHash entry point {entry}")
    return Call(entry, args, ctx, keep)


def msao_select_tokens(segments, n_requests, z, d=None, mas=None, params=None, ctx=None, outputs=None,
                       stream=None):
    """Per-segment top-k selection from z (and d); mas for MAS-guided keep ratios."""
    return _one_shot("msao_select_tokens", segments, n_requests, params, None, ctx, outputs, stream,
                     compact=False, z=z, d=d, mas=mas)


def msao_compact(segments, outputs, ctx=None, stream=None):
    """Packed copy of the kept rows named by outputs.sel (kept_idx, kept_count)."""
    n_req = max((s.request for s in segments), default=-1) + 1
    prepare("msao_compact", segments, n_req, outputs, None, None, ctx)(stream)
    return outputs


def msao_run(segments, n_requests, params=None, alpha=None, ctx=None, outputs=None, stream=None, compact=True):
    """Scoring, MAS, selection and compaction in one call."""
    return _one_shot("msao_run", segments, n_requests, params, alpha, ctx, outputs, stream, compact=compact)


def msao_run_noalloc(segments, n_requests, params=None, alpha=None, ctx=None, outputs=None, stream=None,
                     compact=True):
    """msao_run on the library's own scratch (no workspace; the call
    allocates nothing). `outputs` may be built with workspace=False."""
    return _one_shot("msao_run_noalloc", segments, n_requests, params, alpha, ctx, outputs, stream,
                     compact=compact)


def compacted_rows(segments: Sequence[DeviceSegment], outputs: Outputs, kept_count) -> list:
    """Views of each segment's packed kept rows in outputs.out (after synchronising)."""
    offs, _ = compact_layout(segments)
    rows = []
    for s, off, k in zip(segments, offs, kept_count):
        es = 4 if s.data.dtype == torch.float32 else 2
        nb = int(k) * s.data.shape[1] * es
        view = outputs.out[off:off + nb]
        rows.append(view.view(s.data.dtype).view(int(k), s.data.shape[1]))
    return rows


# ---- Sec. 4.2: draft confidence (GPU) and Algorithm 1 (host) ------------------

def msao_draft_entropy(logits: torch.Tensor, theta: float, vocab: Optional[int] = None, ctx: Optional[Context] = None,
                       stream=None, outputs: Optional[Dict[str, torch.Tensor]] = None) -> Dict[str, torch.Tensor]:
    """Eq. 9-10 per row of a [rows, row_stride] float32/bfloat16 device tensor
    (the first `vocab` columns are the logits). Returns device tensors
    entropy (nats), entropy_norm, draft_token and speculate."""
    if logits.dim() != 2 or logits.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("logits must be a 2-D float32 or bfloat16 tensor")
    if logits.numel() and logits.stride(1) != 1:
        raise ValueError("rows must be contiguous")
    rows = int(logits.shape[0])
    V = int(logits.shape[1]) if vocab is None else int(vocab)
    stride = int(logits.stride(0)) if rows > 1 else int(logits.shape[1])
    dev = logits.device
    if ctx is None:
        ctx = default_context(dev.index if dev.index is not None else torch.cuda.current_device())
    o = outputs or {"entropy": torch.empty(rows, dtype=torch.float32, device=dev),
                    "entropy_norm": torch.empty(rows, dtype=torch.float32, device=dev),
                    "draft_token": torch.empty(rows, dtype=torch.int32, device=dev),
                    "speculate": torch.empty(rows, dtype=torch.uint8, device=dev)}
    out = MsaoEntropyOut(*[_ptr(o.get(k)) for k in ("entropy", "entropy_norm", "draft_token", "speculate")])
    st = _stream_ptr(stream, dev)
    dt = F32 if logits.dtype == torch.float32 else BF16
    _check(lib().msao_draft_entropy(ctx.handle, _ptr(logits) if logits.numel() else None, rows, V, stride, dt,
                                    float(theta), _addr(out), st), ctx)
    return o


def msao_stream_read(data: torch.Tensor, chunk_kib: int = 8, ctx: Optional[Context] = None, stream=None,
                     sink: Optional[torch.Tensor] = None) -> torch.Tensor:
    """A plain streaming read of a contiguous device tensor (the read
    ceiling of the HBM-bound passes); returns the sink of one XOR per
    wavefront."""
    nbytes = data.numel() * data.element_size()
    dev = data.device
    if ctx is None:
        ctx = default_context(dev.index if dev.index is not None else torch.cuda.current_device())
    waves = -(-nbytes // (chunk_kib * 1024))
    if sink is None:
        sink = torch.empty(max(waves, 1), dtype=torch.int32, device=dev)
    st = _stream_ptr(stream, dev)
    _check(lib().msao_stream_read(ctx.handle, _ptr(data), nbytes, int(chunk_kib), _ptr(sink), sink.numel(),
                                  st), ctx)
    return sink


# ---- Sec. 4.2: the paged cache that drafts are verified over -------------------

# (These run before every launch of a serving step, so they ask each tensor once.)

def _same_device(index: int, what: str, *tensors):
    """All on the cache's device (None is no tensor; -1 is host memory)."""
    for t in tensors:
        if t is not None and t.get_device() != index:
            raise ValueError(f"{what} must be on the cache's device")


def _int32(name: str, t: torch.Tensor, dim: int):
    if t.dtype is not torch.int32 or t.dim() != dim:
        raise ValueError(f"{name} must be a {dim}-D int32 tensor")
    if t.stride(-1) != 1 and t.shape[-1] > 1 and t.numel():  # (a single entry is at no distance)
        raise ValueError(f"{name} must be contiguous in its last dimension")


def _head_rows(name: str, t: torch.Tensor, dtype: torch.dtype, heads: Optional[int], dim: int) -> int:
    """Elements between the rows of a [rows, heads, dim] tensor whose heads follow one another."""
    shape = t.shape
    if len(shape) != 3 or shape[2] != dim or (heads is not None and shape[1] != heads):
        raise ValueError(f"{name} must be [rows, {'heads' if heads is None else heads}, {dim}]")
    if t.dtype is not dtype:
        raise ValueError(f"{name} must be of the cache's dtype")
    row, head, value = t.stride()
    if (value != 1 or (head != dim and shape[1] > 1)) and t.numel():
        raise ValueError(f"the heads of {name} must follow one another")
    return row if shape[0] > 1 else shape[1] * dim


class KvCache:
    """A paged cache (msao_kv_cache) over the caller's tensors: k and v [n_pages,
    kv_heads, page_size, head_dim] (float32 or bfloat16; pages, heads and tokens at
    any strides of 16-byte multiples, so a pool that interleaves them is a
    permuted view), pages int32 [n_seqs, pages_per_seq], length int32 [n_seqs],
    weight float32 [n_seqs, kv_heads, >= capacity] or None. The tensors are used in
    place and kept alive; what they hold is read when the kernels run."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, pages: torch.Tensor, length: torch.Tensor,
                 weight: Optional[torch.Tensor] = None):
        if k.dim() != 4 or k.shape != v.shape or k.dtype != v.dtype:
            raise ValueError("k and v must be [n_pages, kv_heads, page_size, head_dim] of one dtype")
        if k.dtype not in (torch.float32, torch.bfloat16):
            raise ValueError("k and v must be float32 or bfloat16")
        if k.numel() and (k.stride(3) != 1 or v.stride(3) != 1):
            raise ValueError("the head_dim values of a token must be contiguous")
        _int32("pages", pages, 2)
        _int32("length", length, 1)
        self.index = k.get_device()
        _same_device(self.index, "v, pages, length and weight", v, pages, length, weight)
        n_seqs = int(length.shape[0])
        if pages.shape[0] != n_seqs:
            raise ValueError("pages and length differ in n_seqs")
        self.k, self.v, self.pages, self.length, self.weight = k, v, pages, length, weight
        self.device, self.dtype, self.n_seqs = k.device, k.dtype, n_seqs  # (a tensor's cuda device has an index)
        self.n_pages, self.kv_heads, self.page_size, self.head_dim = (int(x) for x in k.shape)
        self.pages_per_seq = int(pages.shape[1])
        self.capacity = self.pages_per_seq * self.page_size
        c = self.struct = MsaoKvCache()
        c.k, c.v = (k.data_ptr(), v.data_ptr()) if k.numel() else (None, None)
        for i in range(3):
            # (the only page or head is at no distance, whatever torch says)
            c.k_stride[i], c.v_stride[i] = (k.stride(i), v.stride(i)) if k.shape[i] > 1 else (0, 0)
        c.dtype = F32 if k.dtype == torch.float32 else BF16
        c.head_dim, c.kv_heads, c.page_size, c.n_pages = self.head_dim, self.kv_heads, self.page_size, self.n_pages
        c.n_seqs, c.pages_per_seq = n_seqs, self.pages_per_seq
        c.table_stride = pages.stride(0) if n_seqs > 1 else self.pages_per_seq
        c.pages, c.length = pages.data_ptr(), length.data_ptr()
        if weight is not None:
            if weight.dtype != torch.float32 or weight.dim() != 3 or tuple(weight.shape[:2]) != (n_seqs, self.kv_heads):
                raise ValueError("weight must be float32 [n_seqs, kv_heads, capacity]")
            if weight.shape[2] < self.capacity or not weight.is_contiguous():
                raise ValueError("weight must be contiguous and as long as the capacity")
            c.weight, c.weight_stride = weight.data_ptr(), weight.shape[2]
        self.addr = _addr(c)
        _check(lib().msao_cache_validate(self.addr, None))


def _cache_ctx(cache: KvCache, ctx: Optional[Context], stream) -> Context:
    if cache.index < 0:
        raise ValueError(f"the cache is on {cache.device}, not on a GPU")
    if ctx is None:
        ctx = default_context(cache.index)
    elif ctx.device != cache.index:
        raise ValueError(f"the context is of device {ctx.device}, the cache on {cache.device}")
    if stream is not None and stream.device != cache.device:
        raise ValueError(f"the stream is of {stream.device}, the cache on {cache.device}")
    return ctx


def _stream_of(cache: KvCache, stream) -> int:
    """The handle of `stream`, or of the current stream of the cache's device."""
    return torch._C._cuda_getCurrentRawStream(cache.index) if stream is None else stream.cuda_stream


INT_MAX = 2 ** 31 - 1


def _fits(name: str, value: int) -> int:
    """(ctypes would take the low bits of an integer that its field cannot hold)"""
    if not -INT_MAX <= value <= INT_MAX:
        raise ValueError(f"{name} is out of range")
    return int(value)


def _chunk(cache: KvCache, start: torch.Tensor, n_rows: int, max_new: int) -> MsaoChunk:
    _int32("start", start, 1)
    if start.shape[0] != cache.n_seqs + 1:
        raise ValueError("start must have n_seqs + 1 entries")
    _same_device(cache.index, "start", start)
    return MsaoChunk(start.data_ptr(), _fits("n_rows", n_rows), _fits("max_new", min(max_new, max(n_rows, 0))))


def _scratch(cache: KvCache, nbytes: int, stream) -> torch.Tensor:
    with _on(stream):
        buf = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=cache.device)
        return buf if buf.data_ptr() % 256 == 0 else _workspace(nbytes, cache.device)


def _bytes_of(workspace: torch.Tensor) -> int:
    if not workspace.is_contiguous():  # (its elements may be fewer bytes apart than they have, or none)
        raise ValueError("workspace must be contiguous")
    return workspace.numel() * workspace.element_size()


def _on(stream):
    """Memory allocated inside is `stream`'s, where the call will use it (None: the current stream's)."""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def msao_cache_append(cache: KvCache, start: torch.Tensor, max_new: int, k: torch.Tensor, v: torch.Tensor,
                      q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                      q_norm: Optional[torch.Tensor] = None, k_norm: Optional[torch.Tensor] = None, eps: float = 1e-6,
                      positions: Optional[torch.Tensor] = None, inv_freq: Optional[torch.Tensor] = None,
                      sections: Optional[Sequence[int]] = None, interleaved: bool = False,
                      ctx: Optional[Context] = None, stream=None) -> Optional[torch.Tensor]:
    """The step's keys and values into the cache, queries and keys normed and
    rotated: rows start[s] .. start[s+1]-1 of q [rows, heads, head_dim] and k, v
    [rows, kv_heads, head_dim] are the last tokens of sequence s, counted by
    cache.length already. q_norm and k_norm [head_dim] or None; inv_freq
    float32 [pairs] (None: no rotation) turns the first 2 * pairs values by
    positions int32 [rows] or [axes, rows] (None: the places in the cache),
    sections naming the pairs of each axis; interleaved pairs neighbours. Returns
    q_out (q itself may be passed, or memory that shares none with it)."""
    ctx = _cache_ctx(cache, ctx, stream)
    dim, dtype = cache.head_dim, cache.dtype
    a = MsaoAppend()
    a.k_stride = _head_rows("k", k, dtype, cache.kv_heads, dim)
    a.v_stride = _head_rows("v", v, dtype, cache.kv_heads, dim)
    rows = k.shape[0]
    if v.shape[0] != rows or (q is not None and q.shape[0] != rows):
        raise ValueError("q, k and v differ in rows")
    a.k, a.v, a.eps = k.data_ptr(), v.data_ptr(), eps
    if q is not None:
        a.q_stride = _head_rows("q", q, dtype, None, dim)
        if q_out is None:
            with _on(stream):
                q_out = torch.empty(q.shape, dtype=dtype, device=q.device)
        if q_out.shape != q.shape:
            raise ValueError("q_out must have q's shape")
        a.q_out_stride = _head_rows("q_out", q_out, dtype, None, dim)
        a.q, a.q_out, a.heads = q.data_ptr(), q_out.data_ptr(), q.shape[1]
    elif q_out is not None or q_norm is not None:
        raise ValueError("q_out and q_norm need q")
    for name, w in (("q_norm", q_norm), ("k_norm", k_norm)):
        if w is not None:
            if w.dtype is not dtype or w.shape != (dim,) or not w.is_contiguous():
                raise ValueError(f"{name} must be [head_dim] of the cache's dtype")
            setattr(a, name, w.data_ptr())
    if inv_freq is not None and inv_freq.numel():
        if inv_freq.dtype is not torch.float32 or inv_freq.dim() != 1 or not inv_freq.is_contiguous():
            raise ValueError("inv_freq must be a contiguous 1-D float32 tensor")
        pairs = inv_freq.shape[0]
        a.rot_dim, a.inv_freq, a.n_axes = 2 * pairs, inv_freq.data_ptr(), 1
        if positions is not None:
            dims = positions.dim()
            _int32("positions", positions, 1 if dims == 1 else 2)
            if positions.shape[-1] != rows:
                raise ValueError("positions must be [rows] or [axes, rows]")
            a.n_axes = 1 if dims == 1 else positions.shape[0]
            a.positions = positions.data_ptr()
            a.position_stride = positions.stride(0) if dims == 2 and a.n_axes > 1 else rows
        if sections is None:
            sections = (pairs,)
        if len(sections) != a.n_axes or len(sections) > MAX_AXES:
            raise ValueError("sections must name the pairs of each axis of positions (at most 4)")
        a.sections = tuple(sections)
    elif positions is not None or sections is not None:
        raise ValueError("positions and sections need inv_freq")
    _same_device(cache.index, "every tensor of the step", k, v, q, q_out, q_norm, k_norm, positions, inv_freq)
    if interleaved:
        a.flags = APPEND_NEIGHBOURS
    ch = _chunk(cache, start, rows, max_new)
    _check(lib().msao_cache_append(ctx.handle, cache.addr, ctypes.byref(ch), ctypes.byref(a), _stream_of(cache, stream)),
           ctx)
    return q_out


def cache_attention_workspace(cache: KvCache, start: torch.Tensor, n_rows: int, max_new: int, heads: int,
                              causal: bool = True, accumulate: bool = False) -> int:
    """Bytes of workspace that msao_cache_attention needs for such a call."""
    ch, n = _chunk(cache, start, n_rows, max_new), ctypes.c_size_t()
    flags = (ATTEND_CAUSAL if causal else 0) | (ATTEND_WEIGHT if accumulate else 0)
    _check(lib().msao_cache_attention_workspace(cache.addr, _addr(ch), _fits("heads", heads), flags, ctypes.byref(n)))
    return n.value


def msao_cache_attention(cache: KvCache, start: torch.Tensor, max_new: int, q: torch.Tensor,
                         scale: Optional[float] = None, causal: bool = True, out: Optional[torch.Tensor] = None,
                         lse: Optional[torch.Tensor] = None, accumulate: bool = False,
                         workspace: Optional[torch.Tensor] = None, ctx: Optional[Context] = None,
                         stream=None) -> torch.Tensor:
    """Attention of q [rows, heads, head_dim] (rows of sequences as for
    msao_cache_append) over the cache; scale 1/sqrt(head_dim) when None. lse
    float32 [rows, heads] is filled if given; accumulate adds to cache.weight what
    each token receives. workspace: uint8, 256-byte aligned, of
    cache_attention_workspace bytes (allocated when None). Returns out, which must
    share no memory with q; rows of no sequence, and those from max_new on of a longer
    one, keep what `out` held (0 in one allocated here)."""
    ctx = _cache_ctx(cache, ctx, stream)
    q_stride = _head_rows("q", q, cache.dtype, None, cache.head_dim)
    rows, heads = q.shape[0], q.shape[1]
    if out is None:
        with _on(stream):
            out = torch.zeros(q.shape, dtype=q.dtype, device=q.device)
    elif out.shape != q.shape:
        raise ValueError("out must have q's shape")
    out_stride = _head_rows("out", out, cache.dtype, None, cache.head_dim)
    if lse is not None and (lse.dtype is not torch.float32 or lse.shape != (rows, heads) or not lse.is_contiguous()):
        raise ValueError("lse must be contiguous float32 [rows, heads]")
    _same_device(cache.index, "q, out, lse and workspace", q, out, lse, workspace)
    ch = _chunk(cache, start, rows, max_new)
    flags = (ATTEND_CAUSAL if causal else 0) | (ATTEND_WEIGHT if accumulate else 0)
    if workspace is None:
        need = ctypes.c_size_t()
        _check(lib().msao_cache_attention_workspace(cache.addr, ctypes.byref(ch), heads, flags, ctypes.byref(need)))
        workspace = _scratch(cache, need.value, stream)
    _check(lib().msao_cache_attention(ctx.handle, cache.addr, ctypes.byref(ch), q.data_ptr(), q_stride, heads,
                                      cache.head_dim ** -0.5 if scale is None else scale, flags, out.data_ptr(),
                                      out_stride, None if lse is None else lse.data_ptr(), workspace.data_ptr(),
                                      _bytes_of(workspace), _stream_of(cache, stream)), ctx)
    return out


def msao_cache_evict(cache: KvCache, budget: torch.Tensor, n_first: int = 0, n_recent: int = 0,
                     to: Optional[KvCache] = None, kept_idx: Optional[torch.Tensor] = None,
                     workspace: Optional[torch.Tensor] = None, ctx: Optional[Context] = None,
                     stream=None) -> Dict[str, torch.Tensor]:
    """Each sequence cut to its budget (int32 [n_seqs]) by the accumulated weight,
    per kv head, with the first n_first and the last n_recent tokens kept; into
    `to` or, when None, in place. Lengths (and weight) of the target are updated on
    the device. Returns kept_idx, int32 [n_seqs, kv_heads, capacity]: the kept
    tokens ascending, then -1; and kept_count, the target's lengths."""
    ctx = _cache_ctx(cache, ctx, stream)
    _int32("budget", budget, 1)
    if budget.shape[0] != cache.n_seqs:
        raise ValueError("budget must have n_seqs entries")
    if to is not None and to.index != cache.index:
        raise ValueError("the caches are on different devices")
    if kept_idx is None:
        with _on(stream):
            kept_idx = torch.empty((cache.n_seqs, cache.kv_heads, cache.capacity), dtype=torch.int32,
                                   device=cache.device)
    elif (kept_idx.dtype is not torch.int32 or kept_idx.dim() != 3 or not kept_idx.is_contiguous()
          or kept_idx.shape[:2] != (cache.n_seqs, cache.kv_heads) or kept_idx.shape[2] < cache.capacity):
        raise ValueError("kept_idx must be contiguous int32 [n_seqs, kv_heads, capacity]")
    _same_device(cache.index, "budget, kept_idx and workspace", budget, kept_idx, workspace)
    if workspace is None:
        need = ctypes.c_size_t()
        _check(lib().msao_cache_evict_workspace(cache.addr, ctypes.byref(need)))
        workspace = _scratch(cache, need.value, stream)
    _check(lib().msao_cache_evict(ctx.handle, cache.addr, to.addr if to is not None else None, budget.data_ptr(),
                                  _fits("n_first", min(n_first, INT_MAX)), _fits("n_recent", min(n_recent, INT_MAX)), kept_idx.data_ptr(), kept_idx.shape[2],
                                  workspace.data_ptr(), _bytes_of(workspace), _stream_of(cache, stream)), ctx)
    return {"kept_idx": kept_idx, "kept_count": (to or cache).length}


def sched_default_params() -> MsaoSchedParams:
    return lib().msao_sched_default_params()


def _host_f32(x):
    import numpy as np
    return np.ascontiguousarray(x, dtype=np.float32)


class Scheduler:
    """Algorithm 1 for one request: line 2-3 from calibration entropies, then
    the per-step hold / send / offload loop (host code in libmsao.so)."""

    def __init__(self, calib_h_norm, params: Optional[MsaoSchedParams] = None):
        self.params = params if params is not None else sched_default_params()
        self.state = MsaoSchedState()
        h = _host_f32(calib_h_norm)
        _check(lib().msao_sched_init(h.ctypes.data, h.size, _addr(self.params), _addr(self.state)))

    def step(self, h_norm: float) -> int:
        d = ctypes.c_int32()
        _check(lib().msao_sched_step(_addr(self.state), _addr(self.params), float(h_norm), ctypes.byref(d)))
        return d.value

    def run(self, h_norm):
        import numpy as np
        h = _host_f32(h_norm)
        dec = np.zeros(h.size, np.int8)
        th = np.zeros(h.size, np.float64)
        _check(lib().msao_sched_run(_addr(self.state), _addr(self.params), h.ctypes.data, h.size,
                                    dec.ctypes.data, th.ctypes.data))
        return dec, th


def retention_floor(mas):
    import numpy as np
    m = _host_f32(mas)
    b = np.zeros_like(m)
    _check(lib().msao_retention_floor(m.ctypes.data, m.size, b.ctypes.data))
    return b


def comm_latency(data_bytes: float, bandwidth_bytes_per_s: float, rtt_s: float) -> float:
    return lib().msao_comm_latency(data_bytes, bandwidth_bytes_per_s, rtt_s)


def p_conf(h_norm, theta: float) -> float:
    h = _host_f32(h_norm)
    return lib().msao_p_conf(h.ctypes.data, h.size, theta)


def expected_spec_tokens(p: float) -> float:
    return lib().msao_expected_spec_tokens(p)


def expected_e2e_latency(**terms) -> float:
    m = MsaoLatencyModel(**terms)
    return lib().msao_expected_e2e_latency(_addr(m))


# ---- Sec. 4.1.1 Eq. 3 and Sec. 4.1.3 Eq. 6 with caller weights ----------------

def _learned_args(segments, n_requests, params, heads, mlp, alpha, ctx):
    """Marshalled heads, MLP and logits of a learned call (and what must stay alive)."""
    device = _device_of(segments)
    ctx = ctx or default_context(device.index if device.index is not None else torch.cuda.current_device())
    segt = segment_table(segments)
    prm = params_struct(params)
    n = len(segments)
    keep = [segt, prm]
    harr = None
    if heads is not None:
        harr = (MsaoSpatialHead * max(1, n))()
        for i, h in enumerate(heads):
            if h is None:
                continue
            w = h["weight"]
            keep.append(w)
            harr[i] = MsaoSpatialHead(w.data_ptr(), float(h.get("bias", 0.0)), int(h.get("grid_w", 0)),
                                      int(h.get("pool", 1)))
        keep.append(harr)
    m = None
    if mlp is not None:
        m = MsaoModalMlp(mlp["w1"].data_ptr(), mlp["b1"].data_ptr(), mlp["w2"].data_ptr(), float(mlp.get("b2", 0.0)),
                         int(mlp["b1"].numel()), int(mlp["prompt"].shape[1]) if mlp.get("prompt") is not None else 0,
                         mlp["prompt"].data_ptr() if mlp.get("prompt") is not None else None)
        keep.append(m)
    al = None
    if alpha is not None:
        vals = list(alpha)
        al = (ctypes.c_float * len(vals))(*vals)
        keep.append(al)
    return device, ctx, segt, prm, harr, m, al, keep


def _learned_extra(o, n_requests, device):
    R = n_requests
    return {"importance": torch.empty(max(o.ntok, 1), dtype=torch.float32, device=device)[:o.ntok],
            "alpha": torch.empty(R * NMOD, dtype=torch.float32, device=device),
            "desc": torch.empty(R * NMOD * MODAL_DESC, dtype=torch.float32, device=device)}


def msao_mas_score_learned(segments, n_requests, params=None, heads=None, mlp=None, alpha=None, ctx=None,
                           outputs=None, stream=None):
    """msao_mas_score with learned probe heads: heads[s] is None or a dict
    (weight=[hidden] device tensor in the segment's dtype, bias, grid_w, pool);
    mlp is None or a dict of device float32 tensors (w1 [hidden, prompt_dim +
    8], b1, w2, prompt [n_requests, prompt_dim]) and b2. Returns
    (outputs, extra) with extra = importance, alpha and desc device tensors."""
    device, ctx, segt, prm, harr, m, al, keep = _learned_args(segments, n_requests, params, heads, mlp, alpha, ctx)
    o = outputs or Outputs(segments, n_requests, compact=False)
    n, R = len(segments), n_requests
    extra = _learned_extra(o, R, device)
    st = _stream_ptr(stream, device)
    _check(lib().msao_mas_score_learned(ctx.handle, segt, n, R, _addr(prm),
                                        ctypes.cast(harr, _P) if harr is not None else None,
                                        _addr(m) if m is not None else None, al, _addr(o.c_tok),
                                        _ptr(extra["importance"]) if o.ntok else None, _addr(o.c_frm),
                                        _addr(o.c_req), _ptr(extra["alpha"]), _ptr(extra["desc"]),
                                        _ptr(o.workspace), ctypes.c_size_t(o.ws_bytes), st),
           ctx)
    extra["_keep"] = keep
    return o, extra


def prepare_learned(segments, n_requests, outputs, params=None, heads=None, mlp=None, alpha=None, ctx=None,
                    compact=True):
    """msao_run_learned's arguments marshalled once (as prepare() does for the
    other entry points): returns (call, extra); each call(stream) enqueues one
    run on the same outputs and extra buffers (tables still uploaded per call)."""
    device, ctx, segt, prm, harr, m, al, keep = _learned_args(segments, n_requests, params, heads, mlp, alpha, ctx)
    o = outputs
    n, R = len(segments), n_requests
    extra = _learned_extra(o, R, device)
    use_out = compact and o.out is not None
    args = [ctx.handle, segt, n, R, _addr(prm), ctypes.cast(harr, _P) if harr is not None else None,
            _addr(m) if m is not None else None, al, _addr(o.c_tok),
            _ptr(extra["importance"]) if o.ntok else None, _addr(o.c_frm), _addr(o.c_req),
            _ptr(extra["alpha"]), _ptr(extra["desc"]), _addr(o.c_sel),
            _ptr(o.out) if use_out else None, o.out_off if use_out else None,
            ctypes.c_int64(o.out_bytes if use_out else 0), _ptr(o.workspace), ctypes.c_size_t(o.ws_bytes), None]
    return Call("msao_run_learned", args, ctx, keep + [o, extra]), extra


def msao_run_learned(segments, n_requests, params=None, heads=None, mlp=None, alpha=None, ctx=None, outputs=None,
                     stream=None, compact=True):
    """msao_mas_score_learned plus the selection and compaction of msao_run,
    with segments that have a head ranked by their Eq. 3 importance (heads
    and mlp as for msao_mas_score_learned). Returns (outputs, extra)."""
    device, ctx, segt, prm, harr, m, al, keep = _learned_args(segments, n_requests, params, heads, mlp, alpha, ctx)
    o = outputs or Outputs(segments, n_requests, compact=compact)
    n, R = len(segments), n_requests
    extra = _learned_extra(o, R, device)
    use_out = compact and o.out is not None
    st = _stream_ptr(stream, device)
    _check(lib().msao_run_learned(ctx.handle, segt, n, R, _addr(prm),
                                  ctypes.cast(harr, _P) if harr is not None else None,
                                  _addr(m) if m is not None else None, al, _addr(o.c_tok),
                                  _ptr(extra["importance"]) if o.ntok else None, _addr(o.c_frm), _addr(o.c_req),
                                  _ptr(extra["alpha"]), _ptr(extra["desc"]), _addr(o.c_sel),
                                  _ptr(o.out) if use_out else None, o.out_off if use_out else None,
                                  ctypes.c_int64(o.out_bytes if use_out else 0), _ptr(o.workspace),
                                  ctypes.c_size_t(o.ws_bytes), st), ctx)
    extra["_keep"] = keep
    return o, extra
