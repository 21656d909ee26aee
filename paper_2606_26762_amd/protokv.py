"""Thin ctypes binding of libprotokv (argument marshalling only).

Every step of the hot path runs in the HIP library; this module converts
Python/torch arguments into the C-ABI's pointers and sizes, and raises
``ProtoKVError`` on a non-OK status.  Loading fails loudly if the library has
not been built (``python -m paper_2606_26762_amd.build``).
"""
from __future__ import annotations

import ctypes
import os
from typing import Dict, Optional, Sequence

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libprotokv.so")

ROW_BYTES = 3200
KV_BF16, KV_FP32 = 0, 1
FLAG_PQ, FLAG_MASS_BIAS, FLAG_MAINTENANCE, FLAG_EMA_CENTRES, FLAG_MAH_SQUARED, FLAG_VAR_ALLOC = 1, 2, 4, 8, 16, 32

STATUS = {0: "OK", 1: "E_INVALID", 2: "E_UNSUPPORTED", 3: "E_WORKSPACE", 4: "E_STATE", 5: "E_DEVICE"}

EXPORTED = [
    "protokv_default_config", "protokv_validate_config", "protokv_workspace_size", "protokv_init",
    "protokv_destroy", "protokv_append_frame", "protokv_fold", "protokv_synthesize", "protokv_attend",
    "protokv_stream_info_get", "protokv_get_counters", "protokv_read_assignments", "protokv_read_bank",
    "protokv_read_pseudo", "protokv_read_codebooks", "protokv_profile", "protokv_profile_read",
    "protokv_state_size", "protokv_get_state", "protokv_set_state", "protokv_attend_static",
    "protokv_read_pseudo_counts",
    "protokv_page_plan", "protokv_rotate", "protokv_prompt_attend", "protokv_page_attend",
    "protokv_page_attend_workspace",
    "protokv_norm_rotate", "protokv_page4_store", "protokv_page4_read", "protokv_page4_attend",
    "protokv_page4_attend_workspace", "protokv_page_fork", "protokv_page_copy", "protokv_page_release",
    "protokv_last_error",
]

STATE_MAGIC, STATE_VERSION = 0x53564B50, 1
MAX_EVICTED_TOKENS = 16777214
STATIC_SCRATCH_BYTES = 64 << 20

KERNELS = ["ring_insert", "seed", "screen", "aggregate", "decode", "attend", "attend_merge", "pq_encode",
           "materialize", "maintain", "rope_ring", "rope_q", "warm_collect", "warm_kmeans", "alloc"]


class ProtoKVError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS.get(status, status)}: {msg}")
        self.status = status


class Config(ctypes.Structure):
    _fields_ = [
        ("num_streams", ctypes.c_int32), ("num_layers", ctypes.c_int32),
        ("num_kv_heads", ctypes.c_int32), ("num_q_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("grid_h", ctypes.c_int32), ("grid_w", ctypes.c_int32),
        ("window_frames", ctypes.c_int32), ("capacity", ctypes.c_int32),
        ("pseudo_per_proto", ctypes.c_int32), ("pq_subspaces", ctypes.c_int32),
        ("pq_codewords", ctypes.c_int32), ("beam", ctypes.c_int32), ("t_idle", ctypes.c_int32),
        ("max_query_tokens", ctypes.c_int32), ("kv_dtype", ctypes.c_int32),
        ("flags", ctypes.c_uint32), ("eta", ctypes.c_float), ("pq_eps", ctypes.c_float),
        ("lambda_sp", ctypes.c_double), ("lambda_idle", ctypes.c_double), ("ridge", ctypes.c_double),
        ("gamma", ctypes.c_double), ("eps_k", ctypes.c_double), ("eps_v", ctypes.c_double),
        ("alpha", ctypes.c_float), ("beta", ctypes.c_float), ("rope_theta", ctypes.c_double),
        ("warm_frames", ctypes.c_int32), ("warm_tokens", ctypes.c_int32),
        ("kmeans_epochs", ctypes.c_int32), ("kmeans_batch", ctypes.c_int32), ("pseudo_max", ctypes.c_int32),
    ]


class StreamInfo(ctypes.Structure):
    _fields_ = [("frames", ctypes.c_uint64), ("evicted_tokens", ctypes.c_uint64),
                ("active_slots", ctypes.c_int32), ("pending", ctypes.c_int32)]


class Counters(ctypes.Structure):
    _fields_ = [("folds", ctypes.c_uint64), ("tokens_assigned", ctypes.c_uint64),
                ("tokens_seeded", ctypes.c_uint64), ("refined", ctypes.c_uint64),
                ("refined_full", ctypes.c_uint64), ("near_ties", ctypes.c_uint64),
                ("touched", ctypes.c_uint64), ("aged", ctypes.c_uint64), ("merged", ctypes.c_uint64),
                ("recycled", ctypes.c_uint64)]


class StateHeader(ctypes.Structure):
    _fields_ = [("magic", ctypes.c_uint32), ("version", ctypes.c_uint32), ("units", ctypes.c_uint32),
                ("capacity", ctypes.c_uint32), ("tokens_per_frame", ctypes.c_uint32),
                ("window_frames", ctypes.c_uint32), ("kv_bytes", ctypes.c_uint32),
                ("codewords", ctypes.c_uint32), ("warm_tokens", ctypes.c_uint32), ("rotated", ctypes.c_uint32),
                ("frames", ctypes.c_uint64), ("evicted_tokens", ctypes.c_uint64),
                ("active_slots", ctypes.c_int32), ("folds", ctypes.c_int32),
                ("reservoir_rows", ctypes.c_int32), ("pad", ctypes.c_int32),
                ("off_ring_k", ctypes.c_uint64), ("off_ring_v", ctypes.c_uint64), ("off_bank", ctypes.c_uint64),
                ("off_codebooks", ctypes.c_uint64), ("off_reservoir", ctypes.c_uint64),
                ("off_ring_kr", ctypes.c_uint64), ("total_bytes", ctypes.c_uint64)]


class KernelTimes(ctypes.Structure):
    _fields_ = [("ms", ctypes.c_double * 16), ("launches", ctypes.c_uint64 * 16)]


class Pages(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("num_pages", ctypes.c_int32), ("page_size", ctypes.c_int32)]


class PagePlanArgs(ctypes.Structure):
    _fields_ = [("num_requests", ctypes.c_int32), ("num_pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("table_stride", ctypes.c_int32), ("max_tokens", ctypes.c_int32)] + [
        (f, ctypes.c_void_p) for f in ("ctx", "add", "base", "table", "free_pages", "free_count", "free_count_out",
                                       "cu", "kv_len", "slots", "positions", "refused")]


class RotateArgs(ctypes.Structure):
    _fields_ = [("num_tokens", ctypes.c_int32), ("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("kv_dtype", ctypes.c_int32), ("num_axes", ctypes.c_int32),
                ("positions", ctypes.c_void_p), ("position_stride", ctypes.c_int64), ("axes", ctypes.c_char_p),
                ("theta", ctypes.c_double), ("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("q_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64),
                ("q_out", ctypes.c_void_p), ("k_out", ctypes.c_void_p),
                ("q_out_stride", ctypes.c_int64), ("k_out_stride", ctypes.c_int64),
                ("pages", ctypes.POINTER(Pages)), ("slots", ctypes.c_void_p)]


class PromptArgs(ctypes.Structure):
    _fields_ = [("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("kv_dtype", ctypes.c_int32), ("num_seqs", ctypes.c_int32), ("total", ctypes.c_int32),
                ("cu", ctypes.c_void_p), ("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("q_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64),
                ("o", ctypes.c_void_p), ("lse", ctypes.c_void_p),
                ("prior_o", ctypes.c_void_p), ("prior_lse", ctypes.c_void_p)]


class PageAttendArgs(ctypes.Structure):
    _fields_ = [("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("kv_dtype", ctypes.c_int32), ("num_requests", ctypes.c_int32), ("total", ctypes.c_int32),
                ("max_add", ctypes.c_int32), ("table_stride", ctypes.c_int32),
                ("cu", ctypes.c_void_p), ("kv_len", ctypes.c_void_p), ("table", ctypes.c_void_p),
                ("q", ctypes.c_void_p), ("q_stride", ctypes.c_int64), ("pages", Pages),
                ("o", ctypes.c_void_p), ("lse", ctypes.c_void_p),
                ("prior_o", ctypes.c_void_p), ("prior_lse", ctypes.c_void_p),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


class HeadNorm(ctypes.Structure):
    _fields_ = [("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("eps", ctypes.c_double)]


class Pages4(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("num_pages", ctypes.c_int32), ("page_size", ctypes.c_int32)]


class Page4RowsArgs(ctypes.Structure):
    _fields_ = [("num_tokens", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("kv_dtype", ctypes.c_int32), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64), ("slots", ctypes.c_void_p), ("pages", Pages4)]


class Page4AttendArgs(ctypes.Structure):
    _fields_ = [(f, Pages4 if f == "pages" else t) for f, t in PageAttendArgs._fields_]


class PageForkArgs(ctypes.Structure):
    _fields_ = [("num_forks", ctypes.c_int32), ("num_requests", ctypes.c_int32), ("num_pages", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("table_stride", ctypes.c_int32)] + [
        (f, ctypes.c_void_p) for f in ("ctx", "src", "dst", "at", "table", "shares", "free_pages", "free_count",
                                       "free_count_out", "ctx_out", "lens", "copy_src", "copy_dst", "copy_rows", "refused")]


class PageArray(ctypes.Structure):
    _fields_ = [("base", ctypes.c_void_p), ("row_bytes", ctypes.c_int32), ("layers", ctypes.c_int32),
                ("layer_stride", ctypes.c_int64)]


class PageCopyArgs(ctypes.Structure):
    _fields_ = [("num_copies", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32), ("num_pages", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("num_arrays", ctypes.c_int32), ("arrays", ctypes.POINTER(PageArray)),
                ("src", ctypes.c_void_p), ("dst", ctypes.c_void_p), ("rows", ctypes.c_void_p)]


class PageReleaseArgs(ctypes.Structure):
    _fields_ = [("num_requests", ctypes.c_int32), ("num_pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("table_stride", ctypes.c_int32)] + [
        (f, ctypes.c_void_p) for f in ("ctx", "keep", "table", "shares", "free_pages", "free_count", "free_count_out",
                                       "ctx_out", "refused", "scratch")]


RELEASE_PAGES = 4096   # pages to an entry of page_release's scratch

_lib = None


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built: run `python -m paper_2606_26762_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
        P = ctypes.POINTER
        L.protokv_default_config.argtypes = [P(Config)]
        L.protokv_validate_config.argtypes = [P(Config)]
        L.protokv_workspace_size.argtypes = [P(Config), P(sz)]
        L.protokv_init.argtypes = [P(Config), vp, vp, sz, vp, P(vp)]
        L.protokv_destroy.argtypes = [vp]
        L.protokv_append_frame.argtypes = [vp, P(i32), i32, vp, vp, vp]
        L.protokv_fold.argtypes = [vp, vp]
        L.protokv_synthesize.argtypes = [vp, i32, vp]
        L.protokv_attend.argtypes = [vp, i32, vp, i32, vp, vp, vp]
        L.protokv_attend_static.argtypes = [vp, i32, vp, i32, vp, vp, vp]
        L.protokv_stream_info_get.argtypes = [vp, i32, P(StreamInfo)]
        L.protokv_get_counters.argtypes = [vp, P(Counters), vp]
        L.protokv_read_assignments.argtypes = [vp, i32, vp, sz, vp]
        L.protokv_read_bank.argtypes = [vp, i32, vp, sz, vp]
        L.protokv_read_pseudo.argtypes = [vp, vp, vp, vp, vp]
        L.protokv_read_codebooks.argtypes = [vp, i32, vp, sz, vp]
        L.protokv_read_pseudo_counts.argtypes = [vp, vp, sz, vp]
        L.protokv_profile.argtypes = [vp, ctypes.c_uint32]
        L.protokv_profile_read.argtypes = [vp, P(KernelTimes)]
        L.protokv_state_size.argtypes = [vp, P(sz)]
        L.protokv_get_state.argtypes = [vp, i32, vp, sz, vp]
        L.protokv_set_state.argtypes = [vp, i32, vp, sz, vp]
        L.protokv_page_plan.argtypes = [P(PagePlanArgs), vp]
        L.protokv_rotate.argtypes = [P(RotateArgs), vp]
        L.protokv_prompt_attend.argtypes = [P(PromptArgs), vp]
        L.protokv_page_attend.argtypes = [P(PageAttendArgs), vp]
        L.protokv_page_attend_workspace.argtypes = [P(PageAttendArgs), P(sz)]
        L.protokv_norm_rotate.argtypes = [P(RotateArgs), P(HeadNorm), vp]
        L.protokv_page4_store.argtypes = [P(Page4RowsArgs), vp]
        L.protokv_page4_read.argtypes = [P(Page4RowsArgs), vp]
        L.protokv_page4_attend.argtypes = [P(Page4AttendArgs), vp]
        L.protokv_page4_attend_workspace.argtypes = [P(Page4AttendArgs), P(sz)]
        L.protokv_page_fork.argtypes = [P(PageForkArgs), vp]
        L.protokv_page_copy.argtypes = [P(PageCopyArgs), vp]
        L.protokv_page_release.argtypes = [P(PageReleaseArgs), vp]
        L.protokv_last_error.argtypes = [vp]
        L.protokv_last_error.restype = ctypes.c_char_p
        for name in EXPORTED:
            if name != "protokv_last_error":
                getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def _check(status: int, handle=None):
    if status != 0:
        msg = lib().protokv_last_error(handle)
        raise ProtoKVError(status, msg.decode() if msg else "")


def default_config(**overrides) -> Config:
    cfg = Config()
    _check(lib().protokv_default_config(ctypes.byref(cfg)))
    for k, v in overrides.items():
        if not hasattr(cfg, k):
            raise AttributeError(k)
        setattr(cfg, k, v)
    return cfg


def workspace_size(cfg: Config) -> int:
    n = ctypes.c_size_t()
    _check(lib().protokv_workspace_size(ctypes.byref(cfg), ctypes.byref(n)))
    return n.value


def _stream_ptr(stream) -> Optional[int]:
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream


def decode_bank(raw: np.ndarray, units: int, capacity: int) -> Dict[str, np.ndarray]:
    """Views of the documented bank row layout (uint8 [units*capacity*3200])."""
    rows = raw.reshape(units, capacity, ROW_BYTES)
    f32 = lambda a, b: rows[:, :, a:b].copy().view(np.float32)
    u32 = lambda a, b: rows[:, :, a:b].copy().view(np.uint32)
    meta = rows[:, :, 3072:3104].copy()
    return {
        "sum_k": f32(0, 512), "sum_v": f32(512, 1024), "sq_k": f32(1024, 1536), "sq_v": f32(1536, 2048),
        "hist_k": u32(2048, 2560).reshape(units, capacity, 8, 16),
        "hist_v": u32(2560, 3072).reshape(units, capacity, 8, 16),
        "n": meta[:, :, 0:4].view(np.uint32)[..., 0], "n_res": meta[:, :, 4:8].view(np.uint32)[..., 0],
        "mu": meta[:, :, 8:16].view(np.float32), "sigma": meta[:, :, 16:28].view(np.float32),
        "tau": meta[:, :, 28:32].view(np.int32)[..., 0],
    }


def encode_bank(bank: Dict[str, np.ndarray], units: int, capacity: int) -> np.ndarray:
    """The documented bank row layout (uint8 [units*capacity*3200]) from arrays
    shaped as decode_bank returns them (histograms [units][K][G][C], C <= 16)."""
    rows = np.zeros((units, capacity, ROW_BYTES), dtype=np.uint8)

    def put(a, b, arr, dt):
        rows[:, :, a:b] = np.ascontiguousarray(np.asarray(arr, dtype=dt).reshape(units, capacity, -1)).view(np.uint8)
    put(0, 512, bank["sum_k"], np.float32)
    put(512, 1024, bank["sum_v"], np.float32)
    put(1024, 1536, bank["sq_k"], np.float32)
    put(1536, 2048, bank["sq_v"], np.float32)
    for name, a in (("hist_k", 2048), ("hist_v", 2560)):
        h = np.zeros((units, capacity, 8, 16), dtype=np.uint32)
        src = np.asarray(bank[name])
        h[..., :src.shape[-1]] = src
        put(a, a + 512, h, np.uint32)
    put(3072, 3076, bank["n"], np.uint32)
    put(3076, 3080, bank["n_res"], np.uint32)
    put(3080, 3088, bank["mu"], np.float32)
    put(3088, 3100, bank["sigma"], np.float32)
    put(3100, 3104, bank["tau"], np.int32)
    return rows.reshape(-1)


class State:
    """One stream's state blob (protokv.h) with views of its sections."""

    def __init__(self, blob: np.ndarray, kv_dtype: str):
        self.blob = blob
        self.header = StateHeader.from_buffer_copy(blob[:ctypes.sizeof(StateHeader)].tobytes())
        h = self.header
        if h.magic != STATE_MAGIC:
            raise ValueError("not a protokv state blob")
        self.kv_dtype = kv_dtype
        T, W, U = h.tokens_per_frame, h.window_frames, h.units
        ring = U * (W + 1) * T * 128 * h.kv_bytes
        self._ring_shape = (U, W + 1, T, 128)
        self._ring_bytes = ring

    def _section(self, off, nbytes):
        return self.blob[off:off + nbytes]

    def ring(self, which: str = "k") -> np.ndarray:
        """The ring as float32 [units][W+1][T][D] (a copy)."""
        off = {"k": self.header.off_ring_k, "v": self.header.off_ring_v, "kr": self.header.off_ring_kr}[which]
        raw = self._section(off, self._ring_bytes)
        if self.header.kv_bytes == 4:
            return raw.view(np.float32).reshape(self._ring_shape).copy()
        return (raw.view(np.uint16).astype(np.uint32) << 16).view(np.float32).reshape(self._ring_shape)

    def bank(self) -> Dict[str, np.ndarray]:
        h = self.header
        return decode_bank(self._section(h.off_bank, h.units * h.capacity * ROW_BYTES), h.units, h.capacity)

    def set_bank_rows(self, unit: int, rows: np.ndarray):
        """Replace the rows of one unit (uint8 [capacity * 3200])."""
        h = self.header
        n = h.capacity * ROW_BYTES
        self.blob[h.off_bank + unit * n:h.off_bank + (unit + 1) * n] = rows

    def set_active_slots(self, n: int):
        self.header.active_slots = n
        self.blob[:ctypes.sizeof(StateHeader)] = np.frombuffer(bytes(self.header), dtype=np.uint8)

    def codebooks(self) -> np.ndarray:
        h = self.header
        n = h.units * 2 * 8 * h.codewords * 16
        return self._section(h.off_codebooks, n * 4).view(np.float32).reshape(h.units, 2, 8, h.codewords, 16)


class ProtoKV:
    """One libprotokv handle with its workspace held as a torch uint8 tensor."""

    def __init__(self, cfg: Config, codebooks: np.ndarray, device="cuda", stream=None):
        import torch
        self.torch = torch
        self.cfg = cfg
        self.units = cfg.num_layers * cfg.num_kv_heads
        self.T = cfg.grid_h * cfg.grid_w
        self.kv_dtype = torch.float32 if cfg.kv_dtype == KV_FP32 else torch.bfloat16
        cb = np.ascontiguousarray(codebooks, dtype=np.float32)
        expect = (cfg.num_streams * self.units * 2 * cfg.pq_subspaces * cfg.pq_codewords
                  * (cfg.head_dim // cfg.pq_subspaces))
        if cb.size != expect:
            raise ValueError(f"codebooks: expected {expect} floats, got {cb.size}")
        self.workspace = torch.empty(workspace_size(cfg), dtype=torch.uint8, device=device)
        h = ctypes.c_void_p()
        _check(lib().protokv_init(ctypes.byref(cfg), cb.ctypes.data, self.workspace.data_ptr(),
                                  self.workspace.numel(), _stream_ptr(stream), ctypes.byref(h)))
        self.h = h

    def close(self):
        if getattr(self, "h", None) is not None and self.h.value:
            lib().protokv_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- hot path --------------------------------------------------------
    def append_frame(self, stream_ids: Sequence[int], k, v, stream=None):
        ids = (ctypes.c_int32 * len(stream_ids))(*stream_ids)
        self._check_tensor(k, (len(stream_ids), self.cfg.num_layers, self.cfg.num_kv_heads, self.T,
                               self.cfg.head_dim))
        self._check_tensor(v, tuple(k.shape))
        _check(lib().protokv_append_frame(self.h, ids, len(stream_ids), k.data_ptr(), v.data_ptr(),
                                          _stream_ptr(stream)), self.h)

    def fold(self, stream=None):
        _check(lib().protokv_fold(self.h, _stream_ptr(stream)), self.h)

    def synthesize(self, stream_id: int, stream=None):
        _check(lib().protokv_synthesize(self.h, stream_id, _stream_ptr(stream)), self.h)

    def attend(self, stream_id: int, q, out=None, lse=None, stream=None):
        torch = self.torch
        tq = q.shape[1]
        self._check_tensor(q, (self.cfg.num_layers, tq, self.cfg.num_q_heads, self.cfg.head_dim))
        if out is None:
            out = torch.empty_like(q)
        if lse is None:
            lse = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device)
        _check(lib().protokv_attend(self.h, stream_id, q.data_ptr(), tq, out.data_ptr(),
                                    lse.data_ptr() if lse is not False else None,
                                    _stream_ptr(stream)), self.h)
        return out, lse

    def attend_static(self, stream_id: int, q, out=None, lse=None, stream=None):
        """protokv_attend_static: the readout with its scratch in the library's
        fixed device array (no allocation by the library)."""
        torch = self.torch
        tq = q.shape[1]
        self._check_tensor(q, (self.cfg.num_layers, tq, self.cfg.num_q_heads, self.cfg.head_dim))
        if out is None:
            out = torch.empty_like(q)
        if lse is None:
            lse = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device)
        _check(lib().protokv_attend_static(self.h, stream_id, q.data_ptr(), tq, out.data_ptr(),
                                           lse.data_ptr() if lse is not False else None,
                                           _stream_ptr(stream)), self.h)
        return out, lse

    # -- introspection -----------------------------------------------------
    def stream_info(self, stream_id: int) -> StreamInfo:
        info = StreamInfo()
        _check(lib().protokv_stream_info_get(self.h, stream_id, ctypes.byref(info)), self.h)
        return info

    def counters(self, stream=None) -> Counters:
        c = Counters()
        _check(lib().protokv_get_counters(self.h, ctypes.byref(c), _stream_ptr(stream)), self.h)
        return c

    def read_assignments(self, stream_id: int, stream=None) -> np.ndarray:
        out = np.zeros((self.units, self.T), dtype=np.int32)
        _check(lib().protokv_read_assignments(self.h, stream_id, out.ctypes.data, out.size,
                                              _stream_ptr(stream)), self.h)
        return out

    def read_bank(self, stream_id: int, stream=None) -> Dict[str, np.ndarray]:
        raw = np.zeros(self.units * self.cfg.capacity * ROW_BYTES, dtype=np.uint8)
        _check(lib().protokv_read_bank(self.h, stream_id, raw.ctypes.data, raw.size,
                                       _stream_ptr(stream)), self.h)
        return decode_bank(raw, self.units, self.cfg.capacity)

    def read_codebooks(self, stream_id: int, stream=None) -> np.ndarray:
        """-> float32 [units][2][G][C][D/G]: the stream's PQ codebooks (given, or learned by the warm-up)."""
        c = self.cfg
        out = np.zeros((self.units, 2, c.pq_subspaces, c.pq_codewords, c.head_dim // c.pq_subspaces),
                       dtype=np.float32)
        _check(lib().protokv_read_codebooks(self.h, stream_id, out.ctypes.data, out.size, _stream_ptr(stream)),
               self.h)
        return out

    def read_pseudo(self, stream=None):
        """-> keys, values float32 [units][K*S][D] and bias [units][K]."""
        n = self.units * self.cfg.capacity * self.cfg.pseudo_per_proto * self.cfg.head_dim
        bits = 32 if self.cfg.kv_dtype == KV_FP32 else 16
        raw_k = np.zeros(n, dtype=np.uint32 if bits == 32 else np.uint16)
        raw_v = np.zeros_like(raw_k)
        bias = np.zeros(self.units * self.cfg.capacity, dtype=np.float32)
        _check(lib().protokv_read_pseudo(self.h, raw_k.ctypes.data, raw_v.ctypes.data, bias.ctypes.data,
                                         _stream_ptr(stream)), self.h)
        conv = (lambda r: r.view(np.float32)) if bits == 32 else \
            (lambda r: (r.astype(np.uint32) << 16).view(np.float32))
        shape = (self.units, self.cfg.capacity * self.cfg.pseudo_per_proto, self.cfg.head_dim)
        return conv(raw_k).reshape(shape), conv(raw_v).reshape(shape), bias.reshape(self.units, -1)

    def state_size(self) -> int:
        n = ctypes.c_size_t()
        _check(lib().protokv_state_size(self.h, ctypes.byref(n)), self.h)
        return n.value

    def get_state(self, stream_id: int, stream=None) -> State:
        blob = np.zeros(self.state_size(), dtype=np.uint8)
        _check(lib().protokv_get_state(self.h, stream_id, blob.ctypes.data, blob.size, _stream_ptr(stream)), self.h)
        return State(blob, "fp32" if self.cfg.kv_dtype == KV_FP32 else "bf16")

    def set_state(self, stream_id: int, state, stream=None):
        blob = np.ascontiguousarray(state.blob if isinstance(state, State) else state, dtype=np.uint8)
        _check(lib().protokv_set_state(self.h, stream_id, blob.ctypes.data, blob.size, _stream_ptr(stream)), self.h)

    def read_pseudo_counts(self, stream=None) -> np.ndarray:
        """-> int32 [units][K]: pseudo-tokens per slot of the current synthesis."""
        out = np.zeros((self.units, self.cfg.capacity), dtype=np.int32)
        _check(lib().protokv_read_pseudo_counts(self.h, out.ctypes.data, out.size, _stream_ptr(stream)), self.h)
        return out

    def profile(self, enable, kernels=None):
        """Time every launch (enable=True), only the named kernels, or stop (False)."""
        mask = 0
        if enable:
            mask = 0xFFFFFFFF if kernels is None else sum(1 << KERNELS.index(k) for k in kernels)
        _check(lib().protokv_profile(self.h, mask), self.h)

    def profile_read(self) -> Dict[str, dict]:
        """-> {kernel: {"ms": total, "launches": n, "avg_us": mean}} for timed kernels."""
        kt = KernelTimes()
        _check(lib().protokv_profile_read(self.h, ctypes.byref(kt)), self.h)
        out = {}
        for i, name in enumerate(KERNELS):
            n = int(kt.launches[i])
            if n:
                out[name] = {"ms": kt.ms[i], "launches": n, "avg_us": 1000.0 * kt.ms[i] / n}
        return out

    def _check_tensor(self, t, shape):
        if tuple(t.shape) != tuple(shape):
            raise ValueError(f"expected shape {tuple(shape)}, got {tuple(t.shape)}")
        if t.dtype != self.kv_dtype or not t.is_cuda or not t.is_contiguous():
            raise ValueError(f"expected a contiguous {self.kv_dtype} CUDA tensor")


# -- exact attention around the readout (no handle) ---------------------------
# One token's call takes a few microseconds on the GPU, so what these do in Python
# counts: each tensor is looked at once.  Results carry no gradient: tensors that ask
# for one are refused while gradients are on.


def _device(t, stream) -> int:
    """The current device, which a call's tensors and its stream must be on."""
    import torch
    d = t.get_device()
    if d < 0:
        raise ValueError("expected CUDA tensors")
    if d != torch.cuda.current_device() or (stream is not None and stream.device_index != d):
        raise ValueError(f"the tensors are on cuda:{d}; they and the stream must be on the current device")
    return d


def _raw_stream(stream, dev: int) -> int:
    import torch
    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream


def _kv(dtype) -> int:
    import torch
    if dtype == torch.bfloat16:
        return KV_BF16
    if dtype == torch.float32:
        return KV_FP32
    raise ValueError(f"expected bfloat16 or float32, got {dtype}")


def _no_gradient(name):
    import torch
    if torch.is_grad_enabled():
        raise ValueError(f"{name}: requires a gradient, which these calls do not give (detach it, or call under "
                         "torch.no_grad())")


def _rows(t, name, dtype=None, dev=None):
    """-> (pointer, row stride in elements) of token rows [N][heads][D]."""
    shape = t.shape
    if len(shape) != 3 or shape[2] != 128 or (dtype is not None and t.dtype != dtype) or (
            dev is not None and t.get_device() != dev):
        raise ValueError(f"{name}: expected rows [N, heads, 128] in {dtype} on the current device, got "
                         f"{t.dtype} {tuple(shape)} on {t.device}")
    if t.requires_grad:
        _no_gradient(name)
    s0, s1, s2 = t.stride()
    if shape[0] > 0 and (s2 != 1 or (shape[1] > 1 and s1 != 128)):
        raise ValueError(f"{name}: the heads of a row must be contiguous")
    return t.data_ptr(), s0 if shape[0] > 1 else shape[1] * 128


def _flat(t, name, dtype, dev, *shape) -> int:
    """Pointer of a contiguous tensor of that type and shape."""
    if t.shape != shape or t.dtype != dtype or t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous {dtype} tensor {shape} on the current device, got "
                         f"{t.dtype} {tuple(t.shape)} on {t.device}")
    if t.requires_grad:
        _no_gradient(name)
    return t.data_ptr()


def _pages(pages, dtype, dev, kv_heads) -> Pages:
    """Pages of (k, v) [num_pages][kv heads][page size][D]."""
    k, v = pages
    shape = k.shape
    if len(shape) != 4 or shape[1] != kv_heads or shape[3] != 128:
        raise ValueError(f"pages: expected k and v [num_pages, {kv_heads}, page_size, 128]")
    return Pages(_flat(k, "pages", dtype, dev, *shape), _flat(v, "pages", dtype, dev, *shape), shape[0], shape[2])


def _new(shape, dtype, like, stream):
    """A tensor on like's device for a call on `stream`: allocated there, so that its
    memory is not reused before that stream's work is done.  (new_empty takes 1.5 us,
    torch.empty with a device 1.8.)"""
    import torch
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


def _result(a, q, out, lse, prior, dev, stream):
    """Outputs [N][Hq][D] and [N][Hq] (made where not given; lse=False: none) and the prior into a."""
    import torch
    n, hq, _ = q.shape
    if out is None:
        out = torch.empty_like(q) if stream is None and q.is_contiguous() else _new((n, hq, 128), q.dtype, q, stream)
        a.o = out.data_ptr()
    else:
        a.o = _flat(out, "out", q.dtype, dev, n, hq, 128)
    if lse is None:
        lse = _new((n, hq), torch.float32, q, stream)
        a.lse = lse.data_ptr()
    elif lse is not False:
        a.lse = _flat(lse, "lse", torch.float32, dev, n, hq)
    if prior is not None:
        a.prior_o = _flat(prior[0], "prior", q.dtype, dev, n, hq, 128)
        a.prior_lse = _flat(prior[1], "prior lse", torch.float32, dev, n, hq)
    return out, lse


def pair_axes(sections: Sequence[int], interleaved: bool = False) -> bytes:
    """Axis of each of the 64 rotary pairs, for ``rotate``: sections[a] pairs turn
    by axis a, in one run after the other, or (interleaved) dealt out in turn,
    an axis leaving the round once it has all of its pairs."""
    left = [int(n) for n in sections]
    if not 1 <= len(left) <= 8 or min(left) < 0 or sum(left) != 64:
        raise ValueError("pair_axes: 1 to 8 sections of 64 pairs in all")
    if not interleaved:
        return b"".join(bytes((a,)) * n for a, n in enumerate(left))
    out, dealt = b"", 0
    while len(out) < 64:
        live = [a for a, n in enumerate(left) if n > dealt]
        rounds = min(left[a] for a in live) - dealt
        out += bytes(live) * rounds
        dealt += rounds
    return out


def _rotate_args(who, q, k, positions, axes, theta, q_out, k_out, v, pages, slots, stream):
    """-> the arguments of a rotation, its device, q_out, k_out"""
    import torch
    some = q if q is not None else k
    if some is None:
        raise ValueError(f"{who}: neither q nor k")
    dev, dtype, n = _device(some, stream), some.dtype, some.shape[0]
    a = RotateArgs()
    a.num_tokens, a.head_dim, a.kv_dtype = n, 128, _kv(dtype)
    hk = a.num_kv_heads = k.shape[1] if k is not None else 1
    a.num_q_heads = q.shape[1] if q is not None else hk
    if not isinstance(axes, bytes) or len(axes) != 64:
        raise ValueError(f"{who}: axes are 64 bytes (pair_axes)")
    num_axes = a.num_axes = max(axes) + 1
    a.axes, a.theta = axes, theta
    if positions.dim() == 1:
        a.positions = _flat(positions, "positions", torch.int32, dev, n)
    else:
        if positions.shape[0] < num_axes:
            raise ValueError(f"{who}: positions has fewer axes than axes names")
        a.positions, a.position_stride = _flat(positions, "positions", torch.int32, dev, positions.shape[0], n), n
    if q is not None:
        a.q, a.q_stride = _rows(q, "q", dtype, dev)
        if q_out is None:
            q_out = _new((n, a.num_q_heads, 128), dtype, q, stream)
            a.q_out, a.q_out_stride = q_out.data_ptr(), a.num_q_heads * 128
        else:
            if q_out.shape != q.shape:
                raise ValueError(f"{who}: q_out must have q's shape")
            a.q_out, a.q_out_stride = _rows(q_out, "q_out", dtype, dev)
    elif q_out is not None:
        raise ValueError(f"{who}: q_out without q")
    if k is not None:
        if k.shape[0] != n:
            raise ValueError(f"{who}: q and k must have the same rows")
        a.k, a.k_stride = _rows(k, "k", dtype, dev)
        if k_out is None and pages is None:
            k_out = _new((n, hk, 128), dtype, k, stream)
        if k_out is not None:
            if k_out.shape != k.shape:
                raise ValueError(f"{who}: k_out must have k's shape")
            a.k_out, a.k_out_stride = _rows(k_out, "k_out", dtype, dev)
    elif k_out is not None:
        raise ValueError(f"{who}: k_out without k")
    if pages is not None:
        if k is None or v is None or slots is None or v.shape != k.shape:
            raise ValueError(f"{who}: pages take k, v of its shape, and slots")
        a.v, a.v_stride = _rows(v, "v", dtype, dev)
        p = _pages(pages, dtype, dev, hk)
        a.pages = ctypes.pointer(p)
        a.slots = _flat(slots, "slots", torch.int32, dev, n)
    elif v is not None or slots is not None:
        raise ValueError(f"{who}: v and slots need pages")
    return a, dev, q_out, k_out


def rotate(q, k, positions, axes: bytes, theta: float, *, q_out=None, k_out=None, v=None, pages=None, slots=None,
           stream=None):
    """protokv_rotate on token rows q [N][Hq][D] and k [N][Hkv][D] (either may be
    None; rows may be strided): positions int32 [num_axes][N] (or [N]: every axis
    the same), axes from ``pair_axes``.  With pages=(k, v) tensors [num_pages][Hkv]
    [page_size][D] and slots int32 [N] the turned keys and v's rows are stored, and
    k_out is written only if given.  -> (q_out, k_out)"""
    a, dev, q_out, k_out = _rotate_args("rotate", q, k, positions, axes, theta, q_out, k_out, v, pages, slots, stream)
    _check(lib().protokv_rotate(ctypes.byref(a), _raw_stream(stream, dev)))
    return q_out, k_out


def norm_rotate(q, k, positions, axes: bytes, theta: float, q_norm, k_norm, eps: float, *, q_out=None, k_out=None, v=None,
                pages=None, slots=None, stream=None):
    """protokv_norm_rotate: ``rotate`` of heads that are normalised first, x / sqrt(mean(x^2) + eps)
    times q_norm or k_norm [128] of the rows' type (None: ones).  -> (q_out, k_out)"""
    a, dev, q_out, k_out = _rotate_args("norm_rotate", q, k, positions, axes, theta, q_out, k_out, v, pages, slots, stream)
    dtype = (q if q is not None else k).dtype
    n = HeadNorm(None if q_norm is None else _flat(q_norm, "q_norm", dtype, dev, 128),
                 None if k_norm is None else _flat(k_norm, "k_norm", dtype, dev, 128), eps)
    _check(lib().protokv_norm_rotate(ctypes.byref(a), ctypes.byref(n), _raw_stream(stream, dev)))
    return q_out, k_out


class PagePlan:
    """What protokv_page_plan returned: cu [n+1], kv_len [n], slots and positions
    [max_tokens], count [1] (pages left on the stack), refused [1]."""
    __slots__ = ("cu", "kv_len", "slots", "positions", "count", "refused")


def page_plan(ctx, add, table, free_pages, count, page_size: int, max_tokens: int, *, base=None, count_out=None,
              stream=None) -> PagePlan:
    """protokv_page_plan: one step's slots, positions and lengths from the requests'
    held (ctx) and new (add, < 0: over) tokens, int32 [n]; table int32 [n][width] and
    the stack free_pages [num_pages] are updated in place, count [1] is not
    (count_out or a new tensor holds the pages left).  add < 0 gives back a request's
    pages whoever else holds them: once some may be shared (``page_fork``), requests are
    ended by ``page_release``, and their add is 0 here.  The results are parts of one
    new tensor."""
    import torch
    dev, i32, n = _device(ctx, stream), torch.int32, ctx.shape[0]
    if max_tokens < 1:
        raise ValueError("page_plan: max_tokens must be >= 1")
    out = PagePlan()
    out.cu, out.kv_len, out.slots, out.positions, out.refused, out.count = torch.unsafe_split_with_sizes(
        _new((2 * n + 2 * max_tokens + 3,), i32, ctx, stream), (n + 1, n, max_tokens, max_tokens, 1, 1))
    if count_out is not None:
        out.count = count_out
    width, pages = table.shape[1], free_pages.shape[0]
    cu = out.cu.data_ptr()
    a = PagePlanArgs(n, pages, page_size, width, max_tokens, _flat(ctx, "ctx", i32, dev, n),
                     _flat(add, "add", i32, dev, n), None if base is None else _flat(base, "base", i32, dev, n),
                     _flat(table, "table", i32, dev, n, width), _flat(free_pages, "free_pages", i32, dev, pages),
                     _flat(count, "count", i32, dev, 1), _flat(out.count, "count_out", i32, dev, 1),
                     cu, cu + 4 * (n + 1), cu + 4 * (2 * n + 1), cu + 4 * (2 * n + 1 + max_tokens),
                     cu + 4 * (2 * n + 1 + 2 * max_tokens))
    _check(lib().protokv_page_plan(ctypes.byref(a), _raw_stream(stream, dev)))
    return out


def prompt_attend(q, k, v, cu, *, out=None, lse=None, prior=None, stream=None):
    """protokv_prompt_attend on token rows q [N][Hq][D], k, v [N][Hkv][D] (rows may be
    strided) of the packed sequences cu int32 [n+1]; prior: (o, lse) of the same rows
    over other keys, joined with the result.  -> (o, lse); lse=False: none."""
    import torch
    dev, dtype = _device(q, stream), q.dtype
    a = PromptArgs()
    a.q, a.q_stride = _rows(q, "q", dtype, dev)
    a.k, a.k_stride = _rows(k, "k", dtype, dev)
    a.v, a.v_stride = _rows(v, "v", dtype, dev)
    if k.shape != v.shape or k.shape[0] != q.shape[0]:
        raise ValueError("prompt_attend: q, k and v must have the same rows, k and v the same heads")
    a.total, a.num_q_heads, _ = q.shape
    a.num_kv_heads, a.head_dim, a.kv_dtype = k.shape[1], 128, _kv(dtype)
    a.num_seqs = cu.shape[0] - 1
    a.cu = _flat(cu, "cu", torch.int32, dev, cu.shape[0])
    out, lse = _result(a, q, out, lse, prior, dev, stream)
    _check(lib().protokv_prompt_attend(ctypes.byref(a), _raw_stream(stream, dev)))
    return out, lse


def page_attend(q, pages, table, cu, kv_len, max_add: int, *, out=None, lse=None, prior=None, workspace=None,
                stream=None):
    """protokv_page_attend: rows q [N][Hq][D] of the requests cu int32 [n+1], at most
    max_add each, over their kv_len [n] tokens in pages=(k, v) [num_pages][Hkv]
    [page_size][D] by the block table [n][width].  workspace: a uint8 tensor (None: one
    of this call's own).  -> (o, lse); lse=False: none."""
    import torch
    dev, dtype, i32 = _device(q, stream), q.dtype, torch.int32
    a = PageAttendArgs()
    a.q, a.q_stride = _rows(q, "q", dtype, dev)
    a.total, a.num_q_heads, _ = q.shape
    a.num_kv_heads, a.head_dim, a.kv_dtype = pages[0].shape[1], 128, _kv(dtype)
    a.pages = _pages(pages, dtype, dev, a.num_kv_heads)
    n, width = cu.shape[0] - 1, table.shape[1]
    a.num_requests, a.max_add, a.table_stride = n, max_add, width
    a.cu, a.kv_len = _flat(cu, "cu", i32, dev, n + 1), _flat(kv_len, "kv_len", i32, dev, n)
    a.table = _flat(table, "table", i32, dev, n, width)
    out, lse = _result(a, q, out, lse, prior, dev, stream)
    if workspace is None:
        need = ctypes.c_size_t()
        _check(lib().protokv_page_attend_workspace(ctypes.byref(a), ctypes.byref(need)))
        if need.value:
            workspace = _new((need.value,), torch.uint8, q, stream)
    elif workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError("workspace: expected a contiguous tensor on the current device")
    if workspace is not None:
        a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    _check(lib().protokv_page_attend(ctypes.byref(a), _raw_stream(stream, dev)))
    return out, lse


# -- a cache in 4 bits, and pages that several requests hold ------------------


def _pages4(pages, dev, kv_heads) -> Pages4:
    """Pages of 4 bits: uint8 tensors (k, v) [num_pages][kv heads][page size][64] and their
    scales (k_scale, v_scale) [num_pages][kv heads][page size][4]."""
    import torch
    k, v, ks, vs = pages
    shape, u8 = k.shape, torch.uint8
    if len(shape) != 4 or shape[1] != kv_heads or shape[3] != 64 or v.shape != shape or ks.shape != (*shape[:3], 4) or (
            vs.shape != ks.shape):
        raise ValueError(f"pages: expected k and v [num_pages, {kv_heads}, page_size, 64] and scales [.., 4]")
    for t in pages:
        if t.dtype != u8 or t.get_device() != dev or not t.is_contiguous():
            raise ValueError(f"pages: expected contiguous uint8 tensors on the current device, got {t.dtype} on {t.device}")
    return Pages4(k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(), shape[0], shape[2])


def page4_store(k, v, pages, slots, *, stream=None):
    """protokv_page4_store: token rows k, v [N][Hkv][D] (rows may be strided) into their slots int32 [N]
    of pages=(k, v, k_scale, v_scale), uint8 [num_pages][Hkv][page_size][64] and [..][4]."""
    import torch
    dev, dtype = _device(k, stream), k.dtype
    n, hk = k.shape[:2]
    if v.shape != k.shape:
        raise ValueError("page4_store: k and v must have the same shape")
    (kp, ks), (vp, vs) = _rows(k, "k", dtype, dev), _rows(v, "v", dtype, dev)
    a = Page4RowsArgs(n, hk, 128, _kv(dtype), kp, vp, ks, vs, _flat(slots, "slots", torch.int32, dev, n),
                      _pages4(pages, dev, hk))
    _check(lib().protokv_page4_store(ctypes.byref(a), _raw_stream(stream, dev)))


def page4_read(pages, slots, dtype, *, k_out=None, v_out=None, stream=None):
    """protokv_page4_read: the rows of k and v that the slots int32 [N] of pages (as in ``page4_store``)
    hold, as bfloat16 or float32.  -> (k_out, v_out) [N][Hkv][D]"""
    import torch
    dev, n, hk = _device(slots, stream), slots.shape[0], pages[0].shape[1]
    if k_out is None and v_out is None:
        k_out, v_out = _new((2, n, hk, 128), dtype, pages[0], stream).unbind(0)
    elif k_out is None:
        k_out = _new((n, hk, 128), dtype, pages[0], stream)
    elif v_out is None:
        v_out = _new((n, hk, 128), dtype, pages[0], stream)
    if k_out.shape != (n, hk, 128) or v_out.shape != (n, hk, 128):
        raise ValueError(f"page4_read: k_out and v_out must be [{n}, {hk}, 128]")
    (kp, ks), (vp, vs) = _rows(k_out, "k_out", dtype, dev), _rows(v_out, "v_out", dtype, dev)
    a = Page4RowsArgs(n, hk, 128, _kv(dtype), kp, vp, ks, vs, _flat(slots, "slots", torch.int32, dev, n),
                      _pages4(pages, dev, hk))
    _check(lib().protokv_page4_read(ctypes.byref(a), _raw_stream(stream, dev)))
    return k_out, v_out


def page4_attend(q, pages, table, cu, kv_len, max_add: int, *, out=None, lse=None, prior=None, workspace=None, stream=None):
    """protokv_page4_attend: ``page_attend`` over pages of 4 bits (as in ``page4_store``), the softmax weights
    of bfloat16 calls rounded to bfloat16 as there.  -> (o, lse); lse=False: none."""
    import torch
    dev, dtype, i32, f32 = _device(q, stream), q.dtype, torch.int32, torch.float32
    qp, qs = _rows(q, "q", dtype, dev)
    total, hq, _ = q.shape
    hk, n, width = pages[0].shape[1], cu.shape[0] - 1, table.shape[1]
    paged, kv = _pages4(pages, dev, hk), _kv(dtype)
    if out is None:
        out = torch.empty_like(q) if stream is None and q.is_contiguous() else _new((total, hq, 128), dtype, q, stream)
        o = out.data_ptr()
    else:
        o = _flat(out, "out", dtype, dev, total, hq, 128)
    l = po = pl = None
    if lse is None:
        lse = _new((total, hq), f32, q, stream)
        l = lse.data_ptr()
    elif lse is not False:
        l = _flat(lse, "lse", f32, dev, total, hq)
    if prior is not None:
        po, pl = _flat(prior[0], "prior", dtype, dev, total, hq, 128), _flat(prior[1], "prior lse", f32, dev, total, hq)
    a = Page4AttendArgs(hq, hk, 128, kv, n, total, max_add, width, _flat(cu, "cu", i32, dev, n + 1),
                        _flat(kv_len, "kv_len", i32, dev, n), _flat(table, "table", i32, dev, n, width), qp, qs, paged, o, l,
                        po, pl, None, 0)
    at = ctypes.byref(a)
    if workspace is None:
        need = ctypes.c_size_t()
        _check(lib().protokv_page4_attend_workspace(at, ctypes.byref(need)))
        if need.value:
            workspace = _new((need.value,), torch.uint8, q, stream)
    elif workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError("workspace: expected a contiguous tensor on the current device")
    if workspace is not None:
        a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    _check(lib().protokv_page4_attend(at, _raw_stream(stream, dev)))
    return out, lse


class PageFork:
    """What protokv_page_fork returned: ctx [requests], lens, copy_src, copy_dst and
    copy_rows [forks], count [1] (pages left on the stack), refused [1]."""
    __slots__ = ("ctx", "lens", "copy_src", "copy_dst", "copy_rows", "count", "refused")


def page_fork(ctx, src, dst, table, shares, free_pages, count, page_size: int, *, at=None, stream=None) -> PageFork:
    """protokv_page_fork: requests dst begin as copies of requests src (int32 [forks]), of their first `at`
    tokens (None: all that ctx [requests] says); table [requests][width] and shares [num_pages] are
    updated in place, the stack free_pages [num_pages] and count [1] are not.  ``page_copy`` then
    brings the rows of the last pages.  The results are parts of one new tensor."""
    import torch
    dev, i32, r, n = _device(ctx, stream), torch.int32, ctx.shape[0], src.shape[0]
    out = PageFork()
    out.ctx, out.lens, out.copy_src, out.copy_dst, out.copy_rows, out.count, out.refused = torch.unsafe_split_with_sizes(
        _new((r + 4 * n + 2,), i32, ctx, stream), (r, n, n, n, n, 1, 1))
    width, pages, p = table.shape[1], free_pages.shape[0], out.ctx.data_ptr()
    lens = p + 4 * r
    a = PageForkArgs(n, r, pages, page_size, width, _flat(ctx, "ctx", i32, dev, r), _flat(src, "src", i32, dev, n),
                     _flat(dst, "dst", i32, dev, n), None if at is None else _flat(at, "at", i32, dev, n),
                     _flat(table, "table", i32, dev, r, width), _flat(shares, "shares", i32, dev, pages),
                     _flat(free_pages, "free_pages", i32, dev, pages), _flat(count, "count", i32, dev, 1),
                     lens + 16 * n, p, lens, lens + 4 * n, lens + 8 * n, lens + 12 * n, lens + 16 * n + 4)
    _check(lib().protokv_page_fork(ctypes.byref(a), _raw_stream(stream, dev)))
    return out


def page_copy(arrays, src, dst, rows=None, *, stream=None):
    """protokv_page_copy: the first rows [n] (None: all) of every head of pages src [n] to pages dst [n], in
    each of the arrays: contiguous tensors [num_pages][Hkv][page_size][row] of one layer, or
    [layers][num_pages][Hkv][page_size][row] of several, of any type."""
    import torch
    arrays = list(arrays)
    if not 1 <= len(arrays) <= 128:
        raise ValueError("page_copy: 1 to 128 arrays")
    dev, i32, n = _device(arrays[0], stream), torch.int32, src.shape[0]
    shape = arrays[0].shape[-4:-1]
    if len(shape) != 3:
        raise ValueError("page_copy: expected arrays [num_pages, heads, page_size, row], or of several layers")
    pages, heads, size = shape
    each = (PageArray * len(arrays))()
    for x, t in zip(each, arrays):
        if t.dim() not in (4, 5) or t.shape[-4:-1] != shape or t.get_device() != dev or not t.is_contiguous():
            raise ValueError(f"page_copy: expected contiguous arrays of pages {tuple(shape)} on the current device, got "
                             f"{tuple(t.shape)} on {t.device}")
        if t.requires_grad:
            _no_gradient("page_copy's arrays")
        row = t.shape[-1] * t.element_size()
        x.base, x.row_bytes, x.layers = t.data_ptr(), row, 1 if t.dim() == 4 else t.shape[0]
        x.layer_stride = row * size * heads * pages
    a = PageCopyArgs(n, heads, pages, size, len(arrays), each, _flat(src, "src", i32, dev, n),
                     _flat(dst, "dst", i32, dev, n), None if rows is None else _flat(rows, "rows", i32, dev, n))
    _check(lib().protokv_page_copy(ctypes.byref(a), _raw_stream(stream, dev)))


class PageRelease:
    """What protokv_page_release returned: ctx [requests], count [1] (pages on the stack), refused [1]."""
    __slots__ = ("ctx", "count", "refused")


def page_release(ctx, keep, table, shares, free_pages, count, page_size: int, *, stream=None) -> PageRelease:
    """protokv_page_release: requests of ctx tokens keep the first `keep` (int32 [requests]); pages
    [num_pages] that nobody holds any more go onto the stack free_pages, which is updated in place
    as shares is; count [1] is not.  The results are parts of one new tensor."""
    import torch
    dev, i32, n = _device(ctx, stream), torch.int32, ctx.shape[0]
    width, pages = table.shape[1], free_pages.shape[0]
    blocks = (pages + RELEASE_PAGES - 1) // RELEASE_PAGES
    out = PageRelease()
    out.ctx, out.count, out.refused, scratch = torch.unsafe_split_with_sizes(
        _new((n + 2 + blocks,), i32, ctx, stream), (n, 1, 1, blocks))
    p = out.ctx.data_ptr()
    a = PageReleaseArgs(n, pages, page_size, width, _flat(ctx, "ctx", i32, dev, n), _flat(keep, "keep", i32, dev, n),
                        _flat(table, "table", i32, dev, n, width), _flat(shares, "shares", i32, dev, pages),
                        _flat(free_pages, "free_pages", i32, dev, pages), _flat(count, "count", i32, dev, 1),
                        p + 4 * n, p, p + 4 * n + 4, p + 4 * n + 8)
    _check(lib().protokv_page_release(ctypes.byref(a), _raw_stream(stream, dev)))
    return out
