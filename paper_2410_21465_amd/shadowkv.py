"""ctypes binding of libshadowkv.so: argument marshalling only.

Every step of the path runs in the HIP library; this module turns torch tensors
into pointers, sizes the workspace and picks the streams.  There is no fallback:
if the library is missing, loading raises.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("SHADOWKV_LIB", os.path.join(_HERE, "libshadowkv.so"))

OK, EINVAL, EWORKSPACE, EHIP = 0, -1, -2, -3
VALUES_DEVICE, VALUES_HOST = 0, 1
FLAG_STAGE_VALUES = 1
FLAG_KEEP_REBUILT_KEYS = 2
KV_BF16, KV_FP8_E5M2 = 0, 1     # storage type of the KV-cache tensors (Params.kv_dtype)
LOGITS_BF16, LOGITS_FP16, LOGITS_FP32 = 0, 1, 2
ROPE_HALF, ROPE_INTERLEAVED = 0, 1                                        # Rope.layout
ROPE_PLAIN, ROPE_LINEAR, ROPE_NTK, ROPE_BANDS, ROPE_YARN = 0, 1, 2, 3, 4  # Rope.scaling

EXPORTS = (
    "shadowkv_build_landmarks", "shadowkv_decode_step", "shadowkv_build_workspace_bytes",
    "shadowkv_decode_workspace_bytes", "shadowkv_validate_params", "shadowkv_decode_workspace_view",
    "shadowkv_status_string", "shadowkv_last_error", "shadowkv_version", "shadowkv_shutdown",
    "shadowkv_profile_begin", "shadowkv_profile_end", "shadowkv_decode_step_cached", "shadowkv_value_cache_bytes",
    "shadowkv_value_cache_reset", "shadowkv_append_chunk", "shadowkv_argtopk", "shadowkv_argtopk_workspace_bytes",
    "shadowkv_factorize_keys", "shadowkv_factorize_workspace_bytes", "shadowkv_decode_step_static",
    "shadowkv_static_scratch_bytes", "shadowkv_decode_plan", "shadowkv_factorize_plan",
    "shadowkv_decode_score_rows", "shadowkv_rope_frequencies", "shadowkv_rotate", "shadowkv_paged_append",
    "shadowkv_paged_attention", "shadowkv_paged_attention_workspace_bytes", "shadowkv_beam_select",
    "shadowkv_beam_select_workspace_bytes", "shadowkv_reorder_rows", "shadowkv_pages_update", "shadowkv_pages_compact",
    "shadowkv_pages_workspace_bytes", "shadowkv_pages_copy",
)
STAGES = ("score", "select", "gather_values", "attention")


class CParams(C.Structure):
    _fields_ = [
        ("batch", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
        ("ctx_len", C.c_int32), ("chunk_size", C.c_int32), ("rank", C.c_int32),
        ("n_outlier_chunks", C.c_int32), ("topk_chunks", C.c_int32), ("local_len", C.c_int32),
        ("value_location", C.c_int32), ("flags", C.c_uint32),
        ("rope_theta", C.c_double), ("softmax_scale", C.c_double), ("inv_freq", C.c_void_p),
        ("ctx_capacity", C.c_int32), ("kv_dtype", C.c_int32),
    ]


class CHeads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("seq_stride", C.c_int64), ("token_stride", C.c_int64), ("head_stride", C.c_int64),
                ("n_seqs", C.c_int32), ("n_tokens", C.c_int32), ("n_heads", C.c_int32), ("dtype", C.c_int32)]


class CRope(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("rot_dim", C.c_int32), ("layout", C.c_int32), ("scaling", C.c_int32),
                ("theta", C.c_double), ("factor", C.c_double), ("low", C.c_double), ("high", C.c_double),
                ("original_len", C.c_int32), ("reserved", C.c_int32), ("magnitude", C.c_double), ("inv_freq", C.c_void_p)]


class CPagedCache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p),
                ("k_page_stride", C.c_int64), ("k_head_stride", C.c_int64), ("k_token_stride", C.c_int64),
                ("v_page_stride", C.c_int64), ("v_head_stride", C.c_int64), ("v_token_stride", C.c_int64),
                ("page_table", C.c_void_p), ("table_stride", C.c_int64),
                ("batch", C.c_int32), ("pages_per_seq", C.c_int32), ("n_pages", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("page_size", C.c_int32), ("kv_dtype", C.c_int32), ("reserved", C.c_int32)]


class CLogits(C.Structure):
    _fields_ = [("data", C.c_void_p), ("group_stride", C.c_int64), ("beam_stride", C.c_int64), ("n_groups", C.c_int32),
                ("n_beams", C.c_int32), ("vocab", C.c_int32), ("dtype", C.c_int32)]


class CRows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("row_stride", C.c_int64), ("outer_stride", C.c_int64), ("inner", C.c_int64),
                ("n_outer", C.c_int32), ("reserved", C.c_int32)]


class CPagePool(C.Structure):
    _fields_ = [("page_table", C.c_void_p), ("table_stride", C.c_int64), ("kv_lens", C.c_void_p), ("page_refs", C.c_void_p),
                ("batch", C.c_int32), ("pages_per_seq", C.c_int32), ("n_pages", C.c_int32), ("page_size", C.c_int32)]


class CPageMoves(C.Structure):
    _fields_ = [("src", C.c_void_p), ("dst", C.c_void_p), ("rows", C.c_void_p), ("count", C.c_void_p), ("capacity", C.c_int32),
                ("reserved", C.c_int32)]


class ShadowKVError(RuntimeError):
    def __init__(self, status: int, detail: str):
        super().__init__(f"libshadowkv: {status_string(status)} ({status}): {detail}")
        self.status = status
        self.detail = detail


_lib = None


def lib() -> C.CDLL:
    """Load the HIP library (built beforehand by ``python -m paper_2410_21465_amd.build``)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2410_21465_amd.build` "
                "(there is no non-HIP fallback)")
        L = C.CDLL(LIB_PATH)
        vp, sz, i32 = C.c_void_p, C.c_size_t, C.c_int
        L.shadowkv_build_landmarks.restype = i32
        L.shadowkv_build_landmarks.argtypes = [vp] * 9 + [sz, vp]
        L.shadowkv_decode_step.restype = i32
        L.shadowkv_decode_step.argtypes = [vp] * 15 + [sz, vp, vp]
        L.shadowkv_decode_step_static.restype = i32
        L.shadowkv_decode_step_static.argtypes = [vp] * 15
        L.shadowkv_static_scratch_bytes.restype = sz
        L.shadowkv_static_scratch_bytes.argtypes = []
        L.shadowkv_decode_step_cached.restype = i32
        L.shadowkv_decode_step_cached.argtypes = [vp] * 12 + [i32] + [vp] * 7 + [sz, vp, vp]
        L.shadowkv_value_cache_bytes.restype = sz
        L.shadowkv_value_cache_bytes.argtypes = [vp, i32]
        L.shadowkv_value_cache_reset.restype = i32
        L.shadowkv_value_cache_reset.argtypes = [vp, i32, vp, vp, vp]
        L.shadowkv_argtopk.restype = i32
        L.shadowkv_argtopk.argtypes = [vp, i32, i32, i32, C.c_double, vp, vp, sz, vp]
        L.shadowkv_argtopk_workspace_bytes.restype = sz
        L.shadowkv_argtopk_workspace_bytes.argtypes = [i32, i32, i32]
        L.shadowkv_append_chunk.restype = i32
        L.shadowkv_append_chunk.argtypes = [vp] * 10
        L.shadowkv_factorize_keys.restype = i32
        L.shadowkv_factorize_keys.argtypes = [vp] * 6 + [i32, vp, sz, vp]
        L.shadowkv_factorize_workspace_bytes.restype = sz
        L.shadowkv_factorize_workspace_bytes.argtypes = [vp]
        L.shadowkv_factorize_plan.restype = i32
        L.shadowkv_factorize_plan.argtypes = [vp, vp]
        L.shadowkv_decode_score_rows.restype = i32
        L.shadowkv_decode_score_rows.argtypes = [vp]
        L.shadowkv_rope_frequencies.restype = i32
        L.shadowkv_rope_frequencies.argtypes = [vp, vp]
        L.shadowkv_rotate.restype = i32
        L.shadowkv_rotate.argtypes = [vp] * 5 + [i32, vp]
        L.shadowkv_paged_append.restype = i32
        L.shadowkv_paged_append.argtypes = [vp] * 10
        L.shadowkv_paged_attention.restype = i32
        L.shadowkv_paged_attention.argtypes = [vp] * 6 + [i32, C.c_double, vp, sz, vp]
        L.shadowkv_paged_attention_workspace_bytes.restype = sz
        L.shadowkv_paged_attention_workspace_bytes.argtypes = [vp, i32, i32]
        L.shadowkv_beam_select.restype = i32
        L.shadowkv_beam_select.argtypes = [vp] * 4 + [C.c_double, C.c_double, C.c_int32, C.c_int32] + [vp] * 6 + [sz, vp]
        L.shadowkv_beam_select_workspace_bytes.restype = sz
        L.shadowkv_beam_select_workspace_bytes.argtypes = [vp, C.c_int32]
        L.shadowkv_reorder_rows.restype = i32
        L.shadowkv_reorder_rows.argtypes = [vp, C.c_int32, vp, C.c_int32, vp]
        L.shadowkv_pages_update.restype = i32
        L.shadowkv_pages_update.argtypes = [vp] * 4 + [C.c_int32, vp, vp, sz, vp]
        L.shadowkv_pages_compact.restype = i32
        L.shadowkv_pages_compact.argtypes = [vp, C.c_int32, vp, vp, vp, sz, vp]
        L.shadowkv_pages_workspace_bytes.restype = sz
        L.shadowkv_pages_workspace_bytes.argtypes = [vp]
        L.shadowkv_pages_copy.restype = i32
        L.shadowkv_pages_copy.argtypes = [vp, vp, C.c_int32, vp, vp]
        L.shadowkv_build_workspace_bytes.restype = sz
        L.shadowkv_build_workspace_bytes.argtypes = [vp]
        L.shadowkv_decode_workspace_bytes.restype = sz
        L.shadowkv_decode_workspace_bytes.argtypes = [vp]
        L.shadowkv_validate_params.restype = i32
        L.shadowkv_validate_params.argtypes = [vp, i32]
        L.shadowkv_decode_workspace_view.restype = vp
        L.shadowkv_decode_workspace_view.argtypes = [vp, vp, i32]
        L.shadowkv_status_string.restype = C.c_char_p
        L.shadowkv_status_string.argtypes = [i32]
        L.shadowkv_last_error.restype = C.c_char_p
        L.shadowkv_version.restype = i32
        L.shadowkv_shutdown.restype = None
        L.shadowkv_profile_begin.restype = i32
        L.shadowkv_profile_begin.argtypes = [i32]
        L.shadowkv_profile_end.restype = i32
        L.shadowkv_profile_end.argtypes = [vp, vp]
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().shadowkv_status_string(status).decode()


def last_error() -> str:
    return lib().shadowkv_last_error().decode()


def version() -> int:
    return int(lib().shadowkv_version())


def profile_begin(max_steps: int) -> None:
    _check(lib().shadowkv_profile_begin(int(max_steps)))


def decode_plan(p: "Params") -> dict:
    """shadowkv_decode_plan: how a plain decode step of this shape is laid out on the GPU."""
    st = p.c_struct()
    plan = (C.c_int32 * 8)()
    _check(lib().shadowkv_decode_plan(C.byref(st), plan))
    return {"splits": plan[0], "rows_per_split": plan[1], "resident_rows_in_selection_launch": bool(plan[2]),
            "key_and_value_waves": bool(plan[3]), "selection_threads": plan[4], "selection_candidates_per_thread": plan[5],
            "selection_launches": plan[6], "logit_row_floats": plan[7]}


def decode_score_rows(p: "Params") -> int:
    """shadowkv_decode_score_rows: landmark rows per scoring workgroup of a decode step of this shape."""
    st = p.c_struct()
    return lib().shadowkv_decode_score_rows(C.byref(st))


def profile_end() -> dict:
    """Stops stage timing; returns {"steps": n, "ms": {stage: mean milliseconds per step}}."""
    ms = (C.c_double * 4)()
    n = C.c_int(0)
    _check(lib().shadowkv_profile_end(ms, C.byref(n)))
    steps = max(n.value, 1)
    return {"steps": n.value, "ms": {name: ms[i] / steps for i, name in enumerate(STAGES)}}


def _check(status: int) -> None:
    if status != OK:
        raise ShadowKVError(status, last_error())


@dataclass
class Params:
    batch: int
    n_q_heads: int
    n_kv_heads: int
    head_dim: int
    ctx_len: int
    chunk_size: int = 8
    rank: int = 160
    n_outlier_chunks: int = 48
    topk_chunks: int = 256
    local_len: int = 32
    value_location: int = VALUES_DEVICE
    flags: int = 0
    rope_theta: float = 5e5
    softmax_scale: float = 0.0
    inv_freq: Optional[torch.Tensor] = None   # device float32 [head_dim/2]
    ctx_capacity: int = 0                     # tokens the context arrays are laid out for (0 => ctx_len)
    kv_dtype: int = KV_BF16                   # KV_BF16 | KV_FP8_E5M2: storage of every KV-cache tensor

    @property
    def kv_torch_dtype(self) -> torch.dtype:
        return torch.float8_e5m2 if self.kv_dtype == KV_FP8_E5M2 else torch.bfloat16

    @property
    def kv_bytes(self) -> int:
        return 1 if self.kv_dtype == KV_FP8_E5M2 else 2

    @property
    def n_chunks(self) -> int:
        return self.ctx_len // self.chunk_size

    @property
    def capacity(self) -> int:
        return self.ctx_capacity or self.ctx_len

    @property
    def landmark_capacity(self) -> int:
        return self.capacity // self.chunk_size - self.n_outlier_chunks

    @property
    def n_landmarks(self) -> int:
        return self.n_chunks - self.n_outlier_chunks

    def c_struct(self) -> CParams:
        inv = None
        if self.inv_freq is not None:
            assert self.inv_freq.dtype == torch.float32 and self.inv_freq.is_contiguous()
            inv = self.inv_freq.data_ptr()
        return CParams(self.batch, self.n_q_heads, self.n_kv_heads, self.head_dim, self.ctx_len, self.chunk_size,
                       self.rank, self.n_outlier_chunks, self.topk_chunks, self.local_len, self.value_location,
                       self.flags, float(self.rope_theta), float(self.softmax_scale), inv, int(self.ctx_capacity),
                       int(self.kv_dtype))

    @classmethod
    def from_workload(cls, wl, **kw) -> "Params":
        loc = VALUES_HOST if wl.value_location == "host" else VALUES_DEVICE
        base = dict(batch=wl.batch, n_q_heads=wl.n_q_heads, n_kv_heads=wl.n_kv_heads, head_dim=wl.head_dim,
                    ctx_len=wl.ctx_len, chunk_size=wl.chunk_size, rank=wl.rank,
                    n_outlier_chunks=wl.n_outlier_chunks, topk_chunks=wl.topk_chunks, local_len=wl.local_len,
                    value_location=loc, rope_theta=wl.rope_theta)
        base.update(kw)
        return cls(**base)


def validate_params(p: Params, for_decode: bool = True) -> int:
    st = p.c_struct()
    return int(lib().shadowkv_validate_params(C.addressof(st), 1 if for_decode else 0))


def decode_workspace_bytes(p: Params) -> int:
    st = p.c_struct()
    return int(lib().shadowkv_decode_workspace_bytes(C.addressof(st)))


def build_workspace_bytes(p: Params) -> int:
    st = p.c_struct()
    return int(lib().shadowkv_build_workspace_bytes(C.addressof(st)))


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    assert t.is_contiguous(), "tensors must be contiguous"
    return t.data_ptr()


def _stream_ptr(stream) -> int:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def alloc_workspace(nbytes: int, device="cuda") -> torch.Tensor:
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)


def build_landmarks(p: Params, k_rope: torch.Tensor, v: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None, stream=None) -> dict:
    """Pre-filling algorithm after its SVD line.  Returns the new device tensors."""
    b, h, s, d, c, o = p.batch, p.n_kv_heads, p.ctx_len, p.head_dim, p.chunk_size, p.n_outlier_chunks
    n_c = p.landmark_capacity      # rows allocated; the first p.n_landmarks are written
    dev = k_rope.device
    assert k_rope.dtype == p.kv_torch_dtype and tuple(k_rope.shape) == (b, h, s, d)
    if v is not None:
        assert v.dtype == p.kv_torch_dtype and tuple(v.shape) == (b, h, p.capacity, d)
    bf, i32 = p.kv_torch_dtype, torch.int32
    out = {
        "landmarks": torch.empty(b, h, max(n_c, 0), d, dtype=bf, device=dev),
        "landmark_chunk_ids": torch.empty(b, h, max(n_c, 0), dtype=i32, device=dev),
        "outlier_chunk_ids": torch.empty(b, h, o, dtype=i32, device=dev),
        "k_outlier": torch.empty(b, h, o * c, d, dtype=bf, device=dev),
        "v_outlier": torch.empty(b, h, o * c, d, dtype=bf, device=dev) if v is not None else None,
    }
    st = p.c_struct()
    if workspace is None:
        workspace = alloc_workspace(int(lib().shadowkv_build_workspace_bytes(C.addressof(st))), dev)
    rc = lib().shadowkv_build_landmarks(C.addressof(st), _ptr(k_rope), _ptr(v), _ptr(out["landmarks"]),
                                        _ptr(out["landmark_chunk_ids"]), _ptr(out["outlier_chunk_ids"]),
                                        _ptr(out["k_outlier"]), _ptr(out["v_outlier"]), _ptr(workspace),
                                        workspace.numel(), _stream_ptr(stream))
    _check(rc)
    out["workspace"] = workspace
    return out


def decode_step(p: Params, q, A, B, landmarks, landmark_chunk_ids, k_outlier, v_outlier, k_local, v_local,
                value_store, pos_offset=None, out=None, out_chunk_ids=None, workspace=None, stream=None,
                side_stream=None):
    """One decode step.  Returns ``(out [b,h_q,d] bf16, chunk_ids [b,h_kv,k] int32, workspace)``."""
    dev = q.device
    if out is None:
        out = torch.empty(p.batch, p.n_q_heads, p.head_dim, dtype=torch.bfloat16, device=dev)
    if out_chunk_ids is None:
        out_chunk_ids = torch.empty(p.batch, p.n_kv_heads, p.topk_chunks, dtype=torch.int32, device=dev)
    st = p.c_struct()
    if workspace is None:
        workspace = alloc_workspace(int(lib().shadowkv_decode_workspace_bytes(C.addressof(st))), dev)
    rc = lib().shadowkv_decode_step(C.addressof(st), _ptr(q), _ptr(A), _ptr(B), _ptr(landmarks),
                                    _ptr(landmark_chunk_ids), _ptr(k_outlier), _ptr(v_outlier), _ptr(k_local),
                                    _ptr(v_local), _ptr(value_store), _ptr(pos_offset), _ptr(out),
                                    _ptr(out_chunk_ids), _ptr(workspace), workspace.numel(), _stream_ptr(stream),
                                    None if side_stream is None else _stream_ptr(side_stream))
    _check(rc)
    return out, out_chunk_ids, workspace


def static_scratch_bytes() -> int:
    return int(lib().shadowkv_static_scratch_bytes())


def decode_step_static(p: Params, q, A, B, landmarks, landmark_chunk_ids, k_outlier, v_outlier, k_local, v_local,
                       value_store, pos_offset, out, out_chunk_ids, stream=None) -> None:
    """``decode_step`` on the library's static scratch: nothing is allocated, ``out`` and ``out_chunk_ids`` are
    the caller's."""
    st = p.c_struct()
    _check(lib().shadowkv_decode_step_static(C.addressof(st), _ptr(q), _ptr(A), _ptr(B), _ptr(landmarks),
                                             _ptr(landmark_chunk_ids), _ptr(k_outlier), _ptr(v_outlier),
                                             _ptr(k_local), _ptr(v_local), _ptr(value_store), _ptr(pos_offset),
                                             _ptr(out), _ptr(out_chunk_ids), _stream_ptr(stream)))


def factorize_plan(p: "Params") -> dict:
    """shadowkv_factorize_plan: how the keys of this shape are factored on the GPU."""
    st = p.c_struct()
    plan = (C.c_int64 * 5)()
    _check(lib().shadowkv_factorize_plan(C.addressof(st), plan))
    return {"parts": plan[0], "tokens_per_part": plan[1], "entries_per_list": plan[2], "routes_offset": plan[3],
            "fp64_waves": plan[4]}


def factorize_routes(p: "Params", workspace: torch.Tensor) -> torch.Tensor:
    """Which way each sequence of the last ``factorize_keys`` went, int32 [b] aliasing ``workspace``: 0 Gram matrix and A from
    digits, 1 both from fp64 sums, 2 the Gram matrix from digits and A from fp64 sums."""
    off = factorize_plan(p)["routes_offset"]
    return workspace[off:off + 4 * p.batch].view(torch.int32)


def append_chunk(p: Params, k_pre, k_rope, v, B, A, landmarks, landmark_chunk_ids, value_store, stream=None) -> None:
    """Append one chunk of generated tokens to the context in place (``p.ctx_len`` is the length before)."""
    st = p.c_struct()
    _check(lib().shadowkv_append_chunk(C.addressof(st), _ptr(k_pre), _ptr(k_rope), _ptr(v), _ptr(B), _ptr(A),
                                       _ptr(landmarks), _ptr(landmark_chunk_ids), _ptr(value_store),
                                       _stream_ptr(stream)))


def factorize_keys(p: Params, k_pre: torch.Tensor, n_iter: int = 0, want_vectors: bool = False, workspace=None,
                   stream=None) -> dict:
    """First line of the pre-filling algorithm: rank-r factors of the pre-RoPE keys ``k_pre [b, s, h_kv*d]``.
    Returns ``A [b, cap, r]`` and ``B [b, h_kv, r, d]`` in the storage type of the KV cache, and with
    ``want_vectors`` also ``psi [b, r, h_kv*d]`` and ``sigma [b, r]`` (fp64)."""
    b, h, d, r = p.batch, p.n_kv_heads, p.head_dim, p.rank
    dev = k_pre.device
    assert k_pre.dtype == p.kv_torch_dtype and tuple(k_pre.shape) == (b, p.ctx_len, h * d)
    out = {"A": torch.empty(b, p.capacity, r, dtype=p.kv_torch_dtype, device=dev),
           "B": torch.empty(b, h, r, d, dtype=p.kv_torch_dtype, device=dev),
           "psi": torch.empty(b, r, h * d, dtype=torch.float64, device=dev) if want_vectors else None,
           "sigma": torch.empty(b, r, dtype=torch.float64, device=dev) if want_vectors else None}
    st = p.c_struct()
    if workspace is None:
        need = int(lib().shadowkv_factorize_workspace_bytes(C.addressof(st)))
        if need == 0:
            _check(lib().shadowkv_validate_params(C.addressof(st), 0))
            raise ValueError("rank must be a multiple of 8 in [8, 256] and at most h_kv * d")
        workspace = alloc_workspace(need, dev)
    _check(lib().shadowkv_factorize_keys(C.addressof(st), _ptr(k_pre), _ptr(out["A"]), _ptr(out["B"]), _ptr(out["psi"]),
                                         _ptr(out["sigma"]), int(n_iter), _ptr(workspace), workspace.numel(),
                                         _stream_ptr(stream)))
    out["workspace"] = workspace
    return out


def argtopk(scores: torch.Tensor, k: int, largest: bool = True, stream=None) -> torch.Tensor:
    """Indices of the k largest (or smallest) of each row of ``scores [units, n]`` (fp64, device), ties to the
    lower index, in ascending index order: ``[units, k]`` int32."""
    assert scores.dtype == torch.float64 and scores.dim() == 2
    units, n = scores.shape
    need = int(lib().shadowkv_argtopk_workspace_bytes(units, n, k))
    ws = alloc_workspace(max(need, 256), scores.device)
    out = torch.empty(units, k, dtype=torch.int32, device=scores.device)
    _check(lib().shadowkv_argtopk(_ptr(scores), units, n, k, 1.0 if largest else -1.0, _ptr(out), _ptr(ws), ws.numel(),
                                  _stream_ptr(stream)))
    return out


class ValueCache:
    """Device buffers of the chunk cache of the value store with ``slots`` >= k slots per (batch, KV head):
    ``values [b,h_kv,slots*c,d]`` in the storage type of the KV cache, ``chunk_ids [b,h_kv,slots]`` int32 (-1 = empty), ``stamps
    [b,h_kv,slots+1]`` int32 (last use per slot, then the unit's clock), ``miss_count [b,h_kv]`` of the last step."""

    def __init__(self, p: Params, slots: Optional[int] = None, device="cuda", stream=None):
        self.slots = int(slots) if slots is not None else p.topk_chunks
        st = p.c_struct()
        n = int(lib().shadowkv_value_cache_bytes(C.addressof(st), self.slots))
        if n == 0:
            _check(lib().shadowkv_validate_params(C.addressof(st), 1))
            raise ValueError(f"cache slots {self.slots} outside [topk_chunks, 8192]")
        self.values = torch.empty(p.batch, p.n_kv_heads, self.slots * p.chunk_size, p.head_dim,
                                  dtype=p.kv_torch_dtype, device=device)
        assert self.values.numel() * p.kv_bytes == n
        self.chunk_ids = torch.empty(p.batch, p.n_kv_heads, self.slots, dtype=torch.int32, device=device)
        self.stamps = torch.empty(p.batch, p.n_kv_heads, self.slots + 1, dtype=torch.int32, device=device)
        self.miss_count = torch.zeros(p.batch, p.n_kv_heads, dtype=torch.int32, device=device)
        self.reset(p, stream)

    def reset(self, p: Params, stream=None):
        st = p.c_struct()
        _check(lib().shadowkv_value_cache_reset(C.addressof(st), self.slots, _ptr(self.chunk_ids), _ptr(self.stamps),
                                                _stream_ptr(stream)))


def decode_step_cached(p: Params, q, A, B, landmarks, landmark_chunk_ids, k_outlier, v_outlier, k_local, v_local,
                       value_store, cache: ValueCache, pos_offset=None, out=None, out_chunk_ids=None, workspace=None,
                       stream=None, side_stream=None):
    """One decode step that fetches only the chunks missing from ``cache``.  Returns like ``decode_step``."""
    dev = q.device
    if out is None:
        out = torch.empty(p.batch, p.n_q_heads, p.head_dim, dtype=torch.bfloat16, device=dev)
    if out_chunk_ids is None:
        out_chunk_ids = torch.empty(p.batch, p.n_kv_heads, p.topk_chunks, dtype=torch.int32, device=dev)
    st = p.c_struct()
    if workspace is None:
        workspace = alloc_workspace(int(lib().shadowkv_decode_workspace_bytes(C.addressof(st))), dev)
    rc = lib().shadowkv_decode_step_cached(C.addressof(st), _ptr(q), _ptr(A), _ptr(B), _ptr(landmarks),
                                           _ptr(landmark_chunk_ids), _ptr(k_outlier), _ptr(v_outlier), _ptr(k_local),
                                           _ptr(v_local), _ptr(value_store), _ptr(pos_offset), cache.slots,
                                           _ptr(cache.values), _ptr(cache.chunk_ids), _ptr(cache.stamps),
                                           _ptr(cache.miss_count), _ptr(out),
                                           _ptr(out_chunk_ids), _ptr(workspace), workspace.numel(),
                                           _stream_ptr(stream),
                                           None if side_stream is None else _stream_ptr(side_stream))
    _check(rc)
    return out, out_chunk_ids, workspace


def workspace_view(p: Params, workspace: torch.Tensor, which: str) -> Optional[torch.Tensor]:
    """Intermediate of the last decode step as a tensor aliasing ``workspace``.

    ``"k_sparse"`` fp32 [b,h_kv,k*c,d]; ``"v_sparse"`` in the KV storage type (staged runs only); ``"logits"`` fp32 [b,h_q,n_c] (the copies the search runs on).
    """
    code = {"k_sparse": 0, "v_sparse": 1, "sel_ids": 2, "logits": 3, "miss_slots": 4, "sel_slots": 5}[which]
    st = p.c_struct()
    ptr = lib().shadowkv_decode_workspace_view(C.addressof(st), workspace.data_ptr(), code)
    if not ptr:
        return None
    off = ptr - workspace.data_ptr()
    rows = (p.batch, p.n_kv_heads, p.topk_chunks * p.chunk_size, p.head_dim)
    if which == "k_sparse":
        n = rows[0] * rows[1] * rows[2] * rows[3]
        return workspace[off:off + 4 * n].view(torch.float32).view(rows)
    if which == "v_sparse":
        n = rows[0] * rows[1] * rows[2] * rows[3]
        return workspace[off:off + p.kv_bytes * n].view(p.kv_torch_dtype).view(rows)
    if which in ("sel_ids", "miss_slots", "sel_slots"):
        n = p.batch * p.n_kv_heads * p.topk_chunks
        return workspace[off:off + 4 * n].view(torch.int32).view(p.batch, p.n_kv_heads, p.topk_chunks)
    ld = (p.n_landmarks + 3) // 4 * 4
    n = p.batch * p.n_q_heads * ld
    return workspace[off:off + 4 * n].view(torch.float32).view(p.batch, p.n_q_heads, ld)[:, :, :p.n_landmarks]


# ---- the prompt's way into the cache: rotary positions, a paged KV cache, attention of new tokens over it ----

_DTYPES = {torch.bfloat16: KV_BF16, torch.float8_e5m2: KV_FP8_E5M2}


@dataclass
class Rope:
    """Rotary positions (``shadowkv_rope``): which elements of a head turn, in which pairs, how fast."""
    head_dim: int
    theta: float = 5e5
    rot_dim: int = 0                          # leading elements that are rotated, a multiple of 8 (0 => head_dim)
    layout: int = ROPE_HALF                   # pairs (i, i + rot_dim/2), or ROPE_INTERLEAVED: (2i, 2i + 1)
    scaling: int = ROPE_PLAIN                 # for long contexts: ROPE_LINEAR, ROPE_NTK, ROPE_BANDS, ROPE_YARN
    factor: float = 1.0
    low: float = 0.0                          # turns in original_len (BANDS, YARN)
    high: float = 0.0
    original_len: int = 0
    magnitude: float = 0.0                    # of cosine and sine (0 => 1; YARN: 0.1 ln factor + 1)
    inv_freq: Optional[torch.Tensor] = None   # device float32 [rot_dim/2], replaces the frequencies

    def c_struct(self) -> CRope:
        inv = None
        if self.inv_freq is not None:
            n = (self.rot_dim or self.head_dim) // 2
            _want(self.inv_freq, "inv_freq", torch.float32, (n,))
            inv = self.inv_freq.data_ptr()
        return CRope(self.head_dim, self.rot_dim, self.layout, self.scaling, self.theta, self.factor, self.low, self.high,
                     self.original_len, 0, self.magnitude, inv)

    def frequencies(self) -> torch.Tensor:
        """Radians per position of every pair, float64 on the host.  Rounded, ``inv = frequencies().float().cuda()`` is ``Params.inv_freq``
        of a decode step with the same scaling (whole heads, half layout, magnitude 1).  The rounding turns a pair by up to 2^-25 of
        its position in radians (0.004 at 128K tokens, 0.03 at 1M), so keys and queries of such a context are to be rotated with
        ``Rope(head_dim, inv_freq=inv)``, which uses the same numbers."""
        out = torch.empty((self.rot_dim or self.head_dim) // 2, dtype=torch.float64)
        st = self.c_struct()
        _check(lib().shadowkv_rope_frequencies(C.byref(st), out.data_ptr()))
        return out


def _want(t: torch.Tensor, name: str, dtype, shape, device=None) -> None:
    if t.dtype != dtype or t.shape != tuple(shape) or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)}, not {t.dtype} {tuple(t.shape)}")
    if not t.is_cuda or (device is not None and t.device != device):
        raise ValueError(f"{name} must be on {device or 'the GPU'}, not {t.device}")


def _heads(t: torch.Tensor, name: str, device=None) -> CHeads:
    """[seqs, tokens, heads, d] or [tokens, heads, d] with any strides as ``shadowkv_heads``."""
    sz, st = t.shape, t.stride()
    if len(sz) == 3:
        seqs, seq_stride = 1, 0
    elif len(sz) == 4:
        seqs, seq_stride = sz[0], st[0]
    else:
        raise ValueError(f"{name} must have 3 or 4 dimensions, not {len(sz)}")
    if t.dtype not in _DTYPES:
        raise ValueError(f"{name} must be bfloat16 or float8_e5m2, not {t.dtype}")
    if not t.is_cuda or (device is not None and t.device != device):
        raise ValueError(f"{name} must be on {device or 'the GPU'}, not {t.device}")
    if st[-1] != 1:
        raise ValueError(f"the elements of a head of {name} must be contiguous")
    return CHeads(t.data_ptr(), seq_stride, st[-3], st[-2], seqs, sz[-3], sz[-2], _DTYPES[t.dtype])


class _Launch:
    """Makes ``device`` current, and what is allocated inside belong to ``stream`` (None: the device's current stream)."""

    def __init__(self, device: torch.device, stream):
        if stream is not None and not isinstance(stream, torch.cuda.Stream):
            stream = torch.cuda.ExternalStream(stream, device=device) if stream else torch.cuda.default_stream(device)
        if stream is not None:
            if stream.device != device:
                raise ValueError(f"the stream is on {stream.device}, the tensors on {device}")
            self._ctx = torch.cuda.stream(stream)
        else:
            self._ctx = None if device.index == torch.cuda.current_device() else torch.cuda.device(device)
        self._device = device

    def __enter__(self) -> int:
        if self._ctx is not None:
            self._ctx.__enter__()
        return torch._C._cuda_getCurrentRawStream(self._device.index)   # (a stream object costs 2 us, this 0.1)

    def __exit__(self, *exc):
        if self._ctx is not None:
            self._ctx.__exit__(*exc)


class _OnCurrent:
    """What ``_Launch`` is where there is nothing to enter: entering costs a call less."""

    def __init__(self, raw: int):
        self._raw = raw

    def __enter__(self) -> int:
        return self._raw

    def __exit__(self, *exc):
        pass


def _launch(device: torch.device, stream):
    """``_Launch``, or without its costs where the current device and its current stream are meant."""
    if device.type != "cuda":
        raise ValueError(f"the tensors must be on the GPU, not {device}")
    index = device.index
    if stream is None and index is not None and index == torch._C._cuda_getDevice():
        return _OnCurrent(torch._C._cuda_getCurrentRawStream(index))
    return _Launch(device, stream)


def rotate(rope: Rope, x: torch.Tensor, out: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None,
           pos_offset: Optional[torch.Tensor] = None, transposed: bool = False, stream=None) -> torch.Tensor:
    """Heads ``x [seqs, tokens, heads, d]`` (or ``[tokens, heads, d]``) turned to their positions: ``positions [seqs, tokens]``
    (``[tokens]``) int32, or ``pos_offset [seqs]`` + token.  ``out`` may have any strides (``k_rope.transpose(1, 2)`` of a
    ``[seqs, heads, tokens, d]`` array), be of the other storage type, or be ``x``.  ``transposed`` turns back (the gradient)."""
    dev = x.device
    cx = _heads(x, "x")
    if positions is not None:
        _want(positions, "positions", torch.int32, x.shape[:-2], dev)
    if pos_offset is not None:
        _want(pos_offset, "pos_offset", torch.int32, (cx.n_seqs,), dev)
    if x.shape[-1] != rope.head_dim or (out is not None and out.shape != x.shape):
        raise ValueError(f"x must have heads of {rope.head_dim}, and out its shape")
    if rope.inv_freq is not None and rope.inv_freq.device != dev:
        raise ValueError("inv_freq must be on x's device")
    with _Launch(dev, stream) as st:
        if out is None:
            out = torch.empty_like(x, memory_format=torch.contiguous_format)
        cr, co = rope.c_struct(), _heads(out, "out", dev)
        _check(lib().shadowkv_rotate(C.byref(cr), C.byref(cx), C.byref(co), None if positions is None else positions.data_ptr(),
                                     None if pos_offset is None else pos_offset.data_ptr(), 1 if transposed else 0, st))
    return out


class PagedCache:
    """Keys and values in pages: ``k, v [pages, h_kv, page_size, d]`` with any strides (the last 1), ``page_table [batch,
    pages_per_seq]`` int32.  Entries outside ``[0, pages)`` hold no tokens.  Keeps the tensors; copies nothing."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, page_table: torch.Tensor):
        if k.dim() != 4 or v.shape != k.shape or k.dtype != v.dtype or k.dtype not in _DTYPES:
            raise ValueError("k and v must be [pages, h_kv, page_size, d] arrays of one storage type")
        if not k.is_cuda or v.device != k.device or page_table.device != k.device:
            raise ValueError("k, v and page_table must be on one GPU")
        ks, vs = k.stride(), v.stride()
        if ks[3] != 1 or vs[3] != 1:
            raise ValueError("the elements of a head must be contiguous")
        if page_table.dim() != 2 or page_table.dtype != torch.int32 or (page_table.shape[1] > 1 and page_table.stride(1) != 1):
            raise ValueError("page_table must be int32 [batch, pages_per_seq] with contiguous rows")
        n, h, ps, d = k.shape
        self.k, self.v, self.page_table, self.device = k, v, page_table, k.device
        self.batch = page_table.shape[0]
        self.c = CPagedCache(k.data_ptr(), v.data_ptr(), ks[0], ks[1], ks[2], vs[0], vs[1], vs[2], page_table.data_ptr(),
                             page_table.stride(0), self.batch, page_table.shape[1], n, h, d, ps, _DTYPES[k.dtype], 0)
        self.address, self.n_pages, self.page_size = C.addressof(self.c), n, ps
        self._copyable = False                            # whether ``_check_copyable`` has accepted it

    def _check_copyable(self) -> None:
        """Raises what ``pages_copy`` inside this cache would."""
        one, none = (C.c_void_p * 1)(self.address), CPageMoves()
        _check(lib().shadowkv_pages_copy(one, one, 1, C.byref(none), None))
        self._copyable = True


def dense_pages(k: torch.Tensor, v: torch.Tensor, page_size: int) -> PagedCache:
    """A ``PagedCache`` on dense arrays ``k, v [b, h_kv, cap, d]`` (the value store, the keys of ``build_landmarks``): what is appended
    there lies where those calls expect it.  ``page_size`` must divide ``cap``."""
    if k.dim() != 4 or k.shape != v.shape or not k.is_contiguous() or not v.is_contiguous():
        raise ValueError("k and v must be contiguous [b, h_kv, cap, d] arrays of one shape")
    b, h, cap, d = k.shape
    if b == 0 or page_size < 1 or cap % page_size:
        raise ValueError(f"page_size {page_size} must divide the {cap} tokens of the arrays")
    each = cap // page_size
    shape, stride = ((b - 1) * h * each + each, h, page_size, d), (page_size * d, cap * d, d, 1)
    table = (torch.arange(b, device=k.device)[:, None] * (h * each) + torch.arange(each, device=k.device)).to(torch.int32)
    return PagedCache(k.as_strided(shape, stride), v.as_strided(shape, stride), table)


def _runs(cache: PagedCache, kv_lens, seq_starts):
    _want(kv_lens, "kv_lens", torch.int32, (cache.batch,), cache.device)
    if seq_starts is not None:
        _want(seq_starts, "seq_starts", torch.int32, (cache.batch + 1,), cache.device)
    return None if seq_starts is None else seq_starts.data_ptr(), kv_lens.data_ptr()


def paged_append(cache: PagedCache, k: torch.Tensor, v: torch.Tensor, kv_lens: torch.Tensor, seq_starts: Optional[torch.Tensor] = None,
                 rope: Optional[Rope] = None, q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                 pos_offset: Optional[torch.Tensor] = None, stream=None) -> Optional[torch.Tensor]:
    """Appends ``k, v [tokens, h_kv, d]`` to their sequences' pages, with ``rope`` the keys rotated on the way; ``q [tokens, h_q,
    d]``, if given, is rotated beside them and returned (in ``q_out``, which may be ``q``).  Tokens ``seq_starts[i] ..
    seq_starts[i+1]`` are sequence i's last ones of ``kv_lens[i]``; without ``seq_starts`` every sequence has as many."""
    dev = cache.device
    starts, lens = _runs(cache, kv_lens, seq_starts)
    if k.dim() != 3 or v.dim() != 3 or k.shape[-1] != cache.c.head_dim or v.shape[-1] != cache.c.head_dim:
        raise ValueError(f"k and v must be [tokens, h_kv, {cache.c.head_dim}]")
    if q is not None and (q.dim() != 3 or q.shape[-1] != cache.c.head_dim or (q_out is not None and q_out.shape != q.shape)):
        raise ValueError(f"q must be [tokens, h_q, {cache.c.head_dim}], and q_out of its shape")
    if q is None and q_out is not None:
        raise ValueError("q_out is given without q")
    if pos_offset is not None:
        _want(pos_offset, "pos_offset", torch.int32, (cache.batch,), dev)
    if rope is not None and rope.inv_freq is not None and rope.inv_freq.device != dev:
        raise ValueError("inv_freq must be on the cache's device")
    with _Launch(dev, stream) as st:
        if q is not None and q_out is None:
            q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
        ck, cv = _heads(k, "k", dev), _heads(v, "v", dev)
        cq = C.byref(_heads(q, "q", dev)) if q is not None else None
        co = C.byref(_heads(q_out, "q_out", dev)) if q is not None else None
        cr = C.byref(rope.c_struct()) if rope is not None else None
        _check(lib().shadowkv_paged_append(C.byref(cache.c), cr, C.byref(ck), C.byref(cv), cq, co, starts, lens,
                                           None if pos_offset is None else pos_offset.data_ptr(), st))
    return q_out


def paged_attention_workspace_bytes(cache: PagedCache, n_q_heads: int, n_tokens: int) -> int:
    return int(lib().shadowkv_paged_attention_workspace_bytes(C.byref(cache.c), n_q_heads, n_tokens))


def paged_attention(cache: PagedCache, q: torch.Tensor, kv_lens: torch.Tensor, seq_starts: Optional[torch.Tensor] = None,
                    causal: bool = True, softmax_scale: float = 0.0, out: Optional[torch.Tensor] = None,
                    lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Attention of new tokens ``q [tokens, h_q, d]`` (after their rotation) over the pages, which hold their keys and values already.
    Runs as in ``paged_append``.  Returns ``out`` (bf16, ``q``'s shape); ``lse [tokens, h_q]`` float32 is filled if given."""
    dev = cache.device
    starts, lens = _runs(cache, kv_lens, seq_starts)
    if q.dim() != 3 or q.shape[-1] != cache.c.head_dim or (out is not None and out.shape != q.shape):
        raise ValueError(f"q must be [tokens, h_q, {cache.c.head_dim}], and out of its shape")
    if lse is not None:
        _want(lse, "lse", torch.float32, q.shape[:2], dev)
    with _Launch(dev, stream) as st:
        if out is None:
            out = torch.empty_like(q, dtype=torch.bfloat16, memory_format=torch.contiguous_format)
        if workspace is None:
            workspace = alloc_workspace(paged_attention_workspace_bytes(cache, q.shape[1], q.shape[0]), dev)
        elif workspace.device != dev or not workspace.is_contiguous():
            raise ValueError(f"workspace must be a contiguous tensor on {dev}")
        cq, co = _heads(q, "q", dev), _heads(out, "out", dev)
        _check(lib().shadowkv_paged_attention(C.byref(cache.c), C.byref(cq), C.byref(co), None if lse is None else lse.data_ptr(), starts, lens,
                                              1 if causal else 0, float(softmax_scale), workspace.data_ptr(),
                                              workspace.numel() * workspace.element_size(), st))
    return out


# ---- a search over several continuations: the choice over beams and vocabulary, and the state that follows it ----

_INT32 = 2 ** 31 - 1       # (ctypes cuts longer numbers off without a word)
_LOGITS = {torch.bfloat16: LOGITS_BF16, torch.float16: LOGITS_FP16, torch.float32: LOGITS_FP32}


def beam_select(logits: torch.Tensor, scores: torch.Tensor, n_out: int = 0, finished: Optional[torch.Tensor] = None,
                lengths: Optional[torch.Tensor] = None, length_penalty: float = 0.0, logit_scale: float = 0.0, end_token: int = -1,
                out: Optional[dict] = None, workspace: Optional[torch.Tensor] = None, stream=None) -> dict:
    """The ``n_out`` (0: as many as beams) best continuations of every group from ``logits [groups, beams, vocab]`` (bf16, fp16 or
    fp32; strides of groups and beams as they come) and the beams' summed log-probabilities ``scores [groups, beams]`` float32.
    ``finished`` (bool) beams offer themselves; ranks are scores over (``lengths`` int32 + 1) ** ``length_penalty``.

    Returns ``scores``, ``parents`` (rows ``group * beams + beam``; -1: nothing was left) and ``tokens [groups, n_out]`` in descending
    order of rank; with ``finished`` or an ``end_token`` also ``finished``, with ``lengths`` also ``lengths``.  ``out`` may be such a
    dict, whose scores, finished and lengths may be the arguments themselves where ``n_out`` is ``beams``."""
    if logits.dim() != 3 or logits.dtype not in _LOGITS or not logits.is_cuda:
        raise ValueError("logits must be a bfloat16, float16 or float32 tensor [groups, beams, vocab] on the GPU")
    (groups, beams, vocab), (sg, sb, sv) = logits.shape, logits.stride()
    if vocab > 1 and sv != 1:
        raise ValueError("the logits of a beam must be contiguous")
    dev, n, rows = logits.device, n_out or beams, (groups, beams)
    _want(scores, "scores", torch.float32, rows, dev)
    kinds = [("scores", torch.float32), ("parents", torch.int32), ("tokens", torch.int32)]
    if finished is not None:
        _want(finished, "finished", torch.bool, rows, dev)
    if finished is not None or end_token >= 0:
        kinds.append(("finished", torch.bool))
    if lengths is not None:
        _want(lengths, "lengths", torch.int32, rows, dev)
        kinds.append(("lengths", torch.int32))
    if vocab > _INT32 or groups > _INT32 or abs(end_token) > _INT32:
        raise ValueError("sizes and end_token must fit 32 bits")
    c = C.byref(CLogits(logits.data_ptr(), sg, sb, groups, beams, vocab, _LOGITS[logits.dtype]))
    L = lib()
    need = L.shadowkv_beam_select_workspace_bytes(c, n if 0 < n <= 64 else 0)
    if need == 0:
        raise ShadowKVError(EINVAL, last_error())
    with _launch(dev, stream) as st:
        if out is None:
            whole = torch.empty((3 if lengths is None else 4, groups, n), dtype=torch.int32, device=dev).unbind(0)   # (one allocation)
            out = {"scores": whole[0].view(torch.float32), "parents": whole[1], "tokens": whole[2]}
            if lengths is not None:
                out["lengths"] = whole[3]
            if len(kinds) > len(out):
                out["finished"] = torch.empty((groups, n), dtype=torch.bool, device=dev)
        else:
            if out.keys() != dict(kinds).keys():
                raise ValueError(f"out must have {', '.join(k for k, _ in kinds)}")
            for name, kind in kinds:
                _want(out[name], name, kind, (groups, n), dev)
        if workspace is None:
            workspace, room = torch.empty(need, dtype=torch.uint8, device=dev), need
        elif workspace.device != dev or not workspace.is_contiguous():
            raise ValueError(f"workspace must be a contiguous tensor on {dev}")
        else:
            room = workspace.numel() * workspace.element_size()
        f, l = out.get("finished"), out.get("lengths")
        _check(L.shadowkv_beam_select(
            c, scores.data_ptr(), None if finished is None else finished.data_ptr(), None if lengths is None else lengths.data_ptr(),
            length_penalty, logit_scale, end_token, n, out["scores"].data_ptr(), out["parents"].data_ptr(), out["tokens"].data_ptr(),
            None if f is None else f.data_ptr(), None if l is None else l.data_ptr(), workspace.data_ptr(), room, st))
    return out


def _rows(t: torch.Tensor, n: int, device) -> tuple:
    """[rows, ...] as the fields of ``shadowkv_rows``: what follows the rows has to be pieces of contiguous elements at one stride."""
    shape = t.shape
    if not shape or shape[0] != n:
        raise ValueError(f"an array must have {n} rows, not shape {tuple(shape)}")
    if t.device != device:
        raise ValueError(f"an array must be on {device}, not {t.device}")
    if t.is_contiguous():
        each = t.nbytes // n if n else 0
        return t.data_ptr(), each, 0, each, 1
    stride, eb, inner, outer, step = t.stride(), t.element_size(), 1, 1, 0
    dims = [(s, d) for s, d in zip(shape[1:], stride[1:]) if s != 1]
    while dims and dims[-1][1] == inner:
        inner *= dims.pop()[0]
    if dims:
        outer, step = dims.pop()
    while dims and dims[-1][1] == outer * step:
        outer *= dims.pop()[0]
    if dims:
        raise ValueError(f"rows of shape {tuple(shape[1:])} and strides {stride[1:]} are not pieces at one stride")
    return t.data_ptr(), stride[0] * eb, step * eb, inner * eb, outer


def reorder_rows(arrays, parents: torch.Tensor, stream=None) -> None:
    """Row i of every tensor of ``arrays`` (one tensor or several, ``[rows, ...]`` of any types; views such as ``A[:, prompt:]`` or
    ``k[:, :, -32:]`` too) becomes what row ``parents[i]`` was, in place.  ``parents`` int32, as many as rows (``[groups, beams]`` of
    ``beam_select``, say); rows with a parent outside stay as they are.  The tensors are on the GPU: values in pinned memory cannot follow."""
    arrays = [arrays] if isinstance(arrays, torch.Tensor) else arrays
    n, dev = parents.numel(), parents.device
    _want(parents, "parents", torch.int32, parents.shape)
    fields = []
    for t in arrays:
        fields += _rows(t, n, dev)
    rows = (C.c_int64 * max(len(fields), 1))(*fields)        # five to an array; the upper half of the last is `reserved`
    with _launch(dev, stream) as st:
        _check(lib().shadowkv_reorder_rows(rows, len(fields) // 5, parents.data_ptr(), n, st))


def _pages_copy(caches, to, moves, st) -> None:
    ptrs = C.c_void_p * max(len(caches), 1)
    frm = ptrs(*[c.address for c in caches])
    _check(lib().shadowkv_pages_copy(frm, frm if to is caches else ptrs(*[c.address for c in to]), len(caches), moves, st))


def pages_copy(caches, src: torch.Tensor, dst: torch.Tensor, rows: Optional[torch.Tensor] = None, to=None, stream=None) -> None:
    """Pages ``src [n]`` int32 of every cache of ``caches`` (one for each layer) to pages ``dst [n]`` of the same cache, or of its
    counterpart in ``to``; with ``rows [n]`` int32 only the first so many tokens of each.  Numbers outside a cache are left out; no page may
    be written twice, or be read and written."""
    caches = [caches] if isinstance(caches, PagedCache) else list(caches)
    to = caches if to is None else [to] if isinstance(to, PagedCache) else list(to)
    if len(to) != len(caches):
        raise ValueError(f"{len(caches)} caches go to {len(to)}")
    dev = src.device
    _want(src, "src", torch.int32, (src.numel(),))
    _want(dst, "dst", torch.int32, src.shape, dev)
    if rows is not None:
        _want(rows, "rows", torch.int32, src.shape, dev)
    if src.numel() > _INT32:
        raise ValueError("more than 2^31 - 1 pages")
    if any(c.device != dev for c in caches) or any(c.device != dev for c in to):
        raise ValueError(f"the caches must be on {dev}")
    with _launch(dev, stream) as st:
        _pages_copy(caches, to, C.byref(CPageMoves(src.data_ptr(), dst.data_ptr(), None if rows is None else rows.data_ptr(), None, src.numel(), 0)), st)


class PagePool:
    """Who holds which page of ``n_pages``: ``page_table [batch, pages_per_seq]`` int32 (-1: no page), ``kv_lens [batch]`` int32 and
    ``page_refs [n_pages]`` int32 (holders; 0: free), empty at first.  The caches of all layers share the table (``cache``).  A caller who
    keeps pages for later adds to ``page_refs``, and subtracts when they are done with.

    ``move_src``, ``move_dst``, ``move_rows`` and ``move_count`` are the copies that the last call asked for; the caches that it was given
    have been copied."""

    def __init__(self, batch: int, pages_per_seq: int, n_pages: int, page_size: int, device="cuda"):
        if max(batch, pages_per_seq, n_pages, page_size) > _INT32:
            raise ValueError("sizes must fit 32 bits")
        c = CPagePool(None, pages_per_seq, None, None, batch, pages_per_seq, n_pages, page_size)
        need = int(lib().shadowkv_pages_workspace_bytes(C.byref(c)))
        if need == 0:
            raise ShadowKVError(EINVAL, last_error())
        self.batch, self.pages_per_seq, self.n_pages, self.page_size = batch, pages_per_seq, n_pages, page_size
        ints = lambda n: torch.zeros(n, dtype=torch.int32, device=device)  # noqa: E731
        self.page_table = torch.full((batch, pages_per_seq), -1, dtype=torch.int32, device=device)
        self.kv_lens, self.page_refs = ints(batch), ints(n_pages)
        self.device = self.page_table.device
        room = max(batch, n_pages // 2 + 1)
        self.move_src, self.move_dst, self.move_rows, self.move_count, self.n_used = ints(room), ints(room), ints(room), ints(1), ints(1)
        self.workspace = alloc_workspace(need, self.device)
        c.page_table, c.kv_lens, c.page_refs = self.page_table.data_ptr(), self.kv_lens.data_ptr(), self.page_refs.data_ptr()
        moves = [CPageMoves(self.move_src.data_ptr(), self.move_dst.data_ptr(), self.move_rows.data_ptr(), self.move_count.data_ptr(), most, 0)
                 for most in (batch, room)]
        self._c, self._update_moves, self._compact_moves = C.byref(c), C.byref(moves[0]), C.byref(moves[1])

    def cache(self, k: torch.Tensor, v: torch.Tensor) -> PagedCache:
        """``PagedCache`` of a layer's pages ``k, v [n_pages, h_kv, page_size, d]`` under this pool's table."""
        if k.dim() != 4 or k.shape[0] != self.n_pages or k.shape[2] != self.page_size:
            raise ValueError(f"k and v must be [{self.n_pages}, h_kv, {self.page_size}, d]")
        return PagedCache(k, v, self.page_table)

    def _layers(self, caches) -> list:
        caches = [caches] if isinstance(caches, PagedCache) else list(caches)
        for c in caches:
            if c.page_size != self.page_size or c.n_pages < self.n_pages or c.device != self.device:
                raise ValueError(f"a cache must have {self.n_pages} pages of {self.page_size} tokens on {self.device}")
            if not c._copyable:                           # (before anything of the pool has changed)
                c._check_copyable()
        if len(caches) > 4096:
            raise ValueError("more than 4096 caches")
        return caches

    def update(self, parents: Optional[torch.Tensor] = None, keep_lens: Optional[torch.Tensor] = None, n_new=0, caches=(), stream=None) -> None:
        """Row i becomes the first ``min(kv_lens[parents[i]], keep_lens[i])`` tokens of what row ``parents[i]`` was (empty where that is
        outside the batch), with room for ``n_new`` (a whole number, or int32 ``[batch]``) further ones, which ``kv_lens`` then counts, as
        ``paged_append`` wants it; a row that the pages do not suffice for gets none.  Copies, in every cache of ``caches``, the last pages that
        rows share and are about to write.  Nothing has changed where a call is refused."""
        each = isinstance(n_new, torch.Tensor)
        if not each and not (0 <= n_new <= _INT32 and n_new == int(n_new)):
            raise ValueError(f"n_new must be a whole number in [0, 2^31), not {n_new}")
        for name, t in (("parents", parents), ("keep_lens", keep_lens), ("n_new", n_new if each else None)):
            if t is not None:
                if t.numel() != self.batch:
                    raise ValueError(f"{name} must have {self.batch} elements, not {t.numel()}")
                _want(t, name, torch.int32, t.shape, self.device)
        caches = self._layers(caches)
        with _launch(self.device, stream) as st:
            _check(lib().shadowkv_pages_update(self._c, None if parents is None else parents.data_ptr(),
                                               None if keep_lens is None else keep_lens.data_ptr(), n_new.data_ptr() if each else None,
                                               0 if each else int(n_new), self._update_moves, self.workspace.data_ptr(), self.workspace.numel(), st))
            if caches:
                _pages_copy(caches, caches, self._update_moves, st)

    def compact(self, max_moves: Optional[int] = None, caches=(), stream=None) -> torch.Tensor:
        """Moves the highest used pages into the lowest free ones (at most ``max_moves``), in every cache of ``caches``.  Returns ``n_used [1]``
        int32 on the device: all pages from there on are free."""
        room, caches = self.move_src.numel(), self._layers(caches)
        if max_moves is not None and not (0 <= max_moves <= _INT32 and max_moves == int(max_moves)):
            raise ValueError(f"max_moves must be a whole number in [0, 2^31), not {max_moves}")
        with _launch(self.device, stream) as st:
            _check(lib().shadowkv_pages_compact(self._c, room if max_moves is None else int(max_moves), self._compact_moves, self.n_used.data_ptr(),
                                                self.workspace.data_ptr(), self.workspace.numel(), st))
            if caches:
                _pages_copy(caches, caches, self._compact_moves, st)
        return self.n_used
