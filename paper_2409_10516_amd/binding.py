"""Thin ctypes binding over libra.so (the C ABI in include/ra.h).

Argument marshalling only: every function takes torch tensors that already live on the
GPU, checks dtype/contiguity, passes raw pointers and sizes, and returns the tensors the
library filled. No step of the method is computed here, and there is no CPU fallback:
if the library is missing, loading fails with an error.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import functools
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# RA_LIBRARY names another build of the same library (a tuning build, say); default: the in-tree one
LIB_PATH = os.environ.get("RA_LIBRARY") or os.path.join(_HERE, "libra.so")
CALLS_PATH = os.path.join(_HERE, "_calls.so")

RA_F32, RA_BF16 = 0, 1
RA_CFG_HELPERS, RA_CFG_HELPER_SPIN, RA_CFG_SEEDS, RA_CFG_SEED_SHARES = 0, 1, 2, 3
RA_HELPERS_OFF, RA_HELPERS_ON = 0, 1
# test-only settings (ra_test_configure)
RA_TEST_KNN_SELECTION, RA_TEST_HELPERS_SILENT, RA_TEST_KNN_RESUME = 100, 101, 102
RA_TEST_KNN_RESUME_INTS = 65536
RA_TEST_KNN_AUTO, RA_TEST_KNN_FILTER, RA_TEST_KNN_LDS = 0, 1, 2
BUILD_POOLED_BYTES = 4 << 30        # largest scratch memory of a build stage that comes from torch's allocator
RA_ENOMEM = 4
STATUS = {0: "RA_OK", 1: "RA_EINVAL", 2: "RA_ESHAPE", 3: "RA_EDTYPE", 4: "RA_ENOMEM",
          5: "RA_EHIP", 6: "RA_EUNSUP"}


class RaError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS.get(status, status)}: {message}")
        self.status = status


class _PagedCache(C.Structure):
    """ra_paged_cache"""
    _fields_ = [("K", C.c_void_p), ("V", C.c_void_p), ("table", C.c_void_p), ("table_stride", C.c_int64), ("dt", C.c_int32), ("n_seq", C.c_int32),
                ("n_kv_heads", C.c_int32), ("n_pages", C.c_int32), ("page", C.c_int32), ("table_pages", C.c_int32)]


_lib = None


def lib() -> C.CDLL:
    """Load libra.so (once). Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: run `python -c 'import __graft_entry__ as g; "
                           f"g.build()'` (or python paper_2409_10516_amd/build.py) first")
    L = C.CDLL(LIB_PATH)
    vp, i32, i64 = C.c_void_p, C.c_int, C.c_int64
    L.ra_last_error.restype = C.c_char_p
    L.ra_version.restype = C.c_char_p
    L.ra_knn.argtypes = [vp, vp, i32, i32, i32, i32, i64, i64, i32, i32, vp, vp]
    L.ra_project.argtypes = [vp, i32, i64, i64, i32, i32, vp, vp, vp]
    L.ra_build_index.argtypes = [vp, vp, i32, i32, i32, i32, i64, i64, i32, i32, i32, vp,
                                 C.POINTER(vp)]
    L.ra_knn_ws.argtypes = [vp, vp, i32, i32, i32, i32, i64, i64, i32, i32, vp, C.c_size_t, vp, vp]
    L.ra_knn_ws.restype = i32
    L.ra_knn_scratch_bytes.argtypes = [i32, i32, i32, i32, i64, i64, i32, i32]
    L.ra_knn_scratch_bytes.restype = C.c_size_t
    L.ra_project_ws.argtypes = [vp, i32, i64, i64, i32, i32, vp, C.c_size_t, vp, vp, vp]
    L.ra_project_ws.restype = i32
    L.ra_project_scratch_bytes.argtypes = [i32, i64, i64, i32, i32]
    L.ra_project_scratch_bytes.restype = C.c_size_t
    L.ra_build_index_ws.argtypes = [vp, vp, i32, i32, i32, i32, i64, i64, i32, i32, i32, vp, C.c_size_t, vp,
                                    C.POINTER(vp)]
    L.ra_build_index_ws.restype = i32
    L.ra_build_workspace_bytes.argtypes = [i32, i32, i32, i32, i64, i64, i32, i32, i32]
    L.ra_build_workspace_bytes.restype = C.c_size_t
    L.ra_search.argtypes = [vp, vp, vp, i32, i64, i32, i32, i32, i32, i32, vp, vp, vp]
    L.ra_quantize_keys.argtypes = [vp, i32, i32, i32, i64, vp, vp, vp]
    L.ra_quantize_keys.restype = i32
    L.ra_search_q8.argtypes = [vp, vp, vp, vp, i32, i64, i32, i32, i32, i32, i32, vp, vp, vp]
    L.ra_search_q8.restype = i32
    L.ra_decode_step_q8.argtypes = [vp, vp, vp, vp, i32, vp, vp, i64, i32, i32, i32, i32, i32, vp, vp, vp,
                                    vp, vp]
    L.ra_decode_step_q8.restype = i32
    L.ra_rerank.argtypes = [vp, vp, i32, i32, i32, i32, i64, i32, vp, i32, i32, vp, vp]
    L.ra_rerank.restype = i32
    L.ra_attend.argtypes = [vp, vp, vp, vp, i32, i64, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp]
    L.ra_attend_noalloc.argtypes = [vp, vp, vp, vp, i32, i64, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp]
    L.ra_decode_step.argtypes = [vp, vp, vp, vp, i32, i64, i32, i32, i32, i32, i32, vp, vp, vp,
                                 vp, vp]
    L.ra_decode_step_grown.argtypes = [vp, vp, vp, vp, i32, i64, i64, i32, i32, i32, i32, i32, vp, vp,
                                       vp, vp, vp]
    L.ra_decode_step_grown.restype = i32
    L.ra_decode_step_budgets.argtypes = [vp, vp, vp, vp, i32, i64, i32, i32, i32, vp, i32, i32, vp, vp,
                                         vp, vp, vp]
    L.ra_decode_step_budgets.restype = i32
    L.ra_index_import.argtypes = [vp, vp, i32, i32, i32, i64, i32, C.POINTER(vp)]
    L.ra_index_export.argtypes = [vp, i32, i32, vp, vp]
    L.ra_index_info.argtypes = [vp, i32]
    L.ra_index_info.restype = i64
    L.ra_index_configure.argtypes = [vp, i32, i64]
    L.ra_index_configure.restype = i32
    L.ra_test_configure.argtypes = [vp, i32, i64]
    L.ra_test_configure.restype = i32
    L.ra_index_adj.argtypes = [vp]
    L.ra_index_adj.restype = vp
    L.ra_index_entry.argtypes = [vp]
    L.ra_index_entry.restype = vp
    L.ra_index_free.argtypes = [vp]
    L.ra_index_free.restype = None
    L.ra_flat_workspace_bytes.argtypes = [i32, i32, i64]
    L.ra_flat_workspace_bytes.restype = C.c_size_t
    L.ra_flat_topk.argtypes = [vp, vp, i32, i32, i32, i32, i64, i32, i32, i32, i32, vp, C.c_size_t, vp, vp]
    L.ra_flat_topk.restype = i32
    L.ra_full_attention_workspace_bytes.argtypes = [i32, i32, i32, i64]
    L.ra_full_attention_workspace_bytes.restype = C.c_size_t
    L.ra_hbm_read_probe.argtypes = [vp, C.c_size_t, vp, vp]
    L.ra_hbm_gather_probe.argtypes = [vp, C.c_size_t, C.c_size_t, C.c_uint32, vp, vp]
    L.ra_full_attention.argtypes = [vp, vp, vp, i32, i32, i32, i32, i64, i32, vp, C.c_size_t, vp, vp, vp]
    L.ra_full_attention.restype = i32
    L.ra_append_tokens.argtypes = [vp, vp, vp, i32, i32, i32, i32, i64, i32, i64, i64, i64, vp, vp, C.c_double, vp, i32, i32, vp, vp,
                                   i64, i64, vp, vp, vp, vp, vp, vp, vp, vp]
    L.ra_append_tokens.restype = i32
    L.ra_quantize_kv4.argtypes = [vp, i32, i32, i32, i64, i32, vp, vp, i64, vp, vp, vp]
    L.ra_quantize_kv4.restype = i32
    L.ra_dequantize_kv4.argtypes = [vp, vp, i32, i32, i32, i64, i32, vp, i64, vp, vp]
    L.ra_dequantize_kv4.restype = i32
    L.ra_full_attention_q4_workspace_bytes.argtypes = [i32, i32, i32, i32, i64]
    L.ra_full_attention_q4_workspace_bytes.restype = C.c_size_t
    L.ra_full_attention_q4.argtypes = [vp, i32, vp, vp, vp, vp, i32, i32, i32, i64, i64, i32, vp, vp, C.c_size_t, vp, vp, vp]
    L.ra_full_attention_q4.restype = i32
    L.ra_attend_q4.argtypes = [vp, vp, i32, vp, vp, vp, vp, i64, i64, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp]
    L.ra_attend_q4.restype = i32
    cache = C.POINTER(_PagedCache)
    L.ra_append_tokens_paged.argtypes = [vp, vp, vp, cache, i32, i64, i32, i64, i64, i64, vp, vp, C.c_double, vp, i32, i32, C.c_double, vp, vp, vp, vp]
    L.ra_append_tokens_paged.restype = i32
    L.ra_gather_paged.argtypes = [cache, i32, i64, i32, vp, vp, vp]
    L.ra_gather_paged.restype = i32
    L.ra_full_attention_paged_workspace_bytes.argtypes = [i32, i32, i32, i32, i64]
    L.ra_full_attention_paged_workspace_bytes.restype = C.c_size_t
    L.ra_full_attention_paged.argtypes = [vp, cache, i32, i64, i32, vp, vp, C.c_size_t, vp, vp, vp]
    L.ra_full_attention_paged.restype = i32
    L.ra_attend_paged_workspace_bytes.argtypes = [i32, i32, i32, i32, i64, i32, i32, i32]
    L.ra_attend_paged_workspace_bytes.restype = C.c_size_t
    L.ra_attend_paged.argtypes = [vp, cache, i32, i64, i32, vp, vp, i32, i32, i32, vp, vp, C.c_size_t, vp, vp, vp, vp, vp, vp, vp]
    L.ra_attend_paged.restype = i32
    for name in ("ra_knn", "ra_project", "ra_build_index", "ra_search", "ra_attend",
                 "ra_attend_noalloc", "ra_hbm_read_probe", "ra_hbm_gather_probe", "ra_decode_step", "ra_index_import",
                 "ra_index_export"):
        getattr(L, name).restype = i32
    _lib = L
    return L


def _check(rc: int):
    if rc != 0:
        raise RaError(rc, lib().ra_last_error().decode())


def _room(fn, *args) -> int:
    """fn(*args) -> status, for a call that may allocate: again without the pieces that torch keeps, where the device has no
    room (a build leaves one of up to BUILD_POOLED_BYTES)."""
    rc = fn(*args)
    if rc == RA_ENOMEM:
        torch.cuda.empty_cache()
        rc = fn(*args)
    return rc


def _dt(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return RA_F32
    if t.dtype == torch.bfloat16:
        return RA_BF16
    raise TypeError(f"dtype {t.dtype} is not supported (float32 or bfloat16)")


def _dev(*ts):
    for t in ts:
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError("tensors must live on the GPU")
        if not t.is_contiguous():
            raise ValueError("tensors must be contiguous")


# (ctypes turns plain integers into the pointers of the argtypes: no wrapper objects on the call path)
def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


_RAW = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    """The stream's handle; by default the current device's current stream. torch's own accessor of the
    raw handle is used where it exists: building a Stream object costs as much as the rest of a call."""
    if stream is not None:
        return stream.cuda_stream
    return torch.cuda.current_stream().cuda_stream if _RAW is None else _RAW(torch.cuda.current_device())


# The calls around a 4-bit cache take many tensors and are made once per token and layer: their checks read every attribute once
# and build nothing (us: a tensor's attribute 0.05, a shape 0.1, the C entry's checks 0.6, a launch 3.4, a tensor made of sizes given one by
# one 1.3, as a tuple 1.7).
def _here(*ts):
    """The given tensors live on the current device, where the call is launched -> its index."""
    here = torch.cuda.current_device()
    for t in ts:
        if t is not None and t.get_device() != here:
            raise ValueError(f"tensors must live on the current GPU ({here}), not on {t.device}")
    return here


def _handle(stream, here: int) -> int:
    """_stream, where the current device is known."""
    return _stream(stream) if stream is not None or _RAW is None else _RAW(here)


_CURRENT = contextlib.nullcontext()


def _for(stream, here: int):
    """Where a call on `stream` allocates: there, or what it drops at its end (a workspace) would be another stream's while the
    call still runs, and zeroes could come after its results."""
    if stream is None:
        return _CURRENT
    if stream.device_index != here:
        raise ValueError(f"stream must be one of the current GPU ({here})")
    return torch.cuda.stream(stream)


def _vector(t: torch.Tensor, n: int, dtype, here: int, name: str) -> int:
    """The address of a vector of n elements."""
    if t.dtype is not dtype or t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor [{n}]")
    if t.get_device() != here:
        raise ValueError(f"{name} must live on the current GPU ({here}), not on {t.device}")
    return t.data_ptr()


def _token_rows(t: torch.Tensor, n_seq: int, T: int, dtype, here: int):
    """Heads of tokens [n_seq][T][heads][128] -> (address, heads, elements from token to token)."""
    shape = t.shape
    if len(shape) != 4 or shape[0] != n_seq or shape[1] != T or shape[3] != 128:
        raise ValueError("q, k and v must be [n_seq][T][heads][128]")
    if t.dtype is not dtype:
        raise TypeError("q, k and v must share a dtype")
    if t.get_device() != here:
        raise ValueError(f"tensors must live on the current GPU ({here}), not on {t.device}")
    seq, token, head, one = t.stride()
    heads = shape[2]
    # (the stride of a dimension of one element says nothing)
    row = token if T > 1 else seq if n_seq > 1 else heads * 128
    if one != 1 or (heads > 1 and head != 128) or (n_seq > 1 and seq != T * row):
        raise ValueError("the heads of a token must lie side by side, and all tokens equally far apart")
    return t.data_ptr(), heads, row


def _cache_rows(t: torch.Tensor, n_seq: int, n_kv: int, dtype, here: int, room: int):
    """A cache [n_seq][n_kv][capacity][128] -> (address, capacity); room: the capacity it must have, 0 for any."""
    shape = t.shape
    if t.dtype is not dtype:
        raise TypeError("caches and inputs must share a dtype")
    if len(shape) != 4 or shape != (n_seq, n_kv, room or shape[2], 128) or not t.is_contiguous() or t.get_device() != here:
        raise ValueError("K and V must be contiguous [n_seq][n_kv][capacity][128], of one capacity and where the inputs are")
    return t.data_ptr(), shape[2]


def _kv4(x4, n_seq: int, n_kv: int, name: str, here: int, kv_stride: Optional[int] = None):
    """Checks a cache in 4 bits (codes, scale) -> their addresses and its capacity in rows."""
    codes, scale = x4
    shape = codes.shape
    rows = shape[2] if len(shape) == 4 else -1
    if shape != (n_seq, n_kv, rows, 64) or scale.shape != (n_seq, n_kv, rows, 4):
        raise ValueError(f"{name} must be codes [n_seq][n_kv][capacity][64] and scale [n_seq][n_kv][capacity][4]")
    if codes.dtype is not torch.uint8 or scale.dtype is not torch.uint8:
        raise TypeError(f"{name} must be uint8")
    if not codes.is_contiguous() or not scale.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if codes.get_device() != here or scale.get_device() != here:
        raise ValueError(f"{name} must live on the current GPU ({here}), not on {codes.device} and {scale.device}")
    if kv_stride is not None and rows != kv_stride:
        raise ValueError(f"{name} holds {rows} rows per head, not {kv_stride}")
    return codes.data_ptr(), scale.data_ptr(), rows


class Index:
    """Owns an ra_index handle."""

    def __init__(self, handle: int):
        self._h = C.c_void_p(handle)

    @property
    def handle(self):
        if self._h is None:
            raise RuntimeError("index was freed")
        return self._h

    def info(self, what: int) -> int:
        return int(lib().ra_index_info(self.handle, what))

    n_seq = property(lambda s: s.info(0))
    n_q_heads = property(lambda s: s.info(1))
    n_kv_heads = property(lambda s: s.info(2))
    N = property(lambda s: s.info(3))
    deg = property(lambda s: s.info(4))
    device_bytes = property(lambda s: s.info(5))
    helpers_active = property(lambda s: s.info(6) == 1)
    seed_shares_active = property(lambda s: s.info(8) == 1)
    shared_steps_active = property(lambda s: s.info(9) == 1)
    shared_messages = property(lambda s: s.info(10))
    shared_launches = property(lambda s: s.info(11))

    n_seeds = property(lambda s: s.info(7))

    @functools.cached_property
    def heads(self):
        """(n_seq, n_q_heads, n_kv_heads), which a handle keeps for life."""
        return self.n_seq, self.n_q_heads, self.n_kv_heads

    @functools.cached_property
    def device(self):
        """The index of the GPU it lives on."""
        return self.info(12)

    def configure(self, what: int, value: int) -> None:
        """ra_index_configure: RA_CFG_HELPERS / RA_CFG_HELPER_SPIN / RA_CFG_SEEDS / RA_CFG_SEED_SHARES."""
        _check(_room(lib().ra_index_configure, self.handle, what, value))

    def test_configure(self, what: int, value: int) -> None:
        """ra_test_configure on this handle (test-only settings)."""
        _check(lib().ra_test_configure(self.handle, what, value))

    def free(self):
        if self._h is not None:
            lib().ra_index_free(self._h)
            self._h = None

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass


def ra_test_configure(what: int, value: int) -> None:
    """ra_test_configure without a handle (process-wide test-only settings)."""
    _check(lib().ra_test_configure(None, what, value))


def _with_scratch(stream, need: int, call) -> None:
    """call(workspace, its bytes, stream) -> status, for a call that returns when the stream is done. Up to
    BUILD_POOLED_BYTES of scratch memory, for a call on the current stream, come from torch's allocator, which has the
    piece of the last call at hand and gives it back where torch needs it (or torch.cuda.empty_cache() is called). With the library's
    own allocation and free, 0.3 ms are lost in a build for two prompts of 5K tokens (1.6 ms), and builds with 0.7 GB that
    follow each other every 7 ms wait for the driver most of the time (32 ms each: above some 100 GB a second of freed and
    allocated memory it stops for up to seconds). Where torch finds no room, the library allocates."""
    ws = None
    if stream is None and 0 < need <= BUILD_POOLED_BYTES:
        try:
            ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        except torch.cuda.OutOfMemoryError:
            pass
    rc = call(None, 0, _stream(stream)) if ws is None else call(_ptr(ws), need, _stream(None))
    if rc == RA_ENOMEM:      # pieces that torch keeps, such as an earlier call's, may be what is missing
        del ws
        torch.cuda.empty_cache()
        rc = call(None, 0, _stream(stream))
    _check(rc)


def ra_knn(K, Q_prefill, knn: int, stream=None) -> torch.Tensor:
    _dev(K, Q_prefill)
    n_seq, n_kv, N, d = K.shape
    _, n_q, M, _ = Q_prefill.shape
    L = torch.empty((n_seq, n_q, M, knn), dtype=torch.int32, device=K.device)
    args = (_dt(K), n_seq, n_q, n_kv, N, M, d, knn)
    _with_scratch(stream, lib().ra_knn_scratch_bytes(*args),
                  lambda ws, room, st: lib().ra_knn_ws(_ptr(K), _ptr(Q_prefill), *args, ws, room, st, _ptr(L)))
    return L


def ra_project(L: torch.Tensor, N: int, deg: int, stream=None):
    """L: int32 [n_graphs][M][knn] on the GPU -> (adj [n_graphs][N][deg], entry [n_graphs])."""
    _dev(L)
    if L.dtype != torch.int32:
        raise TypeError("L must be int32")
    n_graphs, M, knn = L.shape
    adj = torch.empty((n_graphs, N, deg), dtype=torch.int32, device=L.device)
    entry = torch.empty((n_graphs,), dtype=torch.int32, device=L.device)
    _with_scratch(stream, lib().ra_project_scratch_bytes(n_graphs, N, M, deg, knn),
                  lambda ws, room, st: lib().ra_project_ws(_ptr(L), n_graphs, N, M, knn, deg, ws, room, st, _ptr(adj), _ptr(entry)))
    return adj, entry


def ra_build_index(K, Q_prefill, deg: int, knn: int, stream=None) -> Index:
    _dev(K, Q_prefill)
    if K.dtype != Q_prefill.dtype:
        raise TypeError("K and Q_prefill must share a dtype")
    n_seq, n_kv, N, d = K.shape
    _, n_q, M, _ = Q_prefill.shape
    h = C.c_void_p()
    args = (_ptr(K), _ptr(Q_prefill), _dt(K), n_seq, n_q, n_kv, N, M, d, deg, knn)
    _with_scratch(stream, lib().ra_build_workspace_bytes(*args[2:]),
                  lambda ws, room, st: lib().ra_build_index_ws(*args, ws, room, st, C.byref(h)))
    return Index(h.value)


def ra_index_import(adj: torch.Tensor, entries: torch.Tensor, n_seq: int, n_q: int,
                    n_kv: int) -> Index:
    """adj: int32 [n_seq*n_q][N][deg] on the HOST; entries: int32 [n_seq*n_q] on the host."""
    adj = adj.to(torch.int32).contiguous().cpu()
    entries = entries.to(torch.int32).contiguous().cpu()
    g, N, deg = adj.shape
    if g != n_seq * n_q or entries.numel() != g:
        raise ValueError("adj/entries do not match n_seq * n_q graphs")
    h = C.c_void_p()
    _check(_room(lib().ra_index_import, _ptr(adj), _ptr(entries), n_seq, n_q, n_kv, N, deg, C.byref(h)))
    return Index(h.value)


def ra_index_export(idx: Index, seq: int, q_head: int):
    adj = torch.empty((idx.N, idx.deg), dtype=torch.int32)
    entry = torch.empty((1,), dtype=torch.int32)
    _check(lib().ra_index_export(idx.handle, seq, q_head, _ptr(adj), _ptr(entry)))
    return adj, int(entry[0])


def _stats_tensor(n_seq, n_q, device):
    return torch.empty((n_seq, n_q, 4), dtype=torch.int32, device=device)     # every walk writes its row


def ra_quantize_keys(K, stream=None):
    """8-bit copy of the keys for the search -> (K8 int8 [n_seq][n_kv][N][128], scale float32
    [n_seq][n_kv][128])."""
    _dev(K)
    n_seq, n_kv, N, d = K.shape
    K8 = torch.empty((n_seq, n_kv, N, d), dtype=torch.int8, device=K.device)
    scale = torch.empty((n_seq, n_kv, d), dtype=torch.float32, device=K.device)
    _check(lib().ra_quantize_keys(_ptr(K), _dt(K), n_seq, n_kv, N, _stream(stream), _ptr(K8), _ptr(scale)))
    return K8, scale


def ra_search(q, idx: Index, K, sink: int, window: int, topk: int, ef: int, expand: int = 1,
              stream=None, with_stats: bool = True, k8=None):
    """-> (ids int32 [n_seq][n_q][topk], stats int32 [n_seq][n_q][4] = visited, expanded,
    iters, returned). With k8 = (K8, scale) from ra_quantize_keys the walk reads the 8-bit keys
    (ra_search_q8) and K may be None."""
    n_seq, n_q, d = q.shape
    ids = torch.empty((n_seq, n_q, topk), dtype=torch.int32, device=q.device)
    st = _stats_tensor(n_seq, n_q, q.device) if with_stats else None
    if k8 is None:
        _dev(q, K)
        _check(_room(lib().ra_search, _ptr(q), idx.handle, _ptr(K), _dt(K), K.shape[2], sink, window, topk,
                     ef, expand, _stream(stream), _ptr(ids), _ptr(st)))
    else:
        K8, scale = k8
        _dev(q, K8, scale)
        _check(_room(lib().ra_search_q8, _ptr(q), idx.handle, _ptr(K8), _ptr(scale), _dt(q), K8.shape[2], sink,
                     window, topk, ef, expand, _stream(stream), _ptr(ids), _ptr(st)))
    return ids, st


def ra_rerank(q, K, cand, topk: int, stream=None):
    """Best topk of the candidate ids [n_seq][n_q][n_cand] under the exact scores <q, K[id]>
    -> ids int32 [n_seq][n_q][topk]."""
    _dev(q, K, cand)
    n_seq, n_q, d = q.shape
    ids = torch.empty((n_seq, n_q, topk), dtype=torch.int32, device=q.device)
    _check(lib().ra_rerank(_ptr(q), _ptr(K), _dt(K), n_seq, n_q, K.shape[1], K.shape[2], d, _ptr(cand),
                           cand.shape[-1], topk, _stream(stream), _ptr(ids)))
    return ids


def ra_attend(q, idx: Index, K, V, sink: int, window: int, ids: torch.Tensor, stream=None,
              partials: bool = False, noalloc: bool = False, out=None, lse=None):
    """-> (out, lse) or, with partials=True, (out, lse, o_omega, lse_omega, o_w, lse_w).
    noalloc=True calls ra_attend_noalloc (pass out and lse in, then nothing is allocated at all)."""
    _dev(q, K, V, ids, out, lse)
    n_seq, n_q, d = q.shape
    topk = ids.shape[-1]
    f = dict(dtype=torch.float32, device=q.device)
    if out is None:
        out = torch.empty((n_seq, n_q, d), **f)
    if lse is None:
        lse = torch.empty((n_seq, n_q), **f)
    extra = [None] * 4
    if partials:
        extra = [torch.empty((n_seq, n_q, d), **f), torch.empty((n_seq, n_q), **f),
                 torch.empty((n_seq, n_q, d), **f), torch.empty((n_seq, n_q), **f)]
    fn = lib().ra_attend_noalloc if noalloc else lib().ra_attend
    _check(_room(fn, _ptr(q), idx.handle, _ptr(K), _ptr(V), _dt(K), K.shape[2], sink, window,
                 topk, _ptr(ids), _stream(stream), _ptr(out), _ptr(lse), *[_ptr(t) for t in extra]))
    return (out, lse, *extra) if partials else (out, lse)


def ra_decode_step(q, idx: Index, K, V, sink: int, window: int, topk: int, ef: int,
                   expand: int = 1, stream=None, out=None, lse=None, ids=None, stats=None,
                   n_tokens: Optional[int] = None, k8=None, topk_per_head=None):
    """One layer's decode-step attention. Output tensors may be passed in to avoid
    allocation; -> (out, lse, ids, stats). With n_tokens given, K/V are caches of capacity
    K.shape[2] rows per head holding n_tokens >= idx.N valid tokens (ra_decode_step_grown). With
    k8 = (K8, scale) from ra_quantize_keys the walk reads the 8-bit keys (ra_decode_step_q8). With
    topk_per_head (device int32 [n_seq][n_q]) every head keeps its own number of ids, at most topk
    (ra_decode_step_budgets)."""
    _dev(q, K, V, out, lse, ids, stats, topk_per_head)
    if topk_per_head is not None and (k8 is not None or n_tokens is not None):
        raise ValueError("topk_per_head goes with neither k8 nor n_tokens")
    n_seq, n_q, d = q.shape
    f = dict(dtype=torch.float32, device=q.device)
    if out is None:
        out = torch.empty((n_seq, n_q, d), **f)
    if lse is None:
        lse = torch.empty((n_seq, n_q), **f)
    if ids is None:
        ids = torch.empty((n_seq, n_q, topk), dtype=torch.int32, device=q.device)
    if stats is None:
        stats = _stats_tensor(n_seq, n_q, q.device)
    if topk_per_head is not None:
        if topk_per_head.dtype != torch.int32 or tuple(topk_per_head.shape) != (n_seq, n_q) \
                or not topk_per_head.is_contiguous():
            raise ValueError("topk_per_head must be a contiguous int32 tensor [n_seq][n_q]")
        _check(_room(lib().ra_decode_step_budgets, _ptr(q), idx.handle, _ptr(K), _ptr(V), _dt(K), K.shape[2], sink,
                     window, topk, _ptr(topk_per_head), ef, expand, _stream(stream),
                     _ptr(out), _ptr(lse), _ptr(ids), _ptr(stats)))
    elif k8 is not None:
        K8, scale = k8
        _dev(K8, scale)
        _check(_room(lib().ra_decode_step_q8, _ptr(q), idx.handle, _ptr(K), _ptr(V), _dt(K), _ptr(K8), _ptr(scale),
                     K.shape[2], sink, window, topk, ef, expand, _stream(stream),
                     _ptr(out), _ptr(lse), _ptr(ids), _ptr(stats)))
    elif n_tokens is None:
        _check(_room(lib().ra_decode_step, _ptr(q), idx.handle, _ptr(K), _ptr(V), _dt(K), K.shape[2], sink,
                     window, topk, ef, expand, _stream(stream), _ptr(out), _ptr(lse),
                     _ptr(ids), _ptr(stats)))
    else:
        _check(_room(lib().ra_decode_step_grown, _ptr(q), idx.handle, _ptr(K), _ptr(V), _dt(K), n_tokens,
                     K.shape[2], sink, window, topk, ef, expand, _stream(stream),
                     _ptr(out), _ptr(lse), _ptr(ids), _ptr(stats)))
    return out, lse, ids, stats


def ra_hbm_read_probe(buf: torch.Tensor, out: torch.Tensor, stream=None) -> None:
    """Stream `buf` (contiguous device tensor) once; xors a fold of it into out (device int64 [1])."""
    _dev(buf, out)
    _check(lib().ra_hbm_read_probe(_ptr(buf), buf.numel() * buf.element_size(), _stream(stream), _ptr(out)))


def ra_hbm_gather_probe(buf: torch.Tensor, n_rows: int, out: torch.Tensor, seed: int = 0, stream=None) -> None:
    """Read n_rows rows of 256 B of `buf` at hashed row numbers; xors a fold into out (device int64 [1])."""
    _dev(buf, out)
    _check(lib().ra_hbm_gather_probe(_ptr(buf), buf.numel() * buf.element_size(), n_rows, seed, _stream(stream),
                                     _ptr(out)))


def ra_flat_topk(q, K, sink: int, window: int, topk: int, stream=None, workspace=None, ids=None):
    """Exact top-k by linear scan for every (sequence, query head) -> ids int32 [n_seq][n_q][topk]."""
    _dev(q, K, workspace, ids)
    n_seq, n_q, d = q.shape
    n_kv, N = K.shape[1], K.shape[2]
    need = lib().ra_flat_workspace_bytes(n_seq, n_q, N)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    if ids is None:
        ids = torch.empty((n_seq, n_q, topk), dtype=torch.int32, device=q.device)
    _check(lib().ra_flat_topk(_ptr(q), _ptr(K), _dt(K), n_seq, n_q, n_kv, N, d, sink, window, topk,
                              _ptr(workspace), workspace.numel(), _stream(stream), _ptr(ids)))
    return ids


def ra_full_attention(q, K, V, stream=None, workspace=None, out=None, lse=None):
    """Eq. 1 over the whole context -> (out float32 [n_seq][n_q][d], lse float32 [n_seq][n_q])."""
    _dev(q, K, V, workspace, out, lse)
    n_seq, n_q, d = q.shape
    n_kv, N = K.shape[1], K.shape[2]
    need = lib().ra_full_attention_workspace_bytes(n_seq, n_q, n_kv, N)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    f = dict(dtype=torch.float32, device=q.device)
    if out is None:
        out = torch.empty((n_seq, n_q, d), **f)
    if lse is None:
        lse = torch.empty((n_seq, n_q), **f)
    _check(lib().ra_full_attention(_ptr(q), _ptr(K), _ptr(V), _dt(K), n_seq, n_q, n_kv, N, d,
                                   _ptr(workspace), workspace.numel(), _stream(stream), _ptr(out),
                                   _ptr(lse)))
    return out, lse


def ra_append_tokens(q, k, v, first, *, n_new=None, q_weight=None, k_weight=None, eps: float = 1e-6, inv_freq=None,
                     interleaved: bool = False, q_out=None, K=None, V=None, k4=None, v4=None, stream=None):
    """The tokens that enter a cache: norm of every query and key head (weight [128], None: no norm), rotation of the first
    2 * len(inv_freq) dimensions at positions first[s] + t, new rows of the caches. q, k, v: [n_seq][T][heads][128] (any may be
    None), the heads of a token side by side, tokens any multiple of 16 bytes apart, so that they may be parts of one buffer; one
    distance for all tokens, from a sequence's last to the next one's first, too (a slice of several tokens of each of several sequences is
    copied first). first, n_new: int32 [n_seq] on the GPU (None: 0, and T). K, V: caches [n_seq][n_kv][capacity][128]; k4, v4: caches in 4 bits, of a
    capacity of their own, (codes, scale) as from ra_quantize_kv4. -> q_out [n_seq][n_q][T][128] (None without q); where tokens are fewer
    than T and no q_out is given, the rows behind the last one are zero."""
    some = q if q is not None else k if k is not None else v
    if some is None:
        raise ValueError("at least one of q, k and v is needed")
    here = torch.cuda.current_device()
    room_for = _for(stream, here)
    dtype, shape = some.dtype, some.shape
    if len(shape) != 4:
        raise ValueError("q, k and v must be [n_seq][T][heads][128]")
    n_seq, T = shape[0], shape[1]
    q_at, n_q, q_row = _token_rows(q, n_seq, T, dtype, here) if q is not None else (None, 0, 0)
    k_at, n_k, k_row = _token_rows(k, n_seq, T, dtype, here) if k is not None else (None, 0, 0)
    v_at, n_v, v_row = _token_rows(v, n_seq, T, dtype, here) if v is not None else (None, 0, 0)
    if n_k and n_v and n_k != n_v:
        raise ValueError("k and v must have the same number of heads")
    n_kv = n_k or n_v or 1
    qw_at = _vector(q_weight, 128, dtype, here, "q_weight") if q_weight is not None else None
    kw_at = _vector(k_weight, 128, dtype, here, "k_weight") if k_weight is not None else None
    f_at, rot = None, 0
    if inv_freq is not None:
        rot = 2 * inv_freq.numel()
        f_at = _vector(inv_freq, rot // 2, torch.float32, here, "inv_freq")
    first_at = _vector(first, n_seq, torch.int32, here, "first") if first is not None else None
    new_at = _vector(n_new, n_seq, torch.int32, here, "n_new") if n_new is not None else None
    K_at = V_at = k4_at = k4s_at = v4_at = v4s_at = None
    room = room4 = 0
    if K is not None:
        K_at, room = _cache_rows(K, n_seq, n_kv, dtype, here, 0)
    if V is not None:
        V_at, room = _cache_rows(V, n_seq, n_kv, dtype, here, room)
    if k4 is not None:
        k4_at, k4s_at, room4 = _kv4(k4, n_seq, n_kv, "k4", here)
    if v4 is not None:
        v4_at, v4s_at, room4 = _kv4(v4, n_seq, n_kv, "v4", here, room4 or None)
    out_at = None
    if q is None:
        if q_out is not None:
            raise ValueError("q_out goes with q")
    else:
        if q_out is None:
            with room_for:
                q_out = (torch.empty if n_new is None else torch.zeros)(n_seq, n_q, T, 128, dtype=dtype, device=here)
        elif q_out.dtype is not dtype or q_out.shape != (n_seq, n_q, T, 128) or not q_out.is_contiguous() or q_out.get_device() != here:
            raise ValueError("q_out must be contiguous [n_seq][n_q][T][128], of the dtype of q and where q is")
        out_at = q_out.data_ptr()
    _check(lib().ra_append_tokens(q_at, k_at, v_at, _dt(some), n_seq, n_q or n_kv, n_kv, T, 128, q_row, k_row, v_row, qw_at, kw_at, eps,
                                  f_at, rot, 1 if interleaved else 0, first_at, new_at, room, room4, _handle(stream, here), out_at, K_at, V_at,
                                  k4_at, k4s_at, v4_at, v4s_at))
    return q_out


def ra_quantize_kv4(X, first=None, n_new=None, out=None, stream=None):
    """Rows [n_seq][n_kv][T][128] into 4 bits -> (codes uint8 [n_seq][n_kv][capacity][64], scale uint8
    [n_seq][n_kv][capacity][4]). With out = (codes, scale) given, row t of sequence s goes to row first[s] + t of these (first: int32
    [n_seq] on the GPU; n_new likewise: only so many rows); without, they are new and hold T rows."""
    _dev(X)
    here = _here(X)
    room_for = _for(stream, here)
    n_seq, n_kv, T, d = X.shape
    if out is None:
        if first is not None or n_new is not None:
            raise ValueError("first and n_new go with out")
        with room_for:
            out = (torch.empty((n_seq, n_kv, T, 64), dtype=torch.uint8, device=here),
                   torch.empty((n_seq, n_kv, T, 4), dtype=torch.uint8, device=here))
    codes, scale, room = _kv4(out, n_seq, n_kv, "out", here)
    _check(lib().ra_quantize_kv4(X.data_ptr(), _dt(X), n_seq, n_kv, T, d, None if first is None else _vector(first, n_seq, torch.int32, here, "first"),
                                 None if n_new is None else _vector(n_new, n_seq, torch.int32, here, "n_new"), room, _handle(stream, here), codes, scale))
    return out


def ra_dequantize_kv4(x4, dtype, first=None, rows: Optional[int] = None, out=None, stream=None):
    """Rows first[s] .. first[s] + rows (None: from 0, all) of a cache in 4 bits -> [n_seq][n_kv][rows][128] of the given dtype, the
    values they stand for."""
    here = _here(out)
    room_for = _for(stream, here)
    n_seq, n_kv = x4[0].shape[:2]
    codes, scale, room = _kv4(x4, n_seq, n_kv, "x4", here)
    rows = room if rows is None else rows
    if out is None:
        with room_for:
            out = torch.empty(n_seq, n_kv, rows, 128, dtype=dtype, device=here)
    elif out.dtype is not dtype or out.shape != (n_seq, n_kv, rows, 128) or not out.is_contiguous():
        raise ValueError("out must be contiguous [n_seq][n_kv][rows][128], of the given dtype")
    _check(lib().ra_dequantize_kv4(codes, scale, _dt(out), n_seq, n_kv, rows, 128, None if first is None else _vector(first, n_seq, torch.int32, here, "first"),
                                   room, _handle(stream, here), out.data_ptr()))
    return out


def _results(n_seq, n_q, d, here, out, lse):
    """out [n_seq][n_q][d] and lse [n_seq][n_q], the given ones or new ones."""
    if out is None:
        out = torch.empty(n_seq, n_q, d, dtype=torch.float32, device=here)
    elif out.dtype is not torch.float32 or out.shape != (n_seq, n_q, d) or not out.is_contiguous() or out.get_device() != here:
        raise ValueError("out must be contiguous float32 [n_seq][n_q][128] on the current GPU")
    if lse is None:
        lse = torch.empty(n_seq, n_q, dtype=torch.float32, device=here)
    elif lse.dtype is not torch.float32 or lse.shape != (n_seq, n_q) or not lse.is_contiguous() or lse.get_device() != here:
        raise ValueError("lse must be contiguous float32 [n_seq][n_q] on the current GPU")
    return out, lse


def _query(q, here: int):
    """Checks q [n_seq][n_q][d] -> its address and sizes."""
    if q.dim() != 3 or not q.is_contiguous() or q.get_device() != here:
        raise ValueError("q must be contiguous [n_seq][n_q][128] on the current GPU")
    return q.data_ptr(), *q.shape


@functools.lru_cache(maxsize=256)
def _full_q4_room(dt: int, n_seq: int, n_q: int, n_kv: int, N: int) -> int:
    """ra_full_attention_q4_workspace_bytes, a function of sizes alone."""
    return max(1, lib().ra_full_attention_q4_workspace_bytes(dt, n_seq, n_q, n_kv, N))


def ra_full_attention_q4(q, k4, v4, n_tokens=None, N: Optional[int] = None, stream=None, workspace=None, out=None, lse=None):
    """Eq. 1 over the first n_tokens[s] rows (int32 [n_seq] on the GPU, at most N; None: N, by default the capacity) of a cache
    in 4 bits -> (out float32 [n_seq][n_q][128], lse float32 [n_seq][n_q])."""
    here = torch.cuda.current_device()
    room_for = _for(stream, here)
    q_at, n_seq, n_q, d = _query(q, here)
    n_kv = k4[0].shape[1]
    K4, K4s, room = _kv4(k4, n_seq, n_kv, "k4", here)
    V4, V4s, _ = _kv4(v4, n_seq, n_kv, "v4", here, room)
    dt = _dt(q)
    N = room if N is None else N
    if workspace is None:
        have = _full_q4_room(dt, n_seq, n_q, n_kv, N)
        with room_for:
            workspace = torch.empty(have, dtype=torch.uint8, device=here)
    else:
        _dev(workspace)
        _here(workspace)
        have = workspace.numel() * workspace.element_size()
    with room_for:
        out, lse = _results(n_seq, n_q, d, here, out, lse)
    _check(lib().ra_full_attention_q4(q_at, dt, K4, K4s, V4, V4s, n_seq, n_q, n_kv, N, room, d,
                                      None if n_tokens is None else _vector(n_tokens, n_seq, torch.int32, here, "n_tokens"),
                                      workspace.data_ptr(), have, _handle(stream, here), out.data_ptr(), lse.data_ptr()))
    return out, lse


def ra_attend_q4(q, idx: Index, k4, v4, sink: int, window: int, ids: torch.Tensor, N: Optional[int] = None, stream=None,
                 partials: bool = False, out=None, lse=None):
    """ra_attend over a cache in 4 bits that holds N >= idx.N tokens (by default as many as its capacity); tokens behind the
    index's are static. -> (out, lse) or, with partials=True, (out, lse, o_omega, lse_omega, o_w, lse_w)."""
    here = torch.cuda.current_device()
    room_for = _for(stream, here)
    q_at, n_seq, n_q, d = _query(q, here)
    n_kv, shape = k4[0].shape[1], ids.shape
    if (n_seq, n_q, n_kv) != idx.heads or d != 128:
        raise ValueError("q must be [n_seq][n_q][128], and its heads and the cache's those of the index")
    if idx.device != here:
        raise ValueError(f"the index must live on the current GPU ({here}), not on {idx.device}")
    if ids.dtype is not torch.int32 or len(shape) != 3 or shape[0] != n_seq or shape[1] != n_q or not ids.is_contiguous() \
            or ids.get_device() != here:
        raise ValueError("ids must be contiguous int32 [n_seq][n_q][topk] on the current GPU")
    K4, K4s, room = _kv4(k4, n_seq, n_kv, "k4", here)
    V4, V4s, _ = _kv4(v4, n_seq, n_kv, "v4", here, room)
    extra = ()
    with room_for:
        out, lse = _results(n_seq, n_q, d, here, out, lse)
        if partials:
            f = dict(dtype=torch.float32, device=here)
            extra = (torch.empty((n_seq, n_q, d), **f), torch.empty((n_seq, n_q), **f),
                     torch.empty((n_seq, n_q, d), **f), torch.empty((n_seq, n_q), **f))
    _check(_room(lib().ra_attend_q4, q_at, idx.handle, _dt(q), K4, K4s, V4, V4s, room if N is None else N, room, sink, window, shape[2],
                 ids.data_ptr(), _handle(stream, here), out.data_ptr(), lse.data_ptr(),
                 *([t.data_ptr() for t in extra] or (None, None, None, None))))
    return (out, lse, *extra) if partials else (out, lse)


_short = None


def _calls():
    """Load _calls.so (once): the calls around a cache in pages made and checked by compiled code, with the same outcome, where nothing is
    out of the ordinary; else they return None. None where it has not been built: the checks below are all there are then."""
    global _short
    if _short is None:
        L = lib()
        if not os.path.exists(CALLS_PATH):
            return None
        try:
            from . import _calls as m
        except ImportError as e:
            raise RuntimeError("_calls.so is broken: build it as libra.so") from e
        at = [C.cast(f, C.c_void_p).value for f in (L.ra_append_tokens_paged, L.ra_gather_paged, L.ra_full_attention_paged,
                                                    L.ra_full_attention_paged_workspace_bytes, L.ra_attend_paged, L.ra_attend_paged_workspace_bytes)]
        m.bind(_RAW or (lambda here: torch.cuda.current_stream(here).cuda_stream), *at)
        _short = m
    return _short


class PagedCache:
    """A cache in pages: K, V [n_pages][n_kv][page][128] (float32 or bfloat16, page a power of two; one of them may be None) and the
    table int32 [n_seq][table_pages] whose entry [s][r // page] is the page of row r of sequence s (outside [0, n_pages): none). Tensors of the
    current GPU, which stay the caller's: their contents, the table's among them, may change at any time, in stream order. Checked here, once."""

    def __init__(self, K, V, table):
        self._here = torch.cuda.current_device()
        some = K if K is not None else V
        if some is None:
            raise ValueError("K or V is needed")
        dt, shape = _dt(some), some.shape
        for t in (K, V):
            if t is not None and (t.dim() != 4 or t.shape != shape or t.shape[3] != 128 or not t.is_contiguous()):
                raise ValueError("K and V must be contiguous [n_pages][n_kv][page][128], of one shape")
            if t is not None and t.dtype is not some.dtype:
                raise TypeError("K and V must share a dtype")
        if table.dtype is not torch.int32 or table.dim() != 2 or (table.shape[1] > 1 and table.stride(1) != 1):
            raise ValueError("table must be an int32 tensor [n_seq][table_pages] whose rows are contiguous")
        _here(K, V, table)
        # (the stride of a dimension of one element says nothing)
        stride = table.stride(0) if table.shape[0] > 1 else table.shape[1]
        if stride < table.shape[1]:
            raise ValueError("the rows of the table must not overlap")
        self._K, self._V, self._table = K, V, table
        # where the tensors that there are were when this was checked
        self._at = tuple((t.data_ptr, t.data_ptr()) for t in (K, V, table) if t is not None)
        self._c = _PagedCache(_ptr(K), _ptr(V), table.data_ptr(), stride, dt, table.shape[0], shape[1], shape[0], shape[2], table.shape[1])
        self._ref = C.byref(self._c)
        short = _calls()
        self._core = short.cache(K, V, table, C.addressof(self._c), self._here) if short else None
        self._dt, self._dtype, self._n_seq, self._n_kv, self._rows = dt, some.dtype, table.shape[0], shape[1], table.shape[1] * shape[2]

    K = property(lambda s: s._K)
    V = property(lambda s: s._V)
    table = property(lambda s: s._table)
    n_seq = property(lambda s: s._n_seq)
    n_kv_heads = property(lambda s: s._n_kv)
    page = property(lambda s: s._c.page)
    rows = property(lambda s: s._rows, doc="Rows that a row of the table has entries for.")
    dtype = property(lambda s: s._dtype)

    def _of(self, here: int):
        """What a call passes on, the tensors being where they were."""
        if here != self._here:
            raise ValueError(f"the cache must live on the current GPU ({here}), not on {self._here}")
        for now, then in self._at:
            if now() != then:
                raise ValueError("the cache's tensors have been given other memory: make another PagedCache")
        return self._ref


def _is_paged(cache) -> None:
    if not isinstance(cache, PagedCache):
        raise TypeError(f"cache must be a PagedCache, not {type(cache).__name__}")


def ra_append_tokens_paged(q, k, v, first, cache: PagedCache, *, n_new=None, q_weight=None, k_weight=None, eps: float = 1e-6, inv_freq=None,
                           interleaved: bool = False, rot_scale: float = 1.0, q_out=None, stream=None):
    """ra_append_tokens into a cache in pages; cosines and sines times rot_scale. k and v may be None: nothing of K or V is
    written. -> q_out [n_seq][n_q][T][128] (None without q), as there."""
    _is_paged(cache)
    if stream is None and cache._core is not None:
        got = _short.append(q, k, v, first, cache._core, n_new, q_weight, k_weight, eps, inv_freq, interleaved, rot_scale, q_out)
        if got.__class__ is tuple:
            return got[0]
        _check(got or 0)
    some = q if q is not None else k if k is not None else v
    if some is None:
        raise ValueError("at least one of q, k and v is needed")
    here = torch.cuda.current_device()
    room_for = _for(stream, here)
    ref = cache._of(here)
    dtype, shape, n_seq, n_kv = cache._dtype, some.shape, cache._n_seq, cache._n_kv
    if len(shape) != 4:
        raise ValueError("q, k and v must be [n_seq][T][heads][128]")
    T = shape[1]
    if q is not None:
        q_at, n_q, q_row = _token_rows(q, n_seq, T, dtype, here)
    else:
        q_at, n_q, q_row = None, n_kv, 0
    k_at, n_k, k_row = _token_rows(k, n_seq, T, dtype, here) if k is not None else (None, n_kv, 0)
    v_at, n_v, v_row = _token_rows(v, n_seq, T, dtype, here) if v is not None else (None, n_kv, 0)
    if n_k != n_kv or n_v != n_kv:
        raise ValueError("k and v must have the heads of the cache")
    qw_at = _vector(q_weight, 128, dtype, here, "q_weight") if q_weight is not None else None
    kw_at = _vector(k_weight, 128, dtype, here, "k_weight") if k_weight is not None else None
    f_at, rot = None, 0
    if inv_freq is not None:
        rot = 2 * inv_freq.numel()
        f_at = _vector(inv_freq, rot // 2, torch.float32, here, "inv_freq")
    first_at = _vector(first, n_seq, torch.int32, here, "first") if first is not None else None
    new_at = _vector(n_new, n_seq, torch.int32, here, "n_new") if n_new is not None else None
    out_at = None
    if q is None:
        if q_out is not None:
            raise ValueError("q_out goes with q")
    else:
        if q_out is None:
            with room_for:
                q_out = (torch.empty if n_new is None else torch.zeros)(n_seq, n_q, T, 128, dtype=dtype, device=here)
        elif q_out.dtype is not dtype or q_out.shape != (n_seq, n_q, T, 128) or not q_out.is_contiguous() or q_out.get_device() != here:
            raise ValueError("q_out must be contiguous [n_seq][n_q][T][128], of the dtype of q and where q is")
        out_at = q_out.data_ptr()
    _check(lib().ra_append_tokens_paged(q_at, k_at, v_at, ref, n_q, T, 128, q_row, k_row, v_row, qw_at, kw_at, eps, f_at, rot,
                                        1 if interleaved else 0, rot_scale, first_at, new_at, _handle(stream, here), out_at))
    return q_out


def ra_gather_paged(cache: PagedCache, values: bool = False, first=None, rows: Optional[int] = None, out=None, stream=None):
    """Rows first[s] .. first[s] + rows (None: from 0, all that the table has entries for) of K, or with `values` of V, side by side
    -> [n_seq][n_kv][rows][128]; rows without a page are zero."""
    _is_paged(cache)
    if stream is None and cache._core is not None:
        got = _short.gather(cache._core, values, first, rows, out)
        if got.__class__ is tuple:
            return got[0]
        _check(got or 0)
    here = torch.cuda.current_device()
    room_for = _for(stream, here)
    ref = cache._of(here)
    shape = (cache._n_seq, cache._n_kv, cache._rows if rows is None else rows, 128)
    if out is None:
        with room_for:
            out = torch.empty(shape, dtype=cache._dtype, device=here)
    elif out.dtype is not cache._dtype or out.shape != shape or not out.is_contiguous() or out.get_device() != here:
        raise ValueError("out must be contiguous [n_seq][n_kv][rows][128], of the cache's dtype and where it is")
    _check(lib().ra_gather_paged(ref, 1 if values else 0, shape[2], 128, None if first is None else _vector(first, shape[0], torch.int32, here, "first"),
                                 _handle(stream, here), out.data_ptr()))
    return out


def _paged_query(q, cache: PagedCache, here: int):
    """Checks q -> its address, query heads and dimensions."""
    q_at, n_seq, n_q, d = _query(q, here)
    if n_seq != cache._n_seq:
        raise ValueError(f"q has {n_seq} sequences, the table {cache._n_seq}")
    if q.dtype is not cache._dtype:
        raise TypeError("q and the cache must share a dtype")
    return q_at, n_q, d


def _workspace(given, need: int, room_for, here: int):
    """The given workspace, or a new one of `need` bytes -> (it, its bytes)."""
    if given is None:
        need = max(1, need)
        if room_for is _CURRENT:
            return torch.empty(need, dtype=torch.uint8, device=here), need
        with room_for:
            return torch.empty(need, dtype=torch.uint8, device=here), need
    _dev(given)
    _here(given)
    return given, given.numel() * given.element_size()


def _paged_results(n_seq: int, n_q: int, d: int, room_for, here: int, out, lse):
    """_results, on the call's stream."""
    if room_for is _CURRENT or (out is not None and lse is not None):
        return _results(n_seq, n_q, d, here, out, lse)
    with room_for:
        return _results(n_seq, n_q, d, here, out, lse)


@functools.lru_cache(maxsize=256)
def _full_paged_room(dt: int, n_seq: int, n_q: int, n_kv: int, N: int) -> int:
    """ra_full_attention_paged_workspace_bytes, a function of sizes alone."""
    return lib().ra_full_attention_paged_workspace_bytes(dt, n_seq, n_q, n_kv, N)


def ra_full_attention_paged(q, cache: PagedCache, n_tokens=None, N: Optional[int] = None, stream=None, workspace=None, out=None, lse=None):
    """Eq. 1 over the first n_tokens[s] rows (int32 [n_seq] on the GPU, at most N; None: N, by default cache.rows) of every sequence of a
    cache in pages, those that have a page -> (out float32 [n_seq][n_q][128], lse float32 [n_seq][n_q])."""
    _is_paged(cache)
    if stream is None and cache._core is not None:
        got = _short.full(q, cache._core, n_tokens, N, workspace, out, lse)
        if got.__class__ is tuple:
            return got
        _check(got or 0)
    here = torch.cuda.current_device()
    room_for = _for(stream, here)
    ref = cache._of(here)
    q_at, n_q, d = _paged_query(q, cache, here)
    n_seq = cache._n_seq
    N = cache._rows if N is None else N
    workspace, have = _workspace(workspace, 0 if workspace is not None else _full_paged_room(cache._dt, n_seq, n_q, cache._n_kv, N), room_for, here)
    out, lse = _paged_results(n_seq, n_q, d, room_for, here, out, lse)
    _check(lib().ra_full_attention_paged(q_at, ref, n_q, N, d, None if n_tokens is None else _vector(n_tokens, n_seq, torch.int32, here, "n_tokens"),
                                         workspace.data_ptr(), have, _handle(stream, here), out.data_ptr(), lse.data_ptr()))
    return out, lse


@functools.lru_cache(maxsize=256)
def _attend_paged_room(dt: int, n_seq: int, n_q: int, n_kv: int, N: int, sink: int, window: int, topk: int) -> int:
    """ra_attend_paged_workspace_bytes, a function of sizes alone."""
    return lib().ra_attend_paged_workspace_bytes(dt, n_seq, n_q, n_kv, N, sink, window, topk)


def ra_attend_paged(q, cache: PagedCache, sink: int, window: int, ids: torch.Tensor, n_tokens=None, n_indexed=None, N: Optional[int] = None,
                    stream=None, partials: bool = False, workspace=None, out=None, lse=None):
    """ra_attend over a cache in pages, of n_tokens[s] rows (int32 [n_seq] on the GPU, at most N; None: N, by default cache.rows), the first
    n_indexed[s] of which (None: all) an index was built over; those behind are static. ids in the static set are
    skipped. -> (out, lse) or, with partials=True, (out, lse, o_omega, lse_omega, o_w, lse_w)."""
    _is_paged(cache)
    if stream is None and not partials and cache._core is not None:
        got = _short.attend(q, cache._core, sink, window, ids, n_tokens, n_indexed, N, workspace, out, lse)
        if got.__class__ is tuple:
            return got
        _check(got or 0)
    here = torch.cuda.current_device()
    room_for = _for(stream, here)
    ref = cache._of(here)
    q_at, n_q, d = _paged_query(q, cache, here)
    n_seq, shape = cache._n_seq, ids.shape
    if ids.dtype is not torch.int32 or len(shape) != 3 or shape[0] != n_seq or shape[1] != n_q or not ids.is_contiguous() \
            or ids.get_device() != here:
        raise ValueError("ids must be contiguous int32 [n_seq][n_q][topk] on the current GPU")
    N = cache._rows if N is None else N
    need = 0 if workspace is not None else _attend_paged_room(cache._dt, n_seq, n_q, cache._n_kv, N, sink, window, shape[2])
    workspace, have = _workspace(workspace, need, room_for, here)
    out, lse = _paged_results(n_seq, n_q, d, room_for, here, out, lse)
    extra = (None, None, None, None)
    if partials:
        f = dict(dtype=torch.float32, device=here)
        with room_for:
            extra = (torch.empty((n_seq, n_q, d), **f), torch.empty((n_seq, n_q), **f),
                     torch.empty((n_seq, n_q, d), **f), torch.empty((n_seq, n_q), **f))
    _check(lib().ra_attend_paged(q_at, ref, n_q, N, d, None if n_tokens is None else _vector(n_tokens, n_seq, torch.int32, here, "n_tokens"),
                                 None if n_indexed is None else _vector(n_indexed, n_seq, torch.int32, here, "n_indexed"), sink, window, shape[2],
                                 ids.data_ptr(), workspace.data_ptr(), have, _handle(stream, here), out.data_ptr(), lse.data_ptr(),
                                 *map(_ptr, extra)))
    return (out, lse, *extra) if partials else (out, lse)
