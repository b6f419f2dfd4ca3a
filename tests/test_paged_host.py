"""What the calls around a cache in pages refuse, before anything touches a device (no GPU)."""
import ctypes as C

import pytest
import torch

import paper_2409_10516_amd as ra
from paper_2409_10516_amd import binding as B


def _p(at=0x10000):
    return C.c_void_p(at)       # non-null; never dereferenced when validation fails first


CACHE = dict(K=0x10000, V=0x20000, table=0x30000, table_stride=8, dt=1, n_seq=2, n_kv_heads=2, n_pages=20, page=16, table_pages=8)
APPEND = dict(q_in=_p(), k_in=_p(), v_in=_p(), cache=None, n_q=4, T=3, d=128, q_row=512, k_row=256, v_row=256, qw=None, kw=None, eps=1e-6,
              inv_freq=_p(), rot=128, inter=0, rot_scale=1.0, first=None, n_new=None, stream=None, q_out=_p())
GATHER = dict(cache=None, values=0, T=5, d=128, first=None, stream=None, X=_p())
FULL = dict(q=_p(), cache=None, n_q=4, N=100, d=128, n_tokens=None, ws=_p(), ws_bytes=1 << 30, stream=None, out=_p(), lse=_p())
ATTEND = dict(q=_p(), cache=None, n_q=4, N=100, d=128, n_tokens=None, n_indexed=None, sink=4, window=8, topk=10, ids=_p(), ws=_p(), ws_bytes=1 << 30,
              stream=None, out=_p(), lse=_p(), o_om=None, lse_om=None, o_w=None, lse_w=None)
CALLS = {"ra_append_tokens_paged": APPEND, "ra_gather_paged": GATHER, "ra_full_attention_paged": FULL, "ra_attend_paged": ATTEND}


def _refused(name, change, cache, status, needle):
    L = ra.lib()
    args = CALLS[name] | dict(cache=None if cache is None else C.byref(B._PagedCache(**(CACHE | cache)))) | change
    assert getattr(L, name)(*args.values()) == status
    assert needle in L.ra_last_error().decode()


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("cache,status,needle", [
    (None, 1, "the cache"), (dict(dt=3), 3, "dtype"), (dict(n_seq=0), 1, "positive"), (dict(n_kv_heads=-1), 1, "positive"),
    (dict(n_pages=0), 1, "positive"), (dict(table_pages=0), 1, "positive"), (dict(page=0), 1, "positive"), (dict(page=-16), 1, "positive"),
    (dict(page=24), 6, "power of two"), (dict(page=1 << 17), 6, "power of two"), (dict(table=None), 1, "table"), (dict(table_stride=7), 2, "table_stride"),
    (dict(table=0x30002), 1, "aligned"), (dict(K=0x10008), 1, "aligned"), (dict(V=0x20004), 1, "aligned"),
    (dict(n_pages=1 << 27), 6, "rows in a pool"), (dict(n_pages=1 << 26, n_kv_heads=2), 6, "rows in a pool"),
    (dict(n_pages=(1 << 31) - 1, page=65536, n_kv_heads=(1 << 31) - 1), 6, "rows in a pool"),
    (dict(table_pages=1 << 26, table_stride=1 << 26), 6, "rows of a sequence"),
])
def test_caches_that_are_refused(name, cache, status, needle):
    _refused(name, {}, cache, status, needle)


@pytest.mark.parametrize("name,change,cache,status,needle", [
    ("ra_append_tokens_paged", dict(q_in=None), {}, 1, "together"), ("ra_append_tokens_paged", dict(q_out=None), {}, 1, "together"),
    ("ra_append_tokens_paged", dict(q_in=None, q_out=None, k_in=None, v_in=None), {}, 1, "no input"),
    ("ra_append_tokens_paged", {}, dict(K=None), 1, "K"), ("ra_append_tokens_paged", {}, dict(V=None), 1, "V"),
    ("ra_append_tokens_paged", dict(n_q=3), {}, 1, "multiple"), ("ra_append_tokens_paged", dict(d=64), {}, 6, "d = 128"),
    ("ra_append_tokens_paged", dict(T=0), {}, 1, "positive"), ("ra_append_tokens_paged", dict(T=1 << 31), {}, 6, "large"),
    ("ra_append_tokens_paged", dict(rot=24), {}, 6, "16"), ("ra_append_tokens_paged", dict(rot=144), {}, 1, "rot_dim"),
    ("ra_append_tokens_paged", dict(inv_freq=None), {}, 1, "inv_freq"), ("ra_append_tokens_paged", dict(q_row=511), {}, 2, "apart"),
    ("ra_append_tokens_paged", dict(k_row=0), {}, 2, "apart"), ("ra_append_tokens_paged", dict(v_row=257), {}, 6, "16 bytes"),
    ("ra_append_tokens_paged", dict(q_in=_p(0x10008)), {}, 1, "aligned"), ("ra_append_tokens_paged", dict(q_out=_p(0x10004)), {}, 1, "aligned"),
    ("ra_append_tokens_paged", dict(qw=_p(), eps=-1.0), {}, 1, "eps"), ("ra_append_tokens_paged", dict(kw=_p(), eps=float("nan")), {}, 1, "eps"),
    ("ra_append_tokens_paged", dict(qw=_p(0x10001)), {}, 1, "aligned"), ("ra_append_tokens_paged", dict(rot_scale=float("inf")), {}, 1, "rot_scale"),
    ("ra_append_tokens_paged", dict(rot_scale=float("nan")), {}, 1, "rot_scale"), ("ra_append_tokens_paged", dict(T=1 << 23), {}, 6, "tokens"),
    ("ra_append_tokens_paged", dict(n_q=1 << 24, q_row=1 << 31), {}, 6, "heads"),
    ("ra_gather_paged", {}, dict(K=None), 1, "K"), ("ra_gather_paged", dict(values=1), dict(V=None), 1, "V"), ("ra_gather_paged", dict(X=None), {}, 1, "NULL"),
    ("ra_gather_paged", dict(T=0), {}, 1, "positive"), ("ra_gather_paged", dict(T=1 << 31), {}, 6, "large"), ("ra_gather_paged", dict(d=96), {}, 6, "d = 128"),
    ("ra_gather_paged", dict(X=_p(0x10008)), {}, 1, "aligned"), ("ra_gather_paged", dict(T=(1 << 30) - 1), {}, 6, "too many rows"),
    ("ra_full_attention_paged", {}, dict(K=None), 1, "K"), ("ra_full_attention_paged", {}, dict(V=None), 1, "V"),
    ("ra_full_attention_paged", dict(q=None), {}, 1, "NULL"), ("ra_full_attention_paged", dict(out=None), {}, 1, "NULL"),
    ("ra_full_attention_paged", dict(lse=None), {}, 1, "NULL"), ("ra_full_attention_paged", dict(ws=None), {}, 1, "NULL"),
    ("ra_full_attention_paged", dict(n_q=5), {}, 1, "multiple"), ("ra_full_attention_paged", dict(d=256), {}, 6, "d = 128"),
    ("ra_full_attention_paged", dict(N=0), {}, 1, "positive"), ("ra_full_attention_paged", dict(N=129), {}, 2, "128 rows"),
    ("ra_full_attention_paged", dict(N=1 << 40), {}, 2, "above"), ("ra_full_attention_paged", dict(q=_p(0x10002)), {}, 1, "aligned"),
    ("ra_full_attention_paged", dict(ws=_p(0x10004)), {}, 1, "aligned"), ("ra_full_attention_paged", dict(ws_bytes=8), {}, 2, "workspace"),
    ("ra_full_attention_paged", dict(n_q=1 << 30, N=1 << 25, ws_bytes=1 << 62), dict(table_pages=1 << 25, table_stride=1 << 25, page=1, n_kv_heads=1), 6, "too many heads"),
    ("ra_attend_paged", {}, dict(K=None), 1, "K"), ("ra_attend_paged", {}, dict(V=None), 1, "V"), ("ra_attend_paged", dict(q=None), {}, 1, "NULL"),
    ("ra_attend_paged", dict(ids=None), {}, 1, "NULL"), ("ra_attend_paged", dict(ws=None), {}, 1, "NULL"), ("ra_attend_paged", dict(n_q=5), {}, 1, "multiple"),
    ("ra_attend_paged", dict(d=64), {}, 6, "d = 128"), ("ra_attend_paged", dict(N=0), {}, 1, "positive"), ("ra_attend_paged", dict(N=129), {}, 2, "128 rows"),
    ("ra_attend_paged", dict(sink=-1), {}, 1, "non-negative"), ("ra_attend_paged", dict(window=-1), {}, 1, "non-negative"),
    ("ra_attend_paged", dict(topk=0), {}, 1, "topk"), ("ra_attend_paged", dict(topk=2049), {}, 6, "RA_MAX_TOPK"),
    ("ra_attend_paged", dict(q=_p(0x10008)), {}, 1, "aligned"), ("ra_attend_paged", dict(ws=_p(0x10008)), {}, 1, "aligned"),
    ("ra_attend_paged", dict(ws_bytes=8, window=100), {}, 2, "workspace"), ("ra_attend_paged", dict(n_q=1 << 28, ws_bytes=1 << 62), {}, 6, "too many heads"),
    ("ra_attend_paged", dict(ws_bytes=1 << 62), dict(n_seq=65536), 6, "too many heads"),
    ("ra_attend_paged", dict(n_q=65536, ws_bytes=1 << 62), dict(n_kv_heads=65536), 6, "too many heads"),
    ("ra_attend_paged", dict(n_q=2048, ws_bytes=1 << 62), dict(n_seq=2048, n_kv_heads=2048), 6, "too many heads"),
    ("ra_full_attention_paged", dict(n_q=4, N=100), dict(n_seq=1 << 22, n_kv_heads=2, n_pages=1), 6, "too many heads"),
])
def test_calls_that_are_refused(name, change, cache, status, needle):
    _refused(name, change, cache, status, needle)


def test_workspace_sizes():
    L = ra.lib()
    full, attend = L.ra_full_attention_paged_workspace_bytes, L.ra_attend_paged_workspace_bytes
    assert full(1, 1, 32, 8, 131072) > 256 and full(0, 1, 4, 1, 1) == 256 and full(2, 1, 4, 1, 1) == 0
    assert full(1, 1, 32, 7, 1000) == 0 and full(1, 1, 32, 8, 0) == 0 and full(1, 1, 32, 8, 1 << 31) == 0 and full(1, 0, 4, 1, 10) == 0
    assert attend(1, 1, 32, 8, 1000, 4, 640, 100) >= 256 + 32 * 2 * 2 * 132 * 4 and attend(0, 1, 32, 8, 1000, 0, 0, 1) == 256
    for bad in ((1, 1, 32, 7, 1000, 4, 640, 100), (1, 1, 32, 8, 0, 4, 640, 100), (1, 1, 32, 8, 1000, -1, 640, 100), (1, 1, 32, 8, 1000, 4, -1, 100),
                (1, 1, 32, 8, 1000, 4, 640, 0), (1, 1, 32, 8, 1000, 4, 640, 2049), (2, 1, 32, 8, 1000, 4, 640, 100)):
        assert attend(*bad) == 0


def test_tensors_that_are_not_on_the_gpu_are_refused():
    K, table = torch.zeros(3, 2, 16, 128), torch.zeros(1, 2, dtype=torch.int32)
    with pytest.raises((ValueError, RuntimeError, AssertionError)):
        ra.PagedCache(K, K, table)
    with pytest.raises((ValueError, RuntimeError, AssertionError)):
        ra.PagedCache(None, None, table)
