"""Attention over a cache in pages where lists of rows are long or many: units of more than 128 rows, more jobs than a list holds, the largest pages, static
rows far past what a job is cut by."""
import numpy as np
import pytest
import torch

import paper_2409_10516_amd as ra
from oracle import paged as OP
from tests.test_gpu_paged import DEV, TYPES, Cache, check, ints, queries
from tests.util import to_np

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("page", [65536, 8])
def test_units_of_many_rows(dtype, page):
    """320 sequences of up to 2^20 tokens: units of 256 rows. Most are short, some end inside a unit, one is long; all share their pages."""
    n_seq, N, long = 320, 1 << 20, 200001
    rng = np.random.default_rng(5)
    lens = rng.integers(0, 3000, n_seq)
    lens[:6], lens[200], lens[-1] = [0, 1, 255, 256, 257, 0], long, 100003
    c = Cache([long], 1, page, dtype, seed=1)
    table = torch.full((n_seq, N // page), -1, dtype=torch.int32, device=DEV)
    table[:, :c.table.shape[1]] = ints(c.table)
    q = queries(n_seq, 2, dtype, 2)
    out, lse = (t.cpu().numpy() for t in ra.ra_full_attention_paged(q.to(DEV), ra.PagedCache(c.K, c.V, table), ints(lens)))
    assert (out[lens == 0] == 0).all() and np.isneginf(lse[lens == 0]).all()
    K, V = c.rows(0, 0, range(long))
    for s in [0, 1, 2, 3, 4, 5, 6, 77, 199, 200, 201, n_seq - 1]:
        for h in range(2):
            check(out[s, h], lse[s, h], to_np(q[s, h]), K[:lens[s]], V[:lens[s]])


@pytest.mark.parametrize("dtype", TYPES)
def test_more_jobs_than_a_list_holds(dtype):
    """2^21 of them, a workgroup's each whatever their length."""
    n_seq, n_kv, n = 1 << 18, 8, 2500
    c = Cache([n], n_kv, 4096, dtype, seed=3)
    table = ints(c.table).expand(n_seq, -1).contiguous()
    lens = torch.randint(0, 3, (n_seq,), dtype=torch.int32, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
    some = {0: n, 1: 0, 4097: 2049, 100000: 17, n_seq - 2: 1, n_seq - 1: n - 1}
    for s, m in some.items():
        lens[s] = m
    q = torch.randn((n_seq, n_kv, 128), device=DEV, generator=torch.Generator(device=DEV).manual_seed(2), dtype=torch.float32).to(dtype)
    out, lse = ra.ra_full_attention_paged(q, ra.PagedCache(c.K, c.V, table), lens, N=n)
    empty = lens == 0
    assert (out[empty] == 0).all() and torch.isneginf(lse[empty]).all() and torch.isfinite(lse[~empty]).all()
    for s, m in some.items():
        for h in (0, 5, n_kv - 1):
            check(out[s, h].cpu().numpy(), float(lse[s, h]), to_np(q[s, h]), *c.rows(0, h, range(m)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens,indexed,n_kv,n_q,sink,window,topk", [
    ([30011], [11], 1, 1, 4, 0, 1), ([30011], [3000], 1, 4, 4, 64, 16), ([20007, 900], [500, 900], 2, 4, 0, 64, 1), ([9000] + [300] * 139, [100] + [300] * 139, 1, 2, 4, 64, 16),
    ([12000] * 3, [12000, 0, 7000], 8, 16, 4, 640, 100)])
def test_static_rows_far_past_the_window(dtype, lens, indexed, n_kv, n_q, sink, window, topk):
    """Tokens behind the index are static, and the parts of a job know of the window alone: one or a few workgroups have thousands of rows."""
    n_seq = len(lens)
    c = Cache(lens, n_kv, 16, dtype, seed=sum(lens), holes=0.05)
    q, rng = queries(n_seq, n_q, dtype, 7), np.random.default_rng(8)
    ids = rng.integers(0, max(lens), (n_seq, n_q, topk)).astype(np.int32)
    got = [t.cpu().numpy() for t in ra.ra_attend_paged(q.to(DEV), c.gpu, sink, window, torch.from_numpy(ids).to(DEV), ints(lens), n_indexed=ints(indexed), partials=True)]
    for s in sorted({0, 1, n_seq // 2, n_seq - 1} & set(range(n_seq))):
        for h in sorted({0, n_q // 2, n_q - 1}):
            W, om = OP.sets(lens[s], indexed[s], sink, window, ids[s, h].tolist())
            for (o, l), rows in zip((got[0:2], got[2:4], got[4:6]), (np.concatenate([W, om]), om, W)):
                check(o[s, h], l[s, h], to_np(q[s, h]), *c.rows(s, h // (n_q // n_kv), rows.tolist()))
