"""Rows that must not get lost on their way through records: NaN rows, non-finite queries and rows with all the weight where a
head's attention over a 4-bit cache is put together from many parts, each of the ways of putting it together."""
import numpy as np
import pytest
import torch

import paper_2409_10516_amd as ra
from oracle import attention as OA
from tests.test_gpu_q4 import _cache, _check, _handle, _queries
from tests.util import to_np

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

FULL = [
    # n_seq, n_q, n_kv, N, tokens of the other sequences, where (of N) the special row is
    (1, 16, 8, 20000, None, 0.6),       # some 64 records a head: combined by 32 dimensions
    (8, 16, 8, 3000, None, 0.7),        # eight records a head, a thread for each dimension
    (10, 4, 2, 50000, 200, 0.9),        # one long sequence, hundreds of records: groups of threads, all dimensions
    (130, 8, 1, 40000, 130, 0.5),       # the same beside so many heads that workgroups are small
    (8, 16, 8, 3000, None, 0.01),       # in the first record
    (1, 4, 2, 60, None, 0.5),           # no records: the workgroup writes the result
]


def _spread(x4, n_seq, n_kv):
    """One head's rows for all."""
    return tuple(t.expand(n_seq, n_kv, -1, -1).contiguous() for t in x4)


def _setup(case, seed):
    n_seq, n_q, n_kv, N, others, at = case
    k4, v4, K, V = _cache(1, 1, N, seed=seed)
    lens = np.full(n_seq, N if others is None else others, np.int32)
    s = n_seq // 2
    lens[s] = N
    return _spread(k4, n_seq, n_kv), _spread(v4, n_seq, n_kv), K[0, 0], V[0, 0], lens, torch.from_numpy(lens).to(DEV), s, int(at * N)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("case", FULL)
def test_a_dominating_row_in_a_late_record(case, dtype):
    """Logits of hundreds, so that records' maxima are hundreds apart; other heads have a flat softmax, or an inverted one."""
    n_seq, n_q, n_kv, N, _, _ = case
    k4, v4, K, V, lens, n_tokens, s, at = _setup(case, 41)
    q = _queries(n_seq, n_q, dtype, 42)
    top = torch.from_numpy(K[at] * 20).to(dtype)
    q[s, 0], q[s, n_q - 1] = top, -top
    q[s, 1] = 0
    out, lse = (t.cpu().numpy() for t in ra.ra_full_attention_q4(q.to(DEV), k4, v4, n_tokens))
    for i in sorted({0, s, n_seq - 1}):
        for h in (0, 1, n_q - 1):
            _check(out[i, h], lse[i, h], to_np(q[i, h]), K, V, np.arange(lens[i]), dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("case", FULL)
def test_a_nan_row_in_a_late_record(case, dtype):
    """A key's NaN is its whole head's, a value's its own block's; nobody else's."""
    n_seq, n_q, n_kv, N, _, _ = case
    k4, v4, K, V, lens, n_tokens, s, at = _setup(case, 43)
    group, last = n_q // n_kv, n_kv - 1
    q = _queries(n_seq, n_q, dtype, 44)
    v4[1][s, 0, at, 1] = 255
    out, lse = (t.cpu().numpy() for t in ra.ra_full_attention_q4(q.to(DEV), k4, v4, n_tokens))
    bad = np.isnan(out[s, :group])
    assert bad[:, 32:64].all() and not bad[:, :32].any() and not bad[:, 64:].any() and np.isfinite(lse[s]).all()
    assert np.isfinite(out[s, group:]).all() and np.isfinite(np.delete(out, s, 0)).all()
    v4[1][s, 0, at, 1] = 127
    k4[1][s, last, at, 3] = 255
    q[0, 0, 5] = float("inf") if n_seq > 1 else q[0, 0, 5]
    out, lse = (t.cpu().numpy() for t in ra.ra_full_attention_q4(q.to(DEV), k4, v4, n_tokens))
    assert np.isnan(out[s, last * group:]).all() and np.isnan(lse[s, last * group:]).all()
    assert np.isfinite(out[s, :last * group]).all() and np.isfinite(lse[s, :last * group]).all()
    if n_seq > 1:
        assert np.isnan(out[0, 0]).all() and np.isnan(lse[0, 0]) and np.isfinite(np.delete(out, s, 0)[1:]).all()
        _check(out[0, 1], lse[0, 1], to_np(q[0, 1]), K, V, np.arange(lens[0]), dtype)


SPARSE = [
    # n_seq, n_q, n_kv, N, index covers, sink, window, topk
    (1, 4, 1, 20011, 500, 4, 17, 9),            # by a second launch, many records: eight threads a dimension
    (1, 16, 1, 40001, 3001, 4, 640, 100),       # the same, of 16 heads together
    (40, 16, 2, 2100, 300, 3, 20, 50),          # by a second one, two records
    (20, 4, 2, 5000, 300, 4, 17, 9),            # in the same launch, 13 records of a few heads each
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("case", SPARSE)
def test_special_rows_in_a_long_static_set(case, dtype):
    n_seq, n_q, n_kv, N, Ng, sink, window, topk = case
    group, s = n_q // n_kv, n_seq // 2
    k1, v1, K, V = _cache(1, 1, N, seed=45)
    K, V = K[0, 0], V[0, 0]
    k4, v4 = _spread(k1, n_seq, n_kv), _spread(v1, n_seq, n_kv)
    at = Ng + (N - Ng) * 2 // 3                  # a static row that came after the index
    W = OA.static_ids(N, sink, window, Ng)
    assert at in W
    ids = np.stack([np.random.default_rng(h).choice(np.arange(sink, Ng - window), topk, replace=False) for h in range(n_q)]).astype(np.int32)
    q = _queries(n_seq, n_q, dtype, 46)
    top = torch.from_numpy(K[at] * 20).to(dtype)
    q[s, 0], q[s, 1], q[s, n_q - 1] = top, 0, -top
    idx = _handle(n_seq, n_q, n_kv, Ng)
    ids_g = torch.from_numpy(ids).expand(n_seq, -1, -1).contiguous().to(DEV)
    call = lambda: [t.cpu().numpy() for t in ra.ra_attend_q4(q.to(DEV), idx, k4, v4, sink, window, ids_g, partials=True)]  # noqa: E731
    got = call()
    for h in (0, 1, n_q - 1):
        for (o, l), rows in zip((got[0:2], got[2:4], got[4:6]), (np.concatenate([W, ids[h]]), ids[h], W)):
            _check(o[s, h], l[s, h], to_np(q[s, h]), K, V, rows.astype(np.int64), dtype)
    v4[1][s, 0, at, 2] = 255
    out, lse, o_om, l_om, o_w, l_w = call()
    for o in (out, o_w):
        bad = np.isnan(o[s, :group])
        assert bad[:, 64:96].all() and not bad[:, :64].any() and not bad[:, 96:].any() and np.isfinite(o[s, group:]).all()
    assert np.isfinite(o_om).all() and all(np.isfinite(x).all() for x in (lse, l_om, l_w))
    v4[1][s, 0, at, 2] = 127
    k4[1][s, n_kv - 1, at, 0] = 255
    out, lse, o_om, l_om, o_w, l_w = call()
    for x in (out, lse, o_w, l_w):
        assert np.isnan(x[s, n_q - group:]).all() and np.isfinite(x[s, :n_q - group]).all() and np.isfinite(np.delete(x, s, 0)).all()
    assert np.isfinite(o_om).all() and np.isfinite(l_om).all()
    idx.free()
