"""Large logits over a cache in pages: rows of equal products have equal weights, whichever workgroup, set or record they are in."""
import numpy as np
import pytest
import torch

import paper_2409_10516_amd as ra
from tests.test_gpu_paged import DEV, TYPES, U, ints

pytestmark = pytest.mark.gpu
TOP, LOW = 2.0 ** 24, 56.0                      # products are TOP or TOP - LOW, exactly


def _inputs(N, n_kv, low, seed):
    """-> pools of one sequence in order, in float64 too. The first 64 dimensions of a value are one where (row // 512) is odd, else zero."""
    page, g = 64, np.random.default_rng(seed)
    K, V = np.zeros((N, n_kv, 128)), g.standard_normal((N, n_kv, 128)).astype(np.float32)
    K[..., 0] = 2.0 ** 12
    K[low, :, 1] = -LOW
    V[..., :64] = (np.arange(N) // 512 % 2)[:, None, None]
    V = torch.from_numpy(V).bfloat16().double().numpy()
    pool = lambda x: torch.from_numpy(x).reshape(-1, page, n_kv, 128).transpose(1, 2).contiguous()  # noqa: E731
    return pool(K), pool(V), V


def _check(out, lse, rows, low, V, added):
    """Products are exact. A weight's argument, at most 62 + 56 units times log2(e) / sqrt(128) in two roundings, is off by 21 U of the weight and the exponential by
    2; it meets at most five more such factors (running maximum, workgroup, slice, records, sets): 6 x 24 U. A row's weight and value go through `added` additions."""
    w = np.where(low[rows], np.exp(-LOW / np.sqrt(128)), 1.0)
    w, total = w / w.sum(), w.sum()
    tol = (added + 150) * U
    assert (np.abs(out - w @ V[rows]) <= tol * (w @ np.abs(V[rows]))).all(), (np.abs(out - w @ V[rows]) / (tol * (w @ np.abs(V[rows])) + 1e-300)).max()
    l = TOP / np.sqrt(128) + np.log(total)
    assert abs(lse - l) <= tol + 6 * U * l


def _query(n_seq, n_q, dtype):
    q = torch.zeros((n_seq, n_q, 128), dtype=dtype, device=DEV)
    q[..., 0], q[..., 1] = 2.0 ** 12, 1.0
    return q


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,n_kv,n_seq", [(131072, 1, 1), (16384, 8, 1), (131072 // 12, 1, 12), (8192, 2, 200)])
def test_full_attention(dtype, N, n_kv, n_seq):
    """Stretches of 512 rows or so, every second of which begins with 128 lower ones, one chunk for each of its wavefronts."""
    N = N // 64 * 64
    low = np.arange(N) // 128 % 8 == 0
    K, V, rows_V = _inputs(N, n_kv, low, 1)
    table = torch.arange(N // 64, dtype=torch.int32, device=DEV).expand(n_seq, -1).contiguous()
    cache = ra.PagedCache(K.to(dtype).to(DEV), V.to(dtype).to(DEV), table)
    out, lse = (t.cpu().numpy() for t in ra.ra_full_attention_paged(_query(n_seq, n_kv, dtype), cache))
    for s in sorted({0, n_seq - 1}):
        for h in range(n_kv):
            _check(out[s, h], lse[s, h], np.arange(N), low, rows_V[:, h], 8192 if n_seq == 200 else 1024)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n_seq,N,window,each", [(1, 131072, 131008, 64), (32, 8192, 8128, 128), (130, 704, 640, 1 << 20)])
def test_static_and_retrieved_attention(dtype, n_seq, N, window, each):
    """Parts of a job that begin with lower rows (every second, the first or its only one), and a retrieved row among the higher."""
    W = np.arange(N - window, N)
    low = np.zeros(N, bool)
    low[W[np.arange(window) // 16 % each < 16]] = True
    K, V, rows_V = _inputs(N, 1, low, 2)
    V[0, :, 5, :32] = 40.0                                  # the retrieved row's
    rows_V[5, :, :32] = 40.0
    table = torch.arange(N // 64, dtype=torch.int32, device=DEV).expand(n_seq, -1).contiguous()
    cache = ra.PagedCache(K.to(dtype).to(DEV), V.to(dtype).to(DEV), table)
    ids = ints([[[5]]]).expand(n_seq, 1, 1).contiguous()
    got = [t.cpu().numpy() for t in ra.ra_attend_paged(_query(n_seq, 1, dtype), cache, 0, window, ids, partials=True)]
    for s in sorted({0, n_seq - 1}):
        for (o, l), rows in zip((got[0:2], got[2:4], got[4:6]), (np.r_[5, W], np.array([5]), W)):
            _check(o[s, 0], l[s, 0], rows, low, rows_V[:, 0], 4096)
