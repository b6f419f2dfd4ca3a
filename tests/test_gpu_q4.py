"""Attention over a cache in 4 bits (ra_full_attention_q4, ra_attend_q4) against the oracle's attention in float64 on the
values that the rows stand for, within bounds that follow from the roundings."""
import numpy as np
import pytest
import torch

import paper_2409_10516_amd as ra
from oracle import attention as OA, decode as OD, kv4 as OK, quant as OQ, search as OS
from paper_2409_10516_amd import binding as B, synth
from tests.util import oracle_graphs, to_np, walk_equivalent

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


def _bounds(q, K, V, ids, dtype):
    """(out, its bound, lse, its bound) of Eq. 2 over rows ids. A logit is a float32 sum of 128 products and is scaled (at most
    132 roundings of 2^-24 of the magnitudes summed), subtracted from the maximum and exponentiated (4 of 2^-24 times either's size,
    and 4 for the exponential): e_i of a weight's relative error. Weights meet values with 16 bits of mantissa for bfloat16 (two
    parts of half a step each: 2^-16) and 24 for float32; sums of N terms in any order lose at most N 2^-24 of the magnitudes, and
    the factors of the running maximum and the division a few more. A weight (the largest is 1, and so their sum is no less), or a
    part of one, below the least normal number 2^-126 may become zero: three parts, of 2^-126 of its value each."""
    o, lse = OA.partial_attention(q, K, V, ids)
    if len(ids) == 0:
        return o, np.zeros_like(o), lse, 0.0
    q, K, V = (np.asarray(x, np.float64) for x in (q, K[ids], V[ids]))
    z = K @ q / np.sqrt(128)
    w = np.exp(z - lse)
    size = np.abs(K) @ np.abs(q) / np.sqrt(128)
    e = U * (132 * size + 4 * (np.abs(z) + np.abs(z).max()) + 4)
    mean = w @ e
    more = (2.0 ** -16 if dtype == torch.bfloat16 else 0.0) + (len(ids) + 64) * U
    bound = 1.01 * ((w * (e + mean + more)) @ np.abs(V)) + 3 * 2.0 ** -126 * np.abs(V).sum(axis=0)
    return o, bound, lse, 1.01 * (mean + (len(ids) + 64) * U + 4 * U * abs(lse))


def _check(out, lse, q, K, V, ids, dtype):
    o, ob, l, lb = _bounds(q, K, V, ids, dtype)
    if len(ids) == 0:
        assert (out == 0).all() and np.isneginf(lse)
        return
    far = np.abs(out - o) / np.maximum(ob, 1e-300)
    if not far.max() <= 1.0:
        raise AssertionError(f"{far.max():.3g} times the bound at {far.argmax()}")
    assert abs(lse - l) <= lb, (lse, l, lb)


def _cache(n_seq, n_kv, cap, seed, junk=()):
    """A cache of random rows with means of their own, as (codes, scale) pairs on the GPU and float64 values; rows `junk[s]` on of
    sequence s hold anything, NaN scales among it."""
    rng = np.random.default_rng(seed)
    x4, vals = [], []
    for which in range(2):
        x = rng.standard_normal((n_seq, n_kv, cap, 128)) * np.exp(0.5 * rng.standard_normal((n_seq, n_kv, 1, 128)))
        if which == 0:
            x = x + rng.standard_normal((n_seq, n_kv, 1, 128)) / 3
        unit = np.exp2(np.ceil(np.log2(np.abs(x).reshape(n_seq, n_kv, cap, 4, 32).max(-1) / 6)))
        y = np.abs(x) / np.repeat(unit, 32, axis=-1)
        code = np.abs(y[..., None] - OK.GRID).argmin(-1).astype(np.uint8) + 8 * (x < 0).astype(np.uint8)
        codes, scale = code[..., 0::2] | (code[..., 1::2] << 4), (np.log2(unit) + 127).astype(np.uint8)
        for s, n in enumerate(junk):
            codes[s, :, n:] = rng.integers(0, 256, codes[s, :, n:].shape)
            scale[s, :, n:] = rng.choice([0, 1, 254, 255], scale[s, :, n:].shape)
        x4.append((torch.from_numpy(codes).to(DEV), torch.from_numpy(scale).to(DEV)))
        vals.append(OK.dequantize_rows(codes, scale))
    return x4[0], x4[1], vals[0], vals[1]


def _queries(n_seq, n_q, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return (2.0 * torch.randn((n_seq, n_q, 128), generator=g)).to(dtype)


HEADS = [(1, 1), (2, 1), (3, 1), (8, 2), (5, 1), (7, 1), (8, 1), (9, 1), (16, 1), (4, 4), (20, 1)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n_q,n_kv", HEADS)
@pytest.mark.parametrize("N,cap", [(1, 1), (37, 40), (700, 701)])
def test_full_attention_of_any_group(dtype, n_q, n_kv, N, cap):
    k4, v4, K, V = _cache(2, n_kv, cap, seed=N + n_q, junk=(N, N))
    q = _queries(2, n_q, dtype, N)
    out, lse = ra.ra_full_attention_q4(q.to(DEV), k4, v4, N=N)
    out, lse = out.cpu().numpy(), lse.cpu().numpy()
    for s in range(2):
        for h in range(n_q):
            g = h // (n_q // n_kv)
            _check(out[s, h], lse[s, h], to_np(q[s, h]), K[s, g], V[s, g], np.arange(N), dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N", [2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 1000, 1023, 1025, 2049, 5003])
def test_full_attention_of_any_length(dtype, N):
    """Every length around the edges of tiles, each sequence with its own, rows behind the last full of junk."""
    lens = [N, N - 1, 0, 1, N // 2]
    k4, v4, K, V = _cache(5, 1, N + 3, seed=N, junk=lens)
    q = _queries(5, 4, dtype, N)
    n_tokens = torch.tensor([N, N - 1, 0, 1, N // 2], dtype=torch.int32, device=DEV)
    out, lse = ra.ra_full_attention_q4(q.to(DEV), k4, v4, n_tokens, N=N)
    out, lse = out.cpu().numpy(), lse.cpu().numpy()
    for s, n in enumerate(lens):
        for h in range(0, 4, 3):
            _check(out[s, h], lse[s, h], to_np(q[s, h]), K[s, 0], V[s, 0], np.arange(n), dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n_seq,n_q,n_kv,N", [(130, 4, 1, 700), (67, 1, 1, 300), (2100, 1, 1, 300), (1030, 2, 2, 257), (2, 40, 1, 3000), (1, 2, 1, 20001),
                                             (1, 17, 1, 40000), (3, 3, 1, 9999), (300, 8, 4, 2500), (2060, 1, 1, 33001)])
def test_full_attention_of_many_sequences_heads_and_records(dtype, n_seq, n_q, n_kv, N):
    """More sequences than lanes, more jobs than are cut, tiles of heads, more records of a head than one thread per dimension
    combines; lengths of zero, one and anything, some of them in a row."""
    rng = np.random.default_rng(N)
    lens = rng.integers(0, N + 1, n_seq)
    lens[rng.random(n_seq) < 0.3] = 0
    lens[-1] = N
    if n_seq > 4:
        lens[1], lens[2], lens[n_seq // 2:n_seq // 2 + 3] = 1, 129, 0
    k4, v4, K, V = _cache(1, n_kv, N, seed=N)                # (the same rows for all sequences)
    k4, v4 = (tuple(t.expand(n_seq, -1, -1, -1).contiguous() for t in x) for x in (k4, v4))
    q = _queries(n_seq, n_q, dtype, N)
    out, lse = ra.ra_full_attention_q4(q.to(DEV), k4, v4, torch.from_numpy(lens.astype(np.int32)).to(DEV))
    out, lse = out.cpu().numpy(), lse.cpu().numpy()
    assert (out[lens == 0] == 0).all() and np.isneginf(lse[lens == 0]).all() and np.isfinite(lse[lens > 0]).all()
    some = {0, 1, 2, n_seq - 1} | set(rng.integers(0, n_seq, 6).tolist())
    for s in sorted(x for x in some if x < n_seq):
        for h in sorted({0, n_q // 2, n_q - 1}):
            g = h // (n_q // n_kv)
            _check(out[s, h], lse[s, h], to_np(q[s, h]), K[0, g], V[0, g], np.arange(lens[s]), dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n_seq,n_q,n_kv,N", [(20, 2, 1, 9000), (40, 17, 1, 40001), (10, 4, 2, 50000), (66, 4, 1, 200003)])
def test_full_attention_of_one_long_sequence_in_a_batch(dtype, n_seq, n_q, n_kv, N):
    """The long one's heads have nearly all the records there are: more than a thread per dimension, than the groups of a workgroup in
    one go, and than a workgroup has threads; the others have one, or none."""
    lens = np.full(n_seq, 200, np.int32)
    lens[1], lens[2], lens[n_seq // 2] = 0, 1, N
    k4, v4, K, V = _cache(1, n_kv, N, seed=N)
    k4, v4 = (tuple(t.expand(n_seq, -1, -1, -1).contiguous() for t in x) for x in (k4, v4))
    q = _queries(n_seq, n_q, dtype, N)
    out, lse = ra.ra_full_attention_q4(q.to(DEV), k4, v4, torch.from_numpy(lens).to(DEV))
    out, lse = out.cpu().numpy(), lse.cpu().numpy()
    for s in (0, 1, 2, n_seq // 2, n_seq - 1):
        for h in sorted({0, n_q // 2, n_q - 1}):
            g = h // (n_q // n_kv)
            _check(out[s, h], lse[s, h], to_np(q[s, h]), K[0, g], V[0, g], np.arange(lens[s]), dtype)


def test_a_capacity_of_hundreds_of_millions():
    """The list of rows is counted in larger units then; most of the capacity is not used."""
    cap, T = 300_000_000, 6001
    k4, v4 = ((torch.empty((1, 1, cap, 64), dtype=torch.uint8, device=DEV), torch.empty((1, 1, cap, 4), dtype=torch.uint8, device=DEV))
              for _ in range(2))
    a4, b4, K, V = _cache(1, 1, T, seed=4)
    for x, y in ((k4, a4), (v4, b4)):
        for s, t in zip(x, y):
            s[:, :, :T] = t
    q = _queries(1, 3, torch.bfloat16, 4)
    out, lse = ra.ra_full_attention_q4(q.to(DEV), k4, v4, torch.tensor([T], dtype=torch.int32, device=DEV))
    for h in range(3):
        _check(out[0, h].cpu().numpy(), float(lse[0, h]), to_np(q[0, h]), K[0, 0], V[0, 0], np.arange(T), torch.bfloat16)


def test_lengths_outside_the_cache_are_cut():
    k4, v4, K, V = _cache(3, 2, 90, seed=1)
    q = _queries(3, 4, torch.float32, 1)
    n = torch.tensor([1 << 30, -5, 90], dtype=torch.int32, device=DEV)
    out, lse = ra.ra_full_attention_q4(q.to(DEV), k4, v4, n, N=80)
    for s, m in enumerate((80, 0, 80)):
        _check(out[s, 1].cpu().numpy(), float(lse[s, 1]), to_np(q[s, 1]), K[s, 0], V[s, 0], np.arange(m), torch.float32)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_large_logits_and_a_dominating_row(dtype):
    """Logits of hundreds: one row has all the weight, first, in the middle or last."""
    for at in (0, 300, 599):
        k4, v4, K, V = _cache(1, 1, 600, seed=at)
        q = torch.from_numpy(K[0, 0, at] * 20).to(dtype).reshape(1, 1, 128).repeat(1, 4, 1)
        q[0, 1] = -q[0, 1]
        q[0, 2] = 0
        out, lse = ra.ra_full_attention_q4(q.to(DEV), k4, v4)
        for h in range(4):
            _check(out[0, h].cpu().numpy(), float(lse[0, h]), to_np(q[0, h]), K[0, 0], V[0, 0], np.arange(600), dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_nan_rows_and_queries_stay_where_they_belong(dtype):
    k4, v4, K, V = _cache(2, 2, 300, seed=3)
    q = _queries(2, 8, dtype, 3)
    q[1, 7, 3] = float("nan")
    q[1, 6, 3] = float("inf")
    k4[1][0, 1, 200, 2] = 255                   # a key of sequence 0, KV head 1
    v4[1][1, 0, 77, 1] = 255                    # a block of a value of sequence 1, KV head 0
    out, lse = ra.ra_full_attention_q4(q.to(DEV), k4, v4)
    out, lse = out.cpu(), lse.cpu()
    assert torch.isnan(out[0, 4:]).all() and torch.isnan(lse[0, 4:]).all()
    bad = torch.isnan(out[1, :4])
    assert bad[:, 32:64].all() and not bad[:, :32].any() and not bad[:, 64:].any() and torch.isfinite(lse[1, :4]).all()
    assert torch.isnan(out[1, 6:]).all() and torch.isnan(lse[1, 6:]).all()
    for s, hs in ((0, (0, 1, 2, 3)), (1, (4, 5))):
        for h in hs:
            _check(out[s, h].numpy(), float(lse[s, h]), to_np(q[s, h]), K[s, h // 4], V[s, h // 4], np.arange(300), dtype)


def test_same_call_same_bits_and_views_at_odd_rows():
    k4, v4, K, V = _cache(1, 1, 3001, seed=9)
    q = _queries(1, 8, torch.bfloat16, 9).to(DEV)
    a = ra.ra_full_attention_q4(q, k4, v4)
    for _ in range(3):
        b = ra.ra_full_attention_q4(q, k4, v4)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    part = lambda x: tuple(t[:, :, 1:] for t in x)  # noqa: E731    (one head: contiguous, codes at 64, scales at 4 bytes)
    out, lse = ra.ra_full_attention_q4(q, part(k4), part(v4))
    for h in (0, 7):
        _check(out[0, h].cpu().numpy(), float(lse[0, h]), to_np(q[0, h]), K[0, 0], V[0, 0], np.arange(1, 3001), torch.bfloat16)


def test_rows_past_four_gigabytes():
    """The second head's rows start 4.5 GB into the codes; its rows are written and read there."""
    cap, T = 70_000_000, 50
    k4, v4 = ((torch.empty((1, 2, cap, 64), dtype=torch.uint8, device=DEV), torch.empty((1, 2, cap, 4), dtype=torch.uint8, device=DEV))
              for _ in range(2))
    g = torch.Generator().manual_seed(2)
    k, v = (torch.randn((1, T, 2, 128), generator=g) for _ in range(2))
    q = _queries(1, 2, torch.float32, 2)
    ra.ra_append_tokens(None, k.to(DEV), v.to(DEV), None, k4=k4, v4=v4)
    end = torch.tensor([cap - 20], dtype=torch.int32, device=DEV)
    ra.ra_append_tokens(None, k[:, :20].contiguous().to(DEV), v[:, :20].contiguous().to(DEV), end, k4=k4, v4=v4)
    n = torch.tensor([T], dtype=torch.int32, device=DEV)
    out, lse = ra.ra_full_attention_q4(q.to(DEV), k4, v4, n, N=64)
    back = to_np(ra.ra_dequantize_kv4(k4, torch.float32, first=end, rows=20))
    for h in range(2):
        K, V = (OK.dequantize_rows(*OK.quantize_rows(x[0, :, h].numpy())) for x in (k, v))
        assert np.array_equal(back[0, h], K[:20])
        _check(out[0, h].cpu().numpy(), float(lse[0, h]), to_np(q[0, h]), K, V, np.arange(T), torch.float32)


def _handle(n_seq, n_q, n_kv, N):
    """ra_attend_q4 takes sizes and workspace from a handle and reads no graph."""
    return ra.ra_index_import(torch.full((n_seq * n_q, N, 2), -1, dtype=torch.int32), torch.zeros(n_seq * n_q, dtype=torch.int32), n_seq,
                              n_q, n_kv)


ATTEND = [
    # n_seq, n_q, n_kv, N, index covers, capacity, sink, window, topk
    (1, 32, 8, 2000, 2000, 2000, 4, 640, 100),
    (2, 4, 2, 300, 300, 333, 4, 64, 1),
    (3, 8, 1, 500, 460, 512, 0, 0, 33),           # static: what came after the index
    (1, 6, 2, 700, 650, 700, 4, 10, 129),
    (2, 3, 3, 90, 90, 90, 100, 100, 7),           # everything static
    (1, 5, 1, 1500, 1500, 1500, 0, 0, 200),       # nothing static
    (4, 16, 2, 260, 200, 264, 1, 31, 64),
    (1, 20, 1, 4000, 4000, 4000, 128, 1400, 300),
    # long static sets: several chunks of a wavefront side by side, sinks that end inside one, many records of a head, one record
    (1, 16, 1, 40001, 3001, 40003, 4, 640, 100),
    (2, 8, 2, 9001, 2000, 9001, 4, 500, 40),
    (5, 20, 2, 5003, 900, 5003, 700, 31, 64),
    (1, 4, 1, 20011, 500, 20011, 333, 17, 9),
    (40, 16, 2, 2100, 300, 2100, 3, 20, 50),
    (30, 32, 1, 700, 300, 700, 5, 20, 40),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("case", ATTEND)
def test_sparse_and_static_attention(case, dtype):
    n_seq, n_q, n_kv, N, Ng, cap, sink, window, topk = case
    k4, v4, K, V = _cache(n_seq, n_kv, cap, seed=N + topk, junk=[N] * n_seq)
    q = _queries(n_seq, n_q, dtype, N)
    W = OA.static_ids(N, sink, min(window, N), Ng)
    rest = np.setdiff1d(np.arange(Ng), W)
    rng = np.random.default_rng(N)
    ids = -np.ones((n_seq, n_q, topk), np.int32)
    for s in range(n_seq):
        for h in range(n_q):
            n = min(len(rest), 0 if h == 1 else topk - (s + h) % 4)
            at = np.sort(rng.choice(topk, max(n, 0), replace=False)) if h % 2 else np.arange(max(n, 0))     # padding anywhere
            ids[s, h, at] = rng.choice(rest, size=max(n, 0), replace=False)
    given = ids.copy()
    given[(ids < 0) & (rng.random(ids.shape) < 0.5)] = N + 5                     # ids past the cache are skipped like -1
    idx = _handle(n_seq, n_q, n_kv, Ng)
    got = [t.cpu().numpy() for t in ra.ra_attend_q4(q.to(DEV), idx, k4, v4, sink, window, torch.from_numpy(given).to(DEV), N=N,
                                                    partials=True)]
    for s in range(n_seq):
        for h in range(n_q):
            g = h // (n_q // n_kv)
            qq, om = to_np(q[s, h]), ids[s, h][ids[s, h] >= 0]
            both = np.concatenate([W, om]).astype(np.int64)
            for (o, l), rows in zip((got[0:2], got[2:4], got[4:6]), (both, om, W)):
                _check(o[s, h], l[s, h], qq, K[s, g], V[s, g], rows, dtype)
    again = ra.ra_attend_q4(q.to(DEV), idx, k4, v4, sink, window, torch.from_numpy(given).to(DEV), N=N)
    assert np.array_equal(again[0].cpu().numpy(), got[0]) and np.array_equal(again[1].cpu().numpy(), got[1])
    idx.free()


def test_an_id_given_twice_counts_twice_and_a_nan_row_makes_nan():
    k4, v4, K, V = _cache(1, 1, 200, seed=5)
    q = _queries(1, 2, torch.float32, 5)
    idx = _handle(1, 2, 1, 200)
    ids = torch.tensor([[[50, 60, 50, -1], [70, -1, -1, -1]]], dtype=torch.int32, device=DEV)
    out, lse = ra.ra_attend_q4(q.to(DEV), idx, k4, v4, 3, 20, ids)
    W = OA.static_ids(200, 3, 20)
    _check(out[0, 0].cpu().numpy(), float(lse[0, 0]), to_np(q[0, 0]), K[0, 0], V[0, 0], np.concatenate([W, [50, 60, 50]]), torch.float32)
    k4[1][0, 0, 70, 0] = 255
    out, lse = ra.ra_attend_q4(q.to(DEV), idx, k4, v4, 3, 20, ids)
    assert torch.isnan(out[0, 1]).all() and torch.isnan(lse[0, 1]) and torch.isfinite(out[0, 0]).all()
    idx.free()


def test_refusals():
    k4, v4, _, _ = _cache(1, 2, 64, seed=1)
    q = _queries(1, 4, torch.float32, 1).to(DEV)
    idx = _handle(1, 4, 2, 60)
    ids = torch.zeros((1, 4, 5), dtype=torch.int32, device=DEV) + 30
    other = tuple(t[:, :, :60].contiguous() for t in v4)
    with pytest.raises(ValueError):
        ra.ra_full_attention_q4(q, k4, other)
    with pytest.raises(ra.RaError):
        ra.ra_full_attention_q4(q, k4, v4, N=65)
    with pytest.raises(ra.RaError):
        ra.ra_full_attention_q4(q[:, :3].contiguous(), k4, v4)
    with pytest.raises(ValueError):
        ra.ra_full_attention_q4(q, k4, v4, torch.tensor([5], device=DEV))
    with pytest.raises(ra.RaError) as e:
        ra.ra_full_attention_q4(q, k4, v4, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
    assert e.value.status == 2
    with pytest.raises(ValueError):
        ra.ra_full_attention_q4(q, k4, v4, out=torch.empty((1, 4, 128), dtype=torch.float64, device=DEV))
    with pytest.raises(TypeError):
        ra.ra_full_attention_q4(q.half(), k4, v4)
    with pytest.raises(ra.RaError):
        ra.ra_attend_q4(q, idx, k4, v4, 4, 8, ids, N=59)                 # fewer than the index covers
    with pytest.raises(ra.RaError):
        ra.ra_attend_q4(q, idx, k4, v4, 4, 8, ids, N=65)                 # more than there is room for
    with pytest.raises(ra.RaError):
        ra.ra_attend_q4(q, idx, k4, v4, -1, 8, ids)
    with pytest.raises(ValueError):
        ra.ra_attend_q4(q, idx, k4, v4, 4, 8, ids.long())
    with pytest.raises(ValueError):
        ra.ra_attend_q4(q[:, :2].contiguous(), idx, k4, v4, 4, 8, ids)
    idx.free()


def test_prompt_index_walk_and_decode_over_4bit_rows():
    """The set as a serving loop uses it: a prompt is normed, rotated and put into the caches, the index is built over
    its keys, they get their 8-bit copy for the walk, and from then on only 4-bit rows are kept: decoded tokens are appended to them and
    attend by walk + sparse attention, and by full attention."""
    n_q, n_kv, N, cap, sink, window, topk, ef, deg, knn = 4, 2, 600, 620, 4, 50, 16, 48, 12, 12
    g = torch.Generator().manual_seed(11)
    tokens = lambda n: torch.randn((1, n, n_q + 2 * n_kv, 128), generator=g).bfloat16().to(DEV).split((n_q, n_kv, n_kv), dim=2)  # noqa: E731
    w = (1 + 0.2 * torch.randn(128, generator=g)).bfloat16().to(DEV)
    f = torch.from_numpy((10000.0 ** (-np.arange(0, 128, 2) / 128)).astype(np.float32)).to(DEV)
    opt = dict(q_weight=w, k_weight=w, inv_freq=f)
    K = torch.zeros((1, n_kv, N, 128), dtype=torch.bfloat16, device=DEV)
    k4, v4 = ((torch.zeros((1, n_kv, cap, 64), dtype=torch.uint8, device=DEV), torch.zeros((1, n_kv, cap, 4), dtype=torch.uint8, device=DEV))
              for _ in range(2))
    q, k, v = tokens(N)
    Qp = ra.ra_append_tokens(q, k, v, None, K=K, v4=v4, **opt)
    ra.ra_quantize_kv4(K, out=k4)
    idx = ra.ra_build_index(K, Qp, deg, knn)
    k8 = ra.ra_quantize_keys(K)
    pos = torch.full((1,), N, dtype=torch.int32, device=DEV)
    r8, rs = zip(*[OQ.quantize_keys(to_np(K[0, i])) for i in range(n_kv)])
    del K
    for step in range(4):
        q, k, v = tokens(1)
        qd = ra.ra_append_tokens(q, k, v, pos, k4=k4, v4=v4, **opt).squeeze(2)
        pos += 1
        n = N + step + 1
        ids, st = ra.ra_search(qd, idx, None, sink, window, topk, ef, 4, k8=k8)
        out, lse = ra.ra_attend_q4(qd, idx, k4, v4, sink, window, ids, N=n)
        full, full_lse = ra.ra_full_attention_q4(qd, k4, v4, pos)
        Kv, Vv = (OK.dequantize_rows(*(t[0].cpu().numpy() for t in x4)) for x4 in (k4, v4))
        for h in range(n_q):
            i = h // (n_q // n_kv)
            qq = to_np(qd[0, h])
            adj, ent = ra.ra_index_export(idx, 0, h)
            r_ids, rst = OS.greedy_search(OQ.scaled_query(qq, rs[i]), r8[i].astype(np.float32), adj.numpy(), ent, ef, topk, 4,
                                          exclude=OA.static_ids(N, sink, window))
            got = ids[0, h].cpu().numpy()
            walk_equivalent(got, None, r_ids, rst, OQ.scaled_query(qq, rs[i]), r8[i].astype(np.float32), OA.static_ids(N, sink, window))
            W = OA.static_ids(n, sink, window, N)
            om = np.setdiff1d(got[got >= 0], W)
            assert len(om) == (got >= 0).sum()
            _check(out[0, h].cpu().numpy(), float(lse[0, h]), qq, Kv[i], Vv[i], np.concatenate([W, om]), torch.bfloat16)
            _check(full[0, h].cpu().numpy(), float(full_lse[0, h]), qq, Kv[i], Vv[i], np.arange(n), torch.bfloat16)
    idx.free()


def test_captured_token_replays_as_positions_advance():
    """Append and both attentions in one captured graph, positions and lengths in device memory: every replay, with eager work
    between them, against the eager calls on a copy of the caches."""
    n_seq, n_q, n_kv, cap = 2, 8, 2, 400
    k4, v4, _, _ = _cache(n_seq, n_kv, cap, seed=13)
    mine = [tuple(t.clone() for t in x) for x in (k4, v4)]
    idx, ref_idx = _handle(n_seq, n_q, n_kv, 100), _handle(n_seq, n_q, n_kv, 100)
    f = torch.from_numpy((10000.0 ** (-np.arange(0, 128, 2) / 128)).astype(np.float32)).to(DEV)
    x = torch.zeros((n_seq, 1, n_q + 2 * n_kv, 128), dtype=torch.bfloat16, device=DEV)
    q, k, v = x.split((n_q, n_kv, n_kv), dim=2)
    pos = torch.tensor([120, 391], dtype=torch.int32, device=DEV)
    ids = torch.randint(10, 60, (n_seq, n_q, 20), dtype=torch.int32, device=DEV)
    q_out = torch.zeros((n_seq, n_q, 1, 128), dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(B.lib().ra_full_attention_q4_workspace_bytes(B.RA_BF16, n_seq, n_q, n_kv, cap), dtype=torch.uint8, device=DEV)
    res = [(torch.empty((n_seq, n_q, 128), device=DEV), torch.empty((n_seq, n_q), device=DEV)) for _ in range(2)]

    def token(cache, handle, results, room):
        ra.ra_append_tokens(q, k, v, pos, inv_freq=f, q_out=q_out, k4=cache[0], v4=cache[1])
        pos.add_(1)
        ra.ra_full_attention_q4(q_out.squeeze(2), *cache, pos, workspace=room, out=results[0][0], lse=results[0][1])
        ra.ra_attend_q4(q_out.squeeze(2), handle, *cache, 4, 32, ids, N=cap - 200, out=results[1][0], lse=results[1][1])

    start = pos.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        token(mine, idx, res, ws)                       # (the handle's workspace grows before the capture)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for a, b in zip(mine, (k4, v4)):
        for c, d in zip(a, b):
            c.copy_(d)
    pos.copy_(start)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        token(mine, idx, res, ws)
    pos.copy_(start)
    for step in range(12):                              # (the second sequence runs into the end of its cache)
        x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(step)).to(DEV))
        here = pos.clone()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for r in res for t in r]
        after = pos.clone()
        pos.copy_(here)
        eager = [(torch.empty_like(o), torch.empty_like(m)) for o, m in res]
        token((k4, v4), ref_idx, eager, torch.empty_like(ws))
        assert torch.equal(pos, after)
        for a, b in zip(got, [t for r in eager for t in r]):
            assert torch.equal(a, b), step
        for a, b in zip(mine, (k4, v4)):
            assert all(torch.equal(c, d) for c, d in zip(a, b))
    idx.free()
    ref_idx.free()


def test_a_captured_call_outlives_the_growth_of_its_workspace():
    """A larger call on the handle takes a larger workspace; a graph captured before goes on with its own."""
    k4, v4, _, _ = _cache(1, 1, 3000, seed=31)
    idx = _handle(1, 4, 1, 3000)
    q = _queries(1, 4, torch.bfloat16, 31).to(DEV)
    ids = torch.randint(10, 2000, (1, 4, 300), dtype=torch.int32, device=DEV)
    ref = [t.clone() for t in ra.ra_attend_q4(q, idx, k4, v4, 4, 100, ids)]
    out, lse = torch.empty_like(ref[0]), torch.empty_like(ref[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ra.ra_attend_q4(q, idx, k4, v4, 4, 100, ids, out=out, lse=lse)
    before = idx.device_bytes
    big = [t.clone() for t in ra.ra_attend_q4(q, idx, k4, v4, 4, 2500, ids[..., :200].contiguous())]
    assert idx.device_bytes > before
    keep = torch.full((1 << 20,), 3.0, device=DEV)
    for _ in range(4):
        out.fill_(float("nan"))
        lse.fill_(float("nan"))
        graph.replay()
        again = ra.ra_attend_q4(q, idx, k4, v4, 4, 2500, ids[..., :200].contiguous())
        torch.cuda.synchronize()
        assert torch.equal(out, ref[0]) and torch.equal(lse, ref[1])
        assert torch.equal(again[0], big[0]) and (keep == 3.0).all()
    idx.free()


def test_calls_on_their_own_streams():
    """Two streams at once, each with workspace and results of its own."""
    k4, v4, _, _ = _cache(2, 2, 5000, seed=21)
    qs = [_queries(2, 8, torch.bfloat16, 30 + i).to(DEV) for i in range(2)]
    refs = [ra.ra_full_attention_q4(q, k4, v4) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    need = B.lib().ra_full_attention_q4_workspace_bytes(B.RA_BF16, 2, 8, 2, 5000)
    room = [torch.empty(need, dtype=torch.uint8, device=DEV) for _ in range(2)]
    outs = [[(torch.empty((2, 8, 128), device=DEV), torch.empty((2, 8), device=DEV)) for _ in range(2)] for _ in range(10)]
    for turn in range(10):
        for i, st in enumerate(streams):
            ra.ra_full_attention_q4(qs[i], k4, v4, stream=st, workspace=room[i], out=outs[turn][i][0], lse=outs[turn][i][1])
    torch.cuda.synchronize()
    for turn in outs:
        for i in range(2):
            assert torch.equal(turn[i][0], refs[i][0]) and torch.equal(turn[i][1], refs[i][1])


def test_calls_on_a_stream_allocate_there():
    """A workspace that a call drops when it returns is not handed to the current stream while the call waits on its own."""
    k4, v4, _, _ = _cache(2, 2, 5000, seed=22)
    q = _queries(2, 8, torch.bfloat16, 33).to(DEV)
    ref = ra.ra_full_attention_q4(q, k4, v4)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    need = B.lib().ra_full_attention_q4_workspace_bytes(B.RA_BF16, 2, 8, 2, 5000)
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    got = ra.ra_full_attention_q4(q, k4, v4, stream=side)
    for _ in range(400):                                     # (work on the current stream, in memory of the workspace's size)
        torch.full((need // 4,), float("nan"), device=DEV)
    torch.cuda.synchronize()
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])


class _Elsewhere:
    """What a stream of another device looks like."""
    cuda_stream, device_index = 0, 7


def test_streams_of_another_device_are_refused():
    k4, v4, _, _ = _cache(1, 1, 40, seed=23)
    q = _queries(1, 4, torch.bfloat16, 34).to(DEV)
    for call in (lambda st: ra.ra_full_attention_q4(q, k4, v4, stream=st),
                 lambda st: ra.ra_append_tokens(q[:, None], None, None, None, stream=st),
                 lambda st: ra.ra_quantize_kv4(torch.zeros(1, 1, 4, 128, device=DEV), stream=st),
                 lambda st: ra.ra_dequantize_kv4(k4, torch.float32, stream=st)):
        with pytest.raises(ValueError, match="current GPU"):
            call(_Elsewhere())


def test_oracle_decode_step_is_what_the_parts_make():
    """On rows that 4 bits hold exactly, ids from the walk over the keys and ra_attend_q4 are the fused decode step."""
    w = synth.make_llama_layer(61, N=500, M=200, T=1, n_q=4, n_kv=2, ef=40, topk=12, window=40, deg=10, knn=10)
    back = {}
    for n, x in (("K", w.K), ("V", w.V)):
        x4 = ra.ra_quantize_kv4(x.to(DEV))
        back[n] = (x4, ra.ra_dequantize_kv4(x4, torch.bfloat16))
    w.K, w.V = back["K"][1].cpu(), back["V"][1].cpu()
    adj, ent, _ = oracle_graphs(w)
    idx = ra.ra_index_import(torch.from_numpy(adj), torch.from_numpy(ent), 1, 4, 2)
    q = w.q_decode[0].to(DEV)
    out, lse, ids, st = ra.ra_decode_step(q, idx, back["K"][1], back["V"][1], w.sink, w.window, w.topk, w.ef, 4)
    o4, l4 = ra.ra_attend_q4(q, idx, back["K"][0], back["V"][0], w.sink, w.window, ids)
    for h in range(4):
        Kf, Vf = to_np(w.K[0, h // 2]), to_np(w.V[0, h // 2])
        r_out, r_lse, r_ids, rst = OD.decode_step(to_np(w.q_decode[0, 0, h]), Kf, Vf, adj[h], ent[h], w.sink, w.window, w.topk, w.ef, 4)
        got = ids[0, h].cpu().numpy()
        both = np.concatenate([OA.static_ids(500, w.sink, w.window), got[got >= 0]])
        _check(o4[0, h].cpu().numpy(), float(l4[0, h]), to_np(w.q_decode[0, 0, h]), Kf, Vf, both, torch.bfloat16)
        assert np.abs(o4[0, h].cpu().numpy() - out[0, h].cpu().numpy()).max() <= 4e-3 * np.abs(r_out).max()
    idx.free()
