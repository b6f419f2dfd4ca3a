"""Tokens that enter a cache (ra_append_tokens) and rows in 4 bits (ra_quantize_kv4, ra_dequantize_kv4) against the float64
oracle (oracle/kv4.py): 4-bit rows and copies equal, normed and rotated rows within the roundings they are made of."""
import numpy as np
import pytest
import torch

import paper_2409_10516_amd as ra
from oracle import kv4 as OK
from tests.util import to_np

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U32 = 2.0 ** -24


def _np(t):
    return to_np(t) if t.is_floating_point() else t.cpu().numpy()


def _row_close(got, ref, size, dtype):
    """A value is n_a c - n_b s (or n): the norm's factor, two products with it, the sine or cosine, the product and the sum are
    rounded once each, 6 roundings of 2^-24 of the magnitudes summed (a further one for what is second order), then one to the
    type, of half a step."""
    last = 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
    tol = 7 * U32 * size + last * (np.abs(ref) + 7 * U32 * size)
    bad = np.abs(got.astype(np.float64) - ref) > tol
    assert not bad.any(), (int(bad.sum()), float(np.max(np.abs(got - ref))))


def _inv_freq(rot, base=500000.0):
    return (base ** (-np.arange(0, rot, 2) / max(rot, 1))).astype(np.float32)


CASES = [
    # dtype, n_seq, n_q, n_kv, T, capacity, first, n_new, rot, interleaved, norm
    ("bf16", 1, 32, 8, 1, 40, [7], None, 128, False, False),
    ("f32", 1, 1, 1, 1, 1, [0], None, 128, False, True),
    ("bf16", 3, 4, 2, 17, 64, [0, 40, 47], [17, 0, 5], 128, False, True),
    ("f32", 4, 6, 2, 5, 33, [28, 1, 30, -2], [5, 9, 5, 5], 64, True, True),        # rows outside the cache, more tokens than T
    ("bf16", 2, 7, 1, 33, 70, None, None, 96, False, True),
    ("f32", 2, 3, 3, 16, 16, None, [-1, 16], 16, False, False),
    ("bf16", 5, 2, 2, 1, 9, [8, 0, 9, 3, -1], None, 128, True, True),
    ("f32", 1, 16, 2, 130, 200, [70], None, 0, False, True),
    ("bf16", 1, 8, 4, 64, 64, [0], None, 32, True, False),
    ("f32", 1, 5, 5, 257, 300, [11], [250], 80, False, True),
]


@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("form", ["both", "4bit", "plain"])
def test_append(case, form):
    name, n_seq, n_q, n_kv, T, cap, first, n_new, rot, inter, norm = case
    dtype = torch.bfloat16 if name == "bf16" else torch.float32
    g = torch.Generator().manual_seed(T + 7 * n_q)
    heads = n_q + 2 * n_kv
    qkv = (torch.randn((n_seq, T, heads * 128), generator=g) * torch.exp(torch.randn((n_seq, T, heads, 1), generator=g)).expand(
        -1, -1, -1, 128).reshape(n_seq, T, -1)).to(dtype)
    w = [(1 + 0.3 * torch.randn(128, generator=g)).to(dtype) for _ in range(2)] if norm else [None, None]
    f = _inv_freq(rot) if rot else None
    dev = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    ints = lambda v: None if v is None else torch.tensor(v, dtype=torch.int32)  # noqa: E731
    q, k, v = dev(qkv).unflatten(-1, (heads, 128)).split((n_q, n_kv, n_kv), dim=2)
    old = {n: (torch.randn((n_seq, n_kv, cap, 128), generator=g).to(dtype)) for n in "KV"}
    old4 = {n: tuple(torch.randint(0, 250, (n_seq, n_kv, cap, c), generator=g, dtype=torch.uint8) for c in (64, 4)) for n in "KV"}
    C = {n: dev(t.clone()) for n, t in old.items()} if form != "4bit" else {}
    C4 = {n: tuple(dev(t.clone()) for t in x) for n, x in old4.items()} if form != "plain" else {}
    q_out = torch.full((n_seq, n_q, T, 128), 7.0, dtype=dtype, device=DEV)
    got = ra.ra_append_tokens(q, k, v, dev(ints(first)), n_new=dev(ints(n_new)), q_weight=dev(w[0]), k_weight=dev(w[1]), eps=1e-5,
                              inv_freq=None if f is None else torch.from_numpy(f).to(DEV), interleaved=inter, q_out=q_out,
                              K=C.get("K"), V=C.get("V"), k4=C4.get("K"), v4=C4.get("V"))
    torch.cuda.synchronize()
    assert got is q_out
    X = to_np(qkv).reshape(n_seq, T, heads, 128)
    for s in range(n_seq):
        f0 = 0 if first is None else first[s]
        n = T if n_new is None else max(0, min(n_new[s], T))
        pos = f0 + np.arange(T)
        ref, size = OK.head_rows(X[s, :, :n_q], pos, None if w[0] is None else to_np(w[0]), 1e-5, f, inter)
        go = _np(got[s])
        _row_close(go[:, :n].transpose(1, 0, 2), ref[:n], size[:n], dtype)
        assert (go[:, n:] == 7.0).all()
        kref, ksize = OK.head_rows(X[s, :, n_q:n_q + n_kv], pos, None if w[1] is None else to_np(w[1]), 1e-5, f, inter)
        there = [t for t in range(n) if 0 <= f0 + t < cap]
        rows = [f0 + t for t in there]
        rest = np.setdiff1d(np.arange(cap), rows)
        x = {"K": None, "V": X[s, :, n_q + n_kv:].transpose(1, 0, 2)[:, there]}
        for n_ in C:
            now = _np(C[n_][s])
            assert np.array_equal(now[:, rest], to_np(old[n_][s])[:, rest])
            if n_ == "V":
                assert np.array_equal(now[:, rows], x["V"])
            else:
                _row_close(now[:, rows].transpose(1, 0, 2), kref[there], ksize[there], dtype)
                x["K"] = now[:, rows]
        for n_ in C4:
            now = [_np(t[s]) for t in C4[n_]]
            for a, b in zip(now, old4[n_]):
                assert np.array_equal(a[:, rest], b[s].numpy()[:, rest])
            if x[n_] is not None:                       # (of the rows as they were rounded)
                for a, b in zip(now, OK.quantize_rows(x[n_])):
                    assert np.array_equal(a[:, rows], b)


def test_append_4bit_only_equals_append_of_both():
    g = torch.Generator().manual_seed(5)
    x = torch.randn((2, 37, 6, 128), generator=g).bfloat16().to(DEV)
    f = torch.from_numpy(_inv_freq(128)).to(DEV)
    first = torch.tensor([900000, 3], dtype=torch.int32, device=DEV)
    cap = 900040
    one, two = ((torch.zeros((2, 6, cap, 64), dtype=torch.uint8, device=DEV), torch.zeros((2, 6, cap, 4), dtype=torch.uint8, device=DEV))
                for _ in range(2))
    K = torch.zeros((2, 6, cap, 128), dtype=torch.bfloat16, device=DEV)
    ra.ra_append_tokens(None, x, None, first, inv_freq=f, k4=one)
    ra.ra_append_tokens(None, x, None, first, inv_freq=f, K=K, k4=two)
    assert all(torch.equal(a, b) for a, b in zip(one, two))
    ref, size = OK.head_rows(to_np(x[0]), 900000 + np.arange(37), inv_freq=_inv_freq(128))
    _row_close(to_np(K[0, :, 900000:900037]).transpose(1, 0, 2), ref, size, torch.bfloat16)


def test_append_of_parts():
    """Each of queries, keys and values by itself does what it does beside the others."""
    g = torch.Generator().manual_seed(6)
    q, k, v = (torch.randn((1, 9, h, 128), generator=g).to(DEV) for h in (4, 2, 2))
    f = torch.from_numpy(_inv_freq(128)).to(DEV)
    w = torch.rand(128, generator=g).to(DEV)
    K, V = (torch.zeros((1, 2, 9, 128), device=DEV) for _ in range(2))
    out = ra.ra_append_tokens(q, k, v, None, q_weight=w, k_weight=w, inv_freq=f, K=K, V=V)
    assert torch.equal(ra.ra_append_tokens(q, None, None, None, q_weight=w, inv_freq=f), out)
    K1, V1 = torch.zeros_like(K), torch.zeros_like(V)
    assert ra.ra_append_tokens(None, k, None, None, k_weight=w, inv_freq=f, K=K1) is None
    assert ra.ra_append_tokens(None, None, v, None, V=V1) is None
    assert torch.equal(K, K1) and torch.equal(V, V1)
    # rows behind the last token of a sequence, in a result that the call makes, are zero
    out = ra.ra_append_tokens(q, None, None, None, n_new=torch.tensor([4], dtype=torch.int32, device=DEV), inv_freq=f)
    assert out[:, :, 4:].abs().max() == 0 and out[:, :, :4].abs().max() > 0


def test_non_finite_values_stay_in_their_head():
    g = torch.Generator().manual_seed(8)
    k = torch.randn((1, 3, 4, 128), generator=g)
    k[0, 1, 2, 5], k[0, 2, 0, 100] = float("nan"), float("inf")
    k4 = (torch.zeros((1, 4, 3, 64), dtype=torch.uint8, device=DEV), torch.zeros((1, 4, 3, 4), dtype=torch.uint8, device=DEV))
    K = torch.zeros((1, 4, 3, 128), device=DEV)
    ra.ra_append_tokens(None, k.to(DEV), None, None, inv_freq=torch.from_numpy(_inv_freq(128)).to(DEV), K=K, k4=k4)
    bad = ~torch.isfinite(K).cpu()
    assert bad[0, 2, 1].nonzero().flatten().tolist() == [5, 69] and bad[0, 0, 2].nonzero().flatten().tolist() == [36, 100]
    assert bad.sum() == 4
    blocks = (k4[1] == 255).cpu()
    assert blocks[0, 2, 1].tolist() == [True, False, True, False] and blocks[0, 0, 2].tolist() == [False, True, False, True]
    assert blocks.sum() == 4


def _special_rows():
    """Rows at which rounding and scales can go wrong: every tie and its neighbours at every binade's edge, zeroes of both signs,
    tiny, huge and non-finite blocks."""
    rng = np.random.default_rng(3)
    base = np.array([m * s + d for m in (0, .25, .5, .75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6) for s in (1, -1)
                     for d in (0.0, 2.0 ** -20, -2.0 ** -20)], np.float32)
    rows = []
    for e in (-126, -125, -124, -40, -1, 0, 1, 17, 100, 124):
        for top in (6.0, 5.999, 3.0, 3.001, 4.5, 6.0000005):
            x = rng.choice(base, 128).astype(np.float64)
            x = np.clip(x, -top, top)
            x[rng.permutation(32)[0] + 32 * np.arange(4)] = top
            rows.append(x * 2.0 ** e)
    x = np.zeros((8, 128))
    x[0, :3] = [np.nan, 1, 2]
    x[1, 40] = np.inf
    x[2, 127] = -np.inf
    x[3, 0] = 2.0 ** 127
    x[4, 0] = 1.99 * 2.0 ** 126
    x[5, 64] = -0.0
    x[6] = 2.0 ** -149
    x[7, ::3] = 1e-39
    return np.concatenate([np.array(rows), x]).astype(np.float32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_into_4_bits_at_ties_edges_and_non_finite_values(dtype):
    X = torch.from_numpy(_special_rows()).to(dtype)
    codes, scale = ra.ra_quantize_kv4(X.to(DEV).reshape(1, 1, -1, 128))
    rc, rs = OK.quantize_rows(to_np(X))
    assert np.array_equal(_np(scale)[0, 0], rs)
    # (the sign of a zero is not looked at: -0.0 has a code of its own)
    assert np.array_equal(OK.dequantize_rows(_np(codes)[0, 0], rs), OK.dequantize_rows(rc, rs), equal_nan=True)
    assert np.array_equal(_np(codes)[0, 0], rc)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n_seq,n_kv,T", [(1, 1, 1), (3, 2, 77), (2, 8, 1001)])
def test_rows_into_4_bits_and_back(dtype, n_seq, n_kv, T):
    X = torch.randn((n_seq, n_kv, T, 128), generator=torch.Generator().manual_seed(T)).to(dtype)
    x4 = ra.ra_quantize_kv4(X.to(DEV))
    rc, rs = OK.quantize_rows(to_np(X))
    assert np.array_equal(_np(x4[0]), rc) and np.array_equal(_np(x4[1]), rs)
    back = ra.ra_dequantize_kv4(x4, dtype)
    assert np.array_equal(to_np(back).astype(np.float64), OK.dequantize_rows(rc, rs))
    again = ra.ra_quantize_kv4(back)
    assert torch.equal(ra.ra_dequantize_kv4(again, dtype), back)


def test_rows_go_where_first_and_n_new_say():
    n_seq, n_kv, T, cap = 5, 3, 21, 50
    g = torch.Generator().manual_seed(4)
    X = torch.randn((n_seq, n_kv, T, 128), generator=g)
    old = tuple(torch.randint(1, 250, (n_seq, n_kv, cap, c), generator=g, dtype=torch.uint8) for c in (64, 4))
    first, n_new = [0, 29, 45, -3, 10], [21, 50, 21, 21, 0]
    out = tuple(t.to(DEV) for t in old)
    got = ra.ra_quantize_kv4(X.to(DEV), first=torch.tensor(first, dtype=torch.int32, device=DEV),
                             n_new=torch.tensor(n_new, dtype=torch.int32, device=DEV), out=out)
    assert got is out
    want = [t.numpy().copy() for t in old]
    for s in range(n_seq):
        for t in range(min(n_new[s], T)):
            if 0 <= first[s] + t < cap:
                for a, b in zip(want, OK.quantize_rows(X[s, :, t].numpy())):
                    a[s, :, first[s] + t] = b
    assert all(np.array_equal(_np(a), b) for a, b in zip(out, want))
    back = ra.ra_dequantize_kv4(out, torch.float32, first=torch.tensor(first, dtype=torch.int32, device=DEV), rows=T)
    ref = np.zeros((n_seq, n_kv, T, 128))
    full = OK.dequantize_rows(*want)
    for s in range(n_seq):
        for t in range(T):
            if 0 <= first[s] + t < cap:
                ref[s, :, t] = full[s, :, first[s] + t]
    assert np.array_equal(_np(back).astype(np.float64), ref)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_every_code_with_every_scale(dtype):
    codes = torch.arange(256, dtype=torch.uint8).repeat(64).reshape(256, 64)
    scale = torch.arange(256, dtype=torch.uint8).reshape(256, 1).repeat(1, 4)
    got = to_np(ra.ra_dequantize_kv4((codes.reshape(1, 1, 256, 64).to(DEV), scale.reshape(1, 1, 256, 4).to(DEV)), dtype))[0, 0]
    ref = OK.dequantize_rows(codes.numpy(), scale.numpy())
    ok = slice(0, 253)          # (6 x 2^(253 - 127) is above the largest float32)
    assert np.array_equal(got[ok].astype(np.float64), ref[ok])
    assert np.isnan(got[255]).all()
    big = np.abs(ref[253:255]) > 3.4e38
    assert np.isinf(got[253:255][big]).all() and np.array_equal(got[253:255][~big].astype(np.float64), ref[253:255][~big])


def test_refusals():
    x4 = (torch.zeros((1, 2, 8, 64), dtype=torch.uint8, device=DEV), torch.zeros((1, 2, 8, 4), dtype=torch.uint8, device=DEV))
    X = torch.zeros((1, 2, 4, 128), device=DEV)
    qkv = torch.zeros((1, 4, 2, 128), device=DEV)
    one = torch.zeros(1, dtype=torch.int32, device=DEV)
    with pytest.raises(ValueError):
        ra.ra_quantize_kv4(X, first=one)
    with pytest.raises(ValueError):
        ra.ra_quantize_kv4(X, first=one.long(), out=x4)
    with pytest.raises(ValueError):
        ra.ra_quantize_kv4(X.transpose(2, 3), out=x4)
    with pytest.raises(ValueError):
        ra.ra_quantize_kv4(X, out=(x4[0], x4[1][:, :, :4]))
    with pytest.raises(TypeError):
        ra.ra_quantize_kv4(X.half(), out=x4)
    with pytest.raises(TypeError):
        ra.ra_dequantize_kv4(x4, torch.float16)
    with pytest.raises(ra.RaError):
        ra.ra_quantize_kv4(torch.zeros((1, 2, 4, 64), device=DEV), out=x4)
    with pytest.raises(ValueError):
        ra.ra_append_tokens(None, qkv, None, None, k4=(x4[0].transpose(1, 2), x4[1]))
    with pytest.raises(ra.RaError):
        ra.ra_append_tokens(qkv, qkv, qkv, None)                       # keys without a cache
    with pytest.raises(TypeError):
        ra.ra_append_tokens(qkv, qkv.bfloat16(), None, None, k4=x4)
    with pytest.raises(ValueError):
        ra.ra_append_tokens(qkv.transpose(1, 2), None, None, None)     # heads not side by side
    with pytest.raises(ValueError):
        ra.ra_append_tokens(qkv, None, None, None, q_weight=torch.ones(64, device=DEV))
    with pytest.raises(ValueError):
        ra.ra_append_tokens(qkv, None, None, None, inv_freq=torch.ones(64, device=DEV, dtype=torch.float64))
    with pytest.raises(ra.RaError):
        ra.ra_append_tokens(qkv, None, None, None, inv_freq=torch.ones(12, device=DEV))      # 24 dimensions
    with pytest.raises(ValueError):
        ra.ra_append_tokens(qkv.expand(1, 4, 2, 128)[:, :1].expand(1, 4, 2, 128).cpu(), None, None, None)
    with pytest.raises(ra.RaError):
        ra.ra_append_tokens(qkv[:, :1].expand(1, 4, 2, 128), None, None, None)               # tokens on top of each other


def test_rows_behind_the_last_token_are_zero_on_another_stream():
    """The zeroes of a q_out that the call makes come before its rows, whatever the current stream is waiting for."""
    x = torch.randn((2, 9, 4, 128), device=DEV)
    n_new = torch.tensor([9, 4], dtype=torch.int32, device=DEV)
    ref = ra.ra_append_tokens(x, None, None, None, n_new=n_new)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    torch.cuda._sleep(20_000_000)
    got = ra.ra_append_tokens(x, None, None, None, n_new=n_new, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got, ref) and (got[1, :, 4:] == 0).all() and torch.equal(got[1, :, :4], x[1, :4].transpose(0, 1))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n_q,n_kv,T,rot,inter", [(1, 1, 9001, 128, False), (6, 2, 8209, 64, True), (16, 2, 8200, 128, True), (28, 4, 2100, 96, False),
                                                 (32, 8, 2049, 128, False), (5, 5, 2500, 16, False), (64, 8, 300, 64, False)])
def test_append_of_many_tokens(dtype, n_q, n_kv, T, rot, inter):
    """As many tokens as change the workgroups' size: every copied row, and normed and rotated rows of some tokens."""
    g = torch.Generator(device=DEV).manual_seed(T)
    heads = n_q + 2 * n_kv
    x = torch.randn((2, T, heads, 128), generator=g, device=DEV).to(dtype)
    q, k, v = x.split((n_q, n_kv, n_kv), dim=2)
    w = [(1 + 0.3 * torch.randn(128, generator=g, device=DEV)).to(dtype) for _ in range(2)]
    f = _inv_freq(rot)
    first, n_new = [5, 0], [T, T - 37]
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
    K, V = (torch.full((2, n_kv, T + 9, 128), 3.0, dtype=dtype, device=DEV) for _ in range(2))
    k4 = (torch.full((2, n_kv, T + 9, 64), 7, dtype=torch.uint8, device=DEV), torch.full((2, n_kv, T + 9, 4), 7, dtype=torch.uint8, device=DEV))
    out = ra.ra_append_tokens(q, k, v, dev(first), n_new=dev(n_new), q_weight=w[0], k_weight=w[1], inv_freq=torch.from_numpy(f).to(DEV),
                              interleaved=inter, K=K, V=V, k4=k4)
    for s in range(2):
        a, n = first[s], n_new[s]
        assert torch.equal(V[s, :, a:a + n], v[s, :n].transpose(0, 1))
        for c in (K, V):
            assert (c[s, :, :a] == 3.0).all() and (c[s, :, a + n:] == 3.0).all()
        assert (out[s, :, n:] == 0).all()
        whole = ra.ra_quantize_kv4(K[s:s + 1, :, a:a + n].contiguous())
        assert all(torch.equal(c[s, :, a:a + n], e[0]) for c, e in zip(k4, whole))
        assert all((c[s, :, :a] == 7).all() and (c[s, :, a + n:] == 7).all() for c in k4)
        some = np.unique(np.concatenate([[0, 1, n - 1], np.random.default_rng(T).integers(0, n, 13)]))
        for rows, got, weight in ((q, out[s][:, some], w[0]), (k, K[s][:, a + some], w[1])):
            ref, size = OK.head_rows(_np(rows[s, some]), a + some, _np(weight), 1e-6, f, inter)
            _row_close(_np(got).transpose(1, 0, 2), ref, size, dtype)


def test_rows_past_four_gigabytes():
    """The second head's rows start 5 GB into the caches and 4.6 GB into q_out."""
    cap, T = 20_000_000, 140_000
    g = torch.Generator(device=DEV).manual_seed(3)
    K, V = (torch.empty((1, 2, cap, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    k, v = (torch.randn((1, 40, 2, 128), generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    end = torch.tensor([cap - 40], dtype=torch.int32, device=DEV)
    ra.ra_append_tokens(None, k, v, end, K=K, V=V)
    assert torch.equal(K[0, :, cap - 40:], k[0].transpose(0, 1)) and torch.equal(V[0, :, cap - 40:], v[0].transpose(0, 1))
    del K, V
    q = torch.randint(-999, 999, (1, T, 130, 128), generator=g, device=DEV, dtype=torch.int16).to(torch.bfloat16)
    out = ra.ra_append_tokens(q, None, None, None)
    assert torch.equal(out[0], q[0].transpose(0, 1))
