"""A cache in pages (ra_append_tokens_paged, ra_gather_paged, ra_full_attention_paged, ra_attend_paged) against the oracle in
float64, within bounds that follow from the roundings. What is not a row of a sequence is NaN in every pool."""
import numpy as np
import pytest
import torch

import paper_2409_10516_amd as ra
from oracle import attention as OA, kv4 as OK, paged as OP
from tests.util import to_np

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = [torch.bfloat16, torch.float32]
NOT_A_PAGE = [-1, -2 ** 31, 2 ** 31 - 1]


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def check(out, lse, q, K, V):
    """out and lse of a head over rows K, V (float64). A logit is a float32 sum of 128 products and is scaled (at most
    132 roundings of 2^-24 of the magnitudes summed), subtracted from the maximum and exponentiated (4 of 2^-24 times either's size,
    and 4 for the exponential): e_i of a weight's relative error. Weights meet values with 24 bits of mantissa; sums of N terms in any
    order lose at most N 2^-24 of the magnitudes, and the factors of the running maximum, the terms of a weight and the division
    64 more. A weight (the largest is 1, and so their sum is no less), or a part of one, below the least normal number
    2^-126 may become zero: three parts, of 2^-126 of its value each."""
    if len(K) == 0:
        assert (out == 0).all() and np.isneginf(lse)
        return
    o, l = OA.full_attention(q, K, V)
    z = K @ q / np.sqrt(128)
    w = np.exp(z - l)
    size = np.abs(K) @ np.abs(q) / np.sqrt(128)
    e = U * (132 * size + 4 * (np.abs(z) + np.abs(z).max()) + 4)
    mean, more = w @ e, (len(K) + 64) * U
    bound = 1.01 * ((w * (e + mean + more)) @ np.abs(V)) + 3 * 2.0 ** -126 * np.abs(V).sum(axis=0)
    far = np.abs(out - o) / np.maximum(bound, 1e-300)
    assert far.max() <= 1.0, f"{far.max():.3g} times the bound at {far.argmax()}"
    assert abs(lse - l) <= 1.01 * (mean + more + 4 * U * abs(l)), (lse, l)


class Cache:
    """Sequences of lens[s] tokens in pages of random places, `holes` of which are gone, with room for `rows` rows; V of unlike sizes."""

    def __init__(self, lens, n_kv, page, dtype, seed, rows=None, holes=0.0, spare=3):
        rng = np.random.default_rng(seed)
        n_seq, per = len(lens), -(-(rows or max(max(lens), 1)) // page)
        self.n_pages, self.page, self.n_kv, self.lens = n_seq * per + spare, page, n_kv, lens
        order = rng.permutation(self.n_pages)[:n_seq * per].reshape(n_seq, per).astype(np.int64)
        bad = rng.choice(NOT_A_PAGE + [self.n_pages, self.n_pages + 7], order.shape)
        mine = np.arange(per) * page < np.asarray(lens)[:, None]
        self.table = np.where(mine & (rng.random(order.shape) >= holes), order, bad).astype(np.int32)
        g = torch.Generator().manual_seed(seed)
        self.pools = []
        for which in range(2):
            x = torch.randn((self.n_pages, n_kv, page, 128), generator=g) * torch.exp(0.5 * torch.randn((1, n_kv, 1, 128), generator=g))
            if which == 0:
                x += torch.randn((1, n_kv, 1, 128), generator=g) / 3
            x = x.to(dtype)
            there = torch.zeros((self.n_pages, page), dtype=torch.bool)
            for s, n in enumerate(lens):
                for i, p in enumerate(self.table[s]):
                    if 0 <= p < self.n_pages:
                        there[p, :max(0, n - i * page)] = True
            self.pools.append(x.masked_fill_(~there[:, None, :, None], float("nan")))
        self.K, self.V = (p.to(DEV) for p in self.pools)
        self.np = [to_np(p).astype(np.float64) for p in self.pools]
        self.gpu = ra.PagedCache(self.K, self.V, ints(self.table))

    def rows(self, s, kv, rows):
        """float64 K and V of those of the rows that have a page."""
        (K, there), (V, _) = (OP.rows_of(x, self.table[s], kv, rows) for x in self.np)
        return K[there], V[there]


def queries(n_seq, n_q, dtype, seed):
    return (2.0 * torch.randn((n_seq, n_q, 128), generator=torch.Generator().manual_seed(seed))).to(dtype)


# ---- all tokens ---------------------------------------------------------------------------------
HEADS = [(1, 1), (2, 1), (3, 1), (8, 2), (5, 1), (16, 1), (17, 1), (4, 4), (40, 2)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n_q,n_kv", HEADS)
@pytest.mark.parametrize("n,page", [(1, 16), (37, 8), (700, 32)])
def test_full_attention_of_any_group(dtype, n_q, n_kv, n, page):
    c = Cache([n, n], n_kv, page, dtype, seed=n + n_q)
    q = queries(2, n_q, dtype, n)
    out, lse = (t.cpu().numpy() for t in ra.ra_full_attention_paged(q.to(DEV), c.gpu, N=n))
    for s in range(2):
        for h in range(n_q):
            check(out[s, h], lse[s, h], to_np(q[s, h]), *c.rows(s, h // (n_q // n_kv), range(n)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("page", [1, 2, 4, 8, 16, 32, 64, 256, 4096])
@pytest.mark.parametrize("n", [2, 15, 17, 31, 32, 33, 63, 65, 127, 129, 257, 1000, 2049])
def test_full_attention_of_any_length_and_page(dtype, n, page):
    """Lengths around the edges of chunks and pages, each sequence its own."""
    lens = [n, n - 1, 0, 1, n // 2]
    c = Cache(lens, 1, page, dtype, seed=n, rows=n + 3)
    q = queries(5, 4, dtype, n)
    out, lse = (t.cpu().numpy() for t in ra.ra_full_attention_paged(q.to(DEV), c.gpu, ints(lens)))
    for s in range(5):
        for h in (0, 3):
            check(out[s, h], lse[s, h], to_np(q[s, h]), *c.rows(s, 0, range(lens[s])))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("page,n,holes", [(1, 700, 0.5), (8, 900, 0.3), (16, 3000, 0.3), (16, 400, 1.0), (64, 5000, 0.5), (256, 9000, 0.4), (512, 9000, 0.9)])
def test_rows_without_a_page_are_not_attended(dtype, page, n, holes):
    lens = [n, n - 37, n // 3]
    c = Cache(lens, 2, page, dtype, seed=page + n, holes=holes)
    q = queries(3, 6, dtype, n)
    out, lse = (t.cpu().numpy() for t in ra.ra_full_attention_paged(q.to(DEV), c.gpu, ints(lens)))
    for s in range(3):
        for h in range(6):
            check(out[s, h], lse[s, h], to_np(q[s, h]), *c.rows(s, h // 3, range(lens[s])))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n_seq,n_q,n_kv,N,page", [(130, 4, 1, 700, 16), (67, 1, 1, 300, 8), (700, 2, 2, 257, 64), (2, 40, 1, 3000, 16), (1, 2, 1, 20001, 32),
                                                  (1, 17, 1, 40000, 16), (3, 3, 1, 9999, 128), (300, 8, 4, 1500, 16), (20, 2, 1, 9000, 4)])
def test_full_attention_of_many_sequences_heads_and_records(dtype, n_seq, n_q, n_kv, N, page):
    """More sequences than lanes, more jobs than workgroups, tiles of heads, many records of a head; sequences share their pages,
    lengths of zero, one and anything, some of them in a row."""
    rng = np.random.default_rng(N)
    lens = rng.integers(0, N + 1, n_seq)
    lens[rng.random(n_seq) < 0.3] = 0
    lens[-1] = N
    if n_seq > 4:
        lens[1], lens[2], lens[n_seq // 2:n_seq // 2 + 3] = 1, 129, 0
    c = Cache([N], n_kv, page, dtype, seed=N)
    table = ints(c.table).expand(n_seq, -1).contiguous()
    q = queries(n_seq, n_q, dtype, N)
    out, lse = (t.cpu().numpy() for t in ra.ra_full_attention_paged(q.to(DEV), ra.PagedCache(c.K, c.V, table), ints(lens), N=N))
    assert (out[lens == 0] == 0).all() and np.isneginf(lse[lens == 0]).all() and np.isfinite(lse[lens > 0]).all()
    some = {0, 1, 2, n_seq - 1} | set(rng.integers(0, n_seq, 6).tolist())
    for s in sorted(x for x in some if x < n_seq):
        for h in sorted({0, n_q // 2, n_q - 1}):
            check(out[s, h], lse[s, h], to_np(q[s, h]), *c.rows(0, h // (n_q // n_kv), range(lens[s])))


@pytest.mark.parametrize("dtype", TYPES)
def test_lengths_past_the_cache_and_below_zero(dtype):
    c = Cache([100, 100, 100], 1, 16, dtype, seed=3)
    q = queries(3, 2, dtype, 3)
    for N in (100, 77):
        out, lse = (t.cpu().numpy() for t in ra.ra_full_attention_paged(q.to(DEV), c.gpu, ints([5000, -3, 40]), N=N))
        for s, n in enumerate((N, 0, 40)):
            check(out[s, 1], lse[s, 1], to_np(q[s, 1]), *c.rows(s, 0, range(n)))


@pytest.mark.parametrize("dtype", TYPES)
def test_values_that_are_no_numbers(dtype):
    """A NaN row that is attended makes its head NaN and no other; logits of -inf have no weight; where there is nothing else the result
    is that of no rows."""
    c = Cache([600, 600, 600], 2, 16, dtype, seed=9)
    at = lambda s, r: (int(c.table[s][r // 16]), r % 16)  # noqa: E731
    q = queries(3, 4, dtype, 9)
    p, slot = at(0, 333)
    c.K[p, 1, slot, 5] = float("nan")
    q[1, 0] = q[1, 0].abs() + 0.5
    for r in range(600):
        if r % 7:
            p, slot = at(1, r)
            c.K[p, 0, slot] = -float("inf")
    for r in range(600):
        p, slot = at(2, r)
        c.K[p, 0, slot] = -float("inf")
    q[2, 0] = q[2, 0].abs() + 0.5
    out, lse = (t.cpu().numpy() for t in ra.ra_full_attention_paged(q.to(DEV), c.gpu, N=600))
    assert np.isnan(out[0, 2:]).all() and np.isnan(lse[0, 2:]).all()
    check(out[0, 1], lse[0, 1], to_np(q[0, 1]), *c.rows(0, 0, range(600)))
    check(out[1, 0], lse[1, 0], to_np(q[1, 0]), *c.rows(1, 0, range(0, 600, 7)))
    assert (out[2, 0] == 0).all() and np.isneginf(lse[2, 0])
    check(out[2, 2], lse[2, 2], to_np(q[2, 2]), *c.rows(2, 1, range(600)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [1e-3, 30.0, 3e4])
def test_flat_and_sharp_softmax(dtype, scale):
    c = Cache([3001], 1, 16, dtype, seed=12)
    q = (scale * queries(1, 5, torch.float32, 12)).to(dtype)
    out, lse = (t.cpu().numpy() for t in ra.ra_full_attention_paged(q.to(DEV), c.gpu, N=3001))
    for h in range(5):
        check(out[0, h], lse[0, h], to_np(q[0, h]), *c.rows(0, 0, range(3001)))


@pytest.mark.parametrize("dtype", TYPES)
def test_logits_near_the_lowest_number(dtype):
    """All logits about -3e37, chunks without rows in front of them: equal weights."""
    c = Cache([300], 1, 16, dtype, seed=10)
    c.K.zero_()
    c.K[..., 3] = -1.5e19
    table = ints(c.table)
    table[0, :9] = -1
    q = torch.zeros((1, 2, 128))
    q[..., 3] = 2.0e19
    cache = ra.PagedCache(c.K, c.V, table)
    ids = torch.arange(300, dtype=torch.int32, device=DEV).expand(1, 2, -1).contiguous()
    V = c.rows(0, 0, range(144, 300))[1]
    for out, lse in (ra.ra_full_attention_paged(q.to(dtype).to(DEV), cache, N=300), ra.ra_attend_paged(q.to(dtype).to(DEV), cache, 2, 20, ids, N=300)):
        # (weights of 1, 156 of them: their sums and the division lose at most 160 roundings)
        assert (np.abs(out[0].cpu().numpy() - V.mean(0)) <= 160 * U * np.abs(V).mean(0)).all()
        assert np.allclose(lse.cpu().numpy(), -3.0e38 / np.sqrt(128), rtol=2.0 ** -7)


# ---- the retrieved and the static set ------------------------------------------------------------
ATTEND = [  # n_q, n_kv, page, lens, indexed (None: not given), sink, window, topk, holes
    (4, 2, 16, [300], None, 4, 32, 10, 0), (6, 2, 8, [700, 1, 0, 33], [650, 1, 0, 20], 4, 10, 129, 0), (3, 3, 64, [90, 50], None, 100, 100, 7, 0),
    (5, 1, 16, [1500], None, 0, 0, 200, 0), (16, 2, 32, [260, 264, 5, 31], [200, 264, 0, 31], 1, 31, 64, 0), (20, 1, 16, [4000], None, 128, 1400, 300, 0),
    (16, 1, 16, [9001], [1001], 4, 640, 100, 0), (8, 2, 4, [3001, 2000], [900, 2000], 4, 500, 40, 0.3), (17, 1, 1, [700, 600], [500, 600], 5, 20, 33, 0.3),
    (32, 8, 64, [2000, 1500], None, 4, 640, 100, 0.2), (16, 2, 16, [900] * 9, [800] * 9, 3, 20, 50, 0), (2, 1, 16, [2000] * 40, [1500] * 40, 3, 20, 300, 0),
    (1, 1, 16, [1], None, 0, 0, 1, 0), (1, 1, 16, [3000], None, 0, 1, 2048, 0), (2, 1, 16, list(range(130)), [n // 2 for n in range(130)], 1, 9, 20, 0),
    (40, 1, 8, [500] * 70, None, 4, 64, 33, 0.1), (16, 8, 64, [700, 3] * 20, [600, 1] * 20, 4, 64, 100, 0),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", range(len(ATTEND)))
def test_sparse_and_static_attention(case, dtype):
    n_q, n_kv, page, lens, indexed, sink, window, topk, holes = ATTEND[case]
    n_seq, N = len(lens), max(lens)
    c = Cache(lens, n_kv, page, dtype, seed=case, rows=N + 5, holes=holes)
    q, rng = queries(n_seq, n_q, dtype, case), np.random.default_rng(case)
    # entries anywhere, members of the static set, of other rows than there are, and given twice among them
    ids = rng.integers(-3, N + 9, (n_seq, n_q, topk)).astype(np.int32)
    ids[rng.random(ids.shape) < 0.1] = -1
    ids[:, 1::3, topk // 2:] = ids[:, 1::3, :topk - topk // 2]
    ids[:, 2::5] = -1
    ids[0, 0, 0] = 2 ** 31 - 1
    args = (q.to(DEV), c.gpu, sink, window, torch.from_numpy(ids).to(DEV), ints(lens))
    kw = dict(n_indexed=None if indexed is None else ints(indexed))
    got = [t.cpu().numpy() for t in ra.ra_attend_paged(*args, partials=True, **kw)]
    for s in range(n_seq):
        if s > 4 and s < n_seq - 1:
            continue
        for h in range(n_q):
            g = h // (n_q // n_kv)
            W, om = OP.sets(lens[s], lens[s] if indexed is None else indexed[s], sink, window, ids[s, h].tolist())
            for (o, l), rows in zip((got[0:2], got[2:4], got[4:6]), (np.concatenate([W, om]), om, W)):
                check(o[s, h], l[s, h], to_np(q[s, h]), *c.rows(s, g, rows.tolist()))
    again = ra.ra_attend_paged(*args, **kw)
    assert np.array_equal(again[0].cpu().numpy(), got[0]) and np.array_equal(again[1].cpu().numpy(), got[1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n_seq", [1, 130])
def test_rows_that_are_no_numbers_are_their_heads_alone(dtype, n_seq):
    """A retrieved row with a NaN key or an infinite or NaN value makes NaN of the heads that retrieved it and of their retrieved set, whether
    the job is one workgroup's or several; the others are what they were."""
    c = Cache([900] * n_seq, 2, 16, dtype, seed=17)
    q = queries(n_seq, 8, dtype, 17).to(DEV)
    n, g = ints([900] * n_seq), torch.Generator(device=DEV).manual_seed(4)
    ids = torch.randint(10, 400, (n_seq, 8, 40), dtype=torch.int32, device=DEV, generator=g)
    ids[:, 2, 7], ids[:, 5, 39] = 500, 600
    ref = ra.ra_attend_paged(q, c.gpu, 4, 100, ids, n, partials=True)
    for s in range(n_seq):
        p, slot = int(c.table[s][500 // 16]), 500 % 16
        c.V[p, 0, slot, 3] = float("nan")
        p, slot = int(c.table[s][600 // 16]), 600 % 16
        c.K[p, 1, slot, 100] = float("nan")
        c.V[p, 1, slot] = float("inf")
    got = ra.ra_attend_paged(q, c.gpu, 4, 100, ids, n, partials=True)
    others = [h for h in range(8) if h not in (2, 5)]
    for i, (a, b) in enumerate(zip(got, ref)):
        assert torch.equal(a[:, others], b[:, others])
        if i >= 4:                                          # (the static set's)
            assert torch.equal(a, b)
    assert torch.isnan(got[0][:, 2, 3]).all() and torch.isfinite(got[0][:, 2, 4:]).all() and torch.isnan(got[2][:, 2, 3]).all()
    assert torch.isnan(got[0][:, 5]).all() and torch.isnan(got[1][:, 5]).all() and torch.isnan(got[3][:, 5]).all()


def test_attention_without_lengths_and_over_fewer_rows():
    c = Cache([512], 1, 16, torch.bfloat16, seed=4)
    q = queries(1, 4, torch.bfloat16, 4)
    ids = torch.randint(0, 512, (1, 4, 30), dtype=torch.int32, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
    for N, given in ((None, 512), (300, 300)):
        out, lse = (t.cpu().numpy() for t in ra.ra_attend_paged(q.to(DEV), c.gpu, 4, 50, ids, N=N))
        for h in range(4):
            W, om = OP.sets(given, given, 4, 50, ids[0, h].tolist())
            check(out[0, h], lse[0, h], to_np(q[0, h]), *c.rows(0, 0, np.concatenate([W, om]).tolist()))


def test_all_rows_by_either_call():
    """A window of everything, and ids of everything, are full attention."""
    for dtype in TYPES:
        c = Cache([1000, 800], 2, 16, dtype, seed=6)
        q, n = queries(2, 4, dtype, 6).to(DEV), ints([1000, 800])
        none, every = torch.full((2, 4, 3), -1, dtype=torch.int32, device=DEV), torch.arange(1000, dtype=torch.int32, device=DEV).expand(2, 4, -1).contiguous()
        full = [t.cpu().numpy() for t in ra.ra_full_attention_paged(q, c.gpu, n)]
        for got in (ra.ra_attend_paged(q, c.gpu, 0, 5000, none, n), ra.ra_attend_paged(q, c.gpu, 0, 0, every, n),
                    ra.ra_attend_paged(q, c.gpu, 7, 0, every, n, n_indexed=ints([0, 300]))):
            o, m = (t.cpu().numpy() for t in got)
            for s in range(2):
                for h in range(4):
                    rows = c.rows(s, h // 2, range([1000, 800][s]))
                    check(o[s, h], m[s, h], to_np(q[s, h].cpu()), *rows)
                    check(full[0][s, h], full[1][s, h], to_np(q[s, h].cpu()), *rows)


# ---- appending -------------------------------------------------------------------------------------
def _inv_freq(rot):
    return (10000.0 ** (-np.arange(0, rot, 2) / max(rot, 1))).astype(np.float32)


def _row_close(got, ref, size, dtype):
    """A row's values after float32 arithmetic (the reciprocal root, two products, a rotation of rounded factors: at most 16 roundings of
    2^-24 of the magnitudes that a value is made of) and one rounding to the type."""
    tol = 16 * U * size + (np.abs(ref) * torch.finfo(dtype).eps / 2 if dtype != torch.float32 else 0.0) + 1e-38
    assert (np.abs(got - ref) <= 1.01 * tol).all(), (np.abs(got - ref) / tol).max()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n_q,n_kv,T,page,rot,inter,norm,scale", [
    (4, 2, 21, 8, 128, False, True, 1.0), (3, 1, 1, 16, 64, True, False, 1.1386), (6, 6, 40, 1, 96, False, True, 0.7), (32, 8, 130, 64, 128, False, True, 1.25),
    (1, 1, 300, 32, 16, True, False, -2.0), (5, 5, 70, 4, 0, False, True, 3.0), (28, 4, 300, 16, 128, True, True, 1.0)])
def test_append(dtype, n_q, n_kv, T, page, rot, inter, norm, scale):
    """Rows of sequences that begin anywhere, end before T, run out of the table or of pages, in front of the cache too."""
    n_seq, cap = 6, T + 41
    g = torch.Generator().manual_seed(T)
    x = torch.randn((n_seq, T, n_q + 2 * n_kv, 128), generator=g).to(dtype).to(DEV)
    q, k, v = x.split((n_q, n_kv, n_kv), dim=2)
    w = [(1 + 0.3 * torch.randn(128, generator=g)).to(dtype).to(DEV) if norm else None for _ in range(2)]
    f = torch.from_numpy(_inv_freq(rot)).to(DEV) if rot else None
    rng = np.random.default_rng(T)
    per = -(-cap // page)
    n_pages = n_seq * per + 2
    table = rng.permutation(n_pages)[:n_seq * per].reshape(n_seq, per).astype(np.int64)
    table[3, ::2] = rng.choice(NOT_A_PAGE + [n_pages], table[3, ::2].shape)
    first, n_new = [0, 29, per * page - 5, -3, 10, 7], [T, T + 50, T, T, 0, max(T - 2, 0)]
    K, V = (torch.full((n_pages, n_kv, page, 128), 3.0, dtype=dtype, device=DEV) for _ in range(2))
    cache = ra.PagedCache(K, V, ints(table))
    out = ra.ra_append_tokens_paged(q, k, v, ints(first), cache, n_new=ints(n_new), q_weight=w[0], k_weight=w[1], eps=1e-5, inv_freq=f, interleaved=inter,
                                    rot_scale=scale)
    opt = dict(weight=None, eps=1e-5, inv_freq=None if f is None else _inv_freq(rot), interleaved=inter)
    want_V, done = to_np(torch.full(V.shape, 3.0)), np.zeros((n_pages, page), bool)
    gotK, gotV, gotQ = (to_np(t.cpu()).astype(np.float64) for t in (K, V, out))
    for s in range(n_seq):
        n = min(T, n_new[s])
        assert (gotQ[s, :, n:] == 0).all()
        if n <= 0:
            continue
        pos = first[s] + np.arange(n)
        for rows, weight, is_q in ((q, w[0], True), (k, w[1], False)):
            ref, size = OK.head_rows(to_np(rows[s, :n].cpu()), pos, **(opt | dict(weight=None if weight is None else to_np(weight.cpu()))))
            if rot:
                ref[..., :rot] *= scale
                size[..., :rot] *= abs(scale)
            if is_q:
                _row_close(gotQ[s, :, :n].transpose(1, 0, 2), ref, size, dtype)
            else:
                kref, ksize = ref, size
        for t, (p, slot) in enumerate(OP.places(table[s], n_pages, page, pos.tolist())):
            if p >= 0:
                assert not done[p, slot]
                done[p, slot] = True
                _row_close(gotK[p, :, slot], kref[t], ksize[t], dtype)
                want_V[p, :, slot] = to_np(v[s, t].cpu())
    assert done.any() and np.array_equal(gotV, want_V)
    assert (gotK.transpose(0, 2, 1, 3)[~done] == 3.0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n_q,n_kv,T,page", [(32, 8, 1, 16), (6, 2, 8209, 16), (16, 2, 8200, 64), (28, 4, 2100, 256), (32, 8, 2049, 8), (64, 8, 300, 1)])
def test_append_writes_the_rows_of_a_cache_without_pages(dtype, n_q, n_kv, T, page):
    """Bit for bit, over the sizes that change the workgroups; rows side by side again are that cache."""
    g = torch.Generator(device=DEV).manual_seed(T)
    x = torch.randn((2, T, n_q + 2 * n_kv, 128), generator=g, device=DEV).to(dtype)
    q, k, v = x.split((n_q, n_kv, n_kv), dim=2)
    w = [(1 + 0.3 * torch.randn(128, generator=g, device=DEV)).to(dtype) for _ in range(2)]
    first, n_new, rows = ints([5, 0]), ints([T, T - 37]), T + 9
    opt = dict(n_new=n_new, q_weight=w[0], k_weight=w[1], inv_freq=torch.from_numpy(_inv_freq(128)).to(DEV))
    K, V = (torch.zeros((2, n_kv, rows, 128), dtype=dtype, device=DEV) for _ in range(2))
    ref = ra.ra_append_tokens(q, k, v, first, K=K, V=V, **opt)
    per = -(-rows // page)
    table = torch.randperm(2 * per, generator=g, device=DEV).int().view(2, per)
    pools = [torch.zeros((2 * per, n_kv, page, 128), dtype=dtype, device=DEV) for _ in range(2)]
    cache = ra.PagedCache(*pools, table)
    got = ra.ra_append_tokens_paged(q, k, v, first, cache, **opt)
    assert torch.equal(got, ref)
    for i, x in enumerate((K, V)):
        assert torch.equal(ra.ra_gather_paged(cache, values=bool(i), rows=rows), x)


def test_append_of_one_of_q_k_and_v():
    x = torch.randn((1, 5, 2, 128), device=DEV)
    K, V = (torch.zeros((3, 2, 4, 128), device=DEV) for _ in range(2))
    table = ints([[2, 0]])
    assert ra.ra_append_tokens_paged(None, x, None, None, ra.PagedCache(K, None, table)) is None
    assert torch.equal(K[2], x[0, :4].transpose(0, 1)) and torch.equal(K[0, :, 0], x[0, 4]) and (K[1] == 0).all()
    ra.ra_append_tokens_paged(None, None, x, None, ra.PagedCache(None, V, table))
    assert torch.equal(V, K)
    out = ra.ra_append_tokens_paged(x, None, None, None, ra.PagedCache(K, V, table))
    assert torch.equal(out[0], x[0].transpose(0, 1)) and torch.equal(V, K)
    with pytest.raises(ra.RaError):
        ra.ra_append_tokens_paged(None, x, x, None, ra.PagedCache(K, None, table))
    with pytest.raises(ra.RaError):
        ra.ra_gather_paged(ra.PagedCache(K, None, table), values=True)
    with pytest.raises(ra.RaError):
        ra.ra_full_attention_paged(x[:, 0], ra.PagedCache(K, None, table))


# ---- rows side by side -----------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens,n_kv,page,T,first", [([100, 0, 37], 3, 8, 45, [60, 0, -4]), ([1], 1, 1, 1, None), ([5000, 5000], 4, 16, 5000, None),
                                                   ([333, 333], 2, 64, 333, [0, 300]), ([700], 2, 2, 40, [-2000000000]), ([700], 2, 2, 40, [2147483640])])
def test_gather(dtype, lens, n_kv, page, T, first):
    c = Cache(lens, n_kv, page, dtype, seed=T, holes=0.2)
    for values in (False, True):
        got = to_np(ra.ra_gather_paged(c.gpu, values=values, first=None if first is None else ints(first), rows=T).cpu()).astype(np.float64)
        for s in range(len(lens)):
            rows = list(range((first or [0] * len(lens))[s], (first or [0] * len(lens))[s] + T))
            for kv in range(n_kv):
                x, there = OP.rows_of(c.np[int(values)], c.table[s], kv, rows)
                assert np.array_equal(got[s, kv], x, equal_nan=True)          # (slots of a page behind a sequence's end are NaN, and come as such)


# ---- tables, pools, streams ----------------------------------------------------------------------------
def test_calls_on_a_given_stream_are_the_same_calls():
    """A stream given by hand goes through the checks in Python, none through compiled ones: every call, with results given and not."""
    c = Cache([300, 77], 2, 16, torch.bfloat16, seed=14)
    q, n, ids = queries(2, 4, torch.bfloat16, 14).to(DEV), ints([300, 77]), torch.randint(0, 300, (2, 4, 9), dtype=torch.int32, device=DEV)
    x = torch.randn((2, 3, 8, 128), device=DEV).bfloat16()
    w, f = torch.rand(128, device=DEV).bfloat16(), torch.from_numpy(_inv_freq(64)).to(DEV)
    here = torch.cuda.current_stream()
    res = lambda: dict(out=torch.empty((2, 4, 128), device=DEV), lse=torch.empty((2, 4), device=DEV),  # noqa: E731
                       workspace=torch.empty(1 << 22, dtype=torch.uint8, device=DEV))
    for N in (None, 200):
        for n_tokens in (None, n):
            a, b = ({**(res() if i else {})} for i in range(2))
            one, two = ra.ra_full_attention_paged(q, c.gpu, n_tokens, N, **a), ra.ra_full_attention_paged(q, c.gpu, n_tokens, N, stream=here, **b)
            assert all(torch.equal(torch.nan_to_num(x), torch.nan_to_num(y)) for x, y in zip(one, two))
            for indexed in (None, ints([250, 70])):
                one, two = (ra.ra_attend_paged(q, c.gpu, 3, 40, ids, n_tokens, indexed, N, stream=s, **kw) for s, kw in ((None, res()), (here, {})))
                assert all(torch.equal(torch.nan_to_num(x), torch.nan_to_num(y)) for x, y in zip(one, two))
    for first, rows, values in ((None, None, False), (ints([3, -2]), 40, True), (ints([290, 0]), 33, False)):
        one, two = (ra.ra_gather_paged(c.gpu, values=values, first=first, rows=rows, stream=s) for s in (None, here))
        three = ra.ra_gather_paged(c.gpu, values, first, rows, out=torch.empty_like(one))
        assert torch.equal(torch.nan_to_num(one), torch.nan_to_num(two)) and torch.equal(torch.nan_to_num(one), torch.nan_to_num(three))
    for parts in ((0, 1, 2), (0,), (1,), (2, 1)):
        for n_new in (None, ints([2, 3])):
            got = []
            for s in (None, here):
                t = [v if i in parts else None for i, v in enumerate(x.split((4, 2, 2), dim=2))]
                cache = ra.PagedCache(torch.zeros_like(c.K), torch.zeros_like(c.V), ints(c.table))
                out = ra.ra_append_tokens_paged(*t, ints([5, 60]), cache, n_new=n_new, q_weight=w, k_weight=w, eps=1e-5, inv_freq=f, interleaved=True,
                                                rot_scale=1.5, stream=s)
                got.append((out, cache.K, cache.V))
            for one, two in zip(*got):
                assert (one is None and two is None) or torch.equal(one, two)
            assert (got[0][0] is None) == (0 not in parts) and (got[0][1] != 0).any() == (1 in parts) and (got[0][2] != 0).any() == (2 in parts)


def test_tables_that_are_parts_of_larger_ones():
    c = Cache([300, 250, 100], 2, 16, torch.bfloat16, seed=8)
    big = torch.full((7, 50), 9, dtype=torch.int32, device=DEV)
    big[1:6:2, 3:3 + c.table.shape[1]] = ints(c.table)
    part = ra.PagedCache(c.K, c.V, big[1:6:2, 3:3 + c.table.shape[1]])
    one = ra.PagedCache(c.K, c.V, big[3:4, 3:3 + c.table.shape[1]])
    q, n, ids = queries(3, 4, torch.bfloat16, 8).to(DEV), ints([300, 250, 100]), torch.randint(0, 250, (3, 4, 9), dtype=torch.int32, device=DEV)
    for call in (lambda x, s: ra.ra_full_attention_paged(q[s], x, n[s]), lambda x, s: ra.ra_attend_paged(q[s], x, 4, 40, ids[s].contiguous(), n[s]),
                 lambda x, s: (ra.ra_gather_paged(x),)):
        whole = call(c.gpu, slice(0, 3))
        for a, b in zip(call(part, slice(0, 3)), whole):
            assert torch.equal(torch.nan_to_num(a), torch.nan_to_num(b))
        for a, b in zip(call(one, slice(1, 2)), whole):
            a, b = torch.nan_to_num(a.float()), torch.nan_to_num(b[1:2].float())
            assert torch.allclose(a, b, rtol=1e-5, atol=1e-6)
    x = torch.randn((3, 2, 8, 128), device=DEV).bfloat16()
    qx, k, v = x.split((4, 2, 2), dim=2)
    first = ints([10, 200, 90])
    ra.ra_append_tokens_paged(qx, k, v, first, part)
    assert all(torch.equal(c.V[int(c.table[s][(f + t) // 16]), :, (f + t) % 16], v[s, t]) for s, f in enumerate((10, 200, 90)) for t in range(2))


def test_rows_past_four_gigabytes():
    """Pages whose rows start up to 5 GB into the pool, and a table entry's number times the bytes of a page past 32 bits."""
    n_pages, n_kv, page = 40000, 2, 256
    K, V = (torch.empty((n_pages, n_kv, page, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    g = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randn((1, 600, n_kv, 128), generator=g, device=DEV).bfloat16()
    table = ints([[39999, 20000, 35001]])
    cache = ra.PagedCache(K, V, table)
    ra.ra_append_tokens_paged(None, x, x, None, cache)
    assert torch.equal(K[39999], x[0, :256].transpose(0, 1)) and torch.equal(V[35001, :, :88], x[0, 512:].transpose(0, 1))
    assert torch.equal(ra.ra_gather_paged(cache, rows=600), x.transpose(1, 2)) and torch.equal(ra.ra_gather_paged(cache, values=True, rows=600), x.transpose(1, 2))
    q = queries(1, 4, torch.bfloat16, 3)
    rows = to_np(x[0].cpu()).astype(np.float64)
    ids = torch.randint(0, 600, (1, 4, 20), dtype=torch.int32, device=DEV, generator=g)
    full, sparse = ra.ra_full_attention_paged(q.to(DEV), cache, N=600), ra.ra_attend_paged(q.to(DEV), cache, 4, 40, ids, N=600)
    for h in range(4):
        check(full[0][0, h].cpu().numpy(), float(full[1][0, h]), to_np(q[0, h]), rows[:, h // 2], rows[:, h // 2])
        both = np.concatenate(OP.sets(600, 600, 4, 40, ids[0, h].tolist()))
        check(sparse[0][0, h].cpu().numpy(), float(sparse[1][0, h]), to_np(q[0, h]), rows[both, h // 2], rows[both, h // 2])


def test_calls_on_their_own_streams():
    """Two streams at once, each with workspace and results of its own, and a call on a stream that allocates there."""
    c = Cache([5000, 4000], 2, 16, torch.bfloat16, seed=21)
    n, ids = ints([5000, 4000]), torch.randint(0, 4000, (2, 8, 40), dtype=torch.int32, device=DEV)
    qs = [queries(2, 8, torch.bfloat16, 30 + i).to(DEV) for i in range(2)]
    calls = [lambda q, **kw: ra.ra_full_attention_paged(q, c.gpu, n, **kw), lambda q, **kw: ra.ra_attend_paged(q, c.gpu, 4, 700, ids, n, **kw)]
    refs = [[call(q) for q in qs] for call in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    room = [torch.empty(1 << 24, dtype=torch.uint8, device=DEV) for _ in range(2)]
    outs = [[[(torch.empty((2, 8, 128), device=DEV), torch.empty((2, 8), device=DEV)) for _ in range(2)] for _ in calls] for _ in range(10)]
    torch.cuda.synchronize()
    for turn in range(10):
        for j, call in enumerate(calls):
            for i, st in enumerate(streams):
                call(qs[i], stream=st, workspace=room[i], out=outs[turn][j][i][0], lse=outs[turn][j][i][1])
    torch.cuda.synchronize()
    for turn in outs:
        for j in range(2):
            for i in range(2):
                assert torch.equal(turn[j][i][0], refs[j][i][0]) and torch.equal(turn[j][i][1], refs[j][i][1])
    side = torch.cuda.Stream()
    for j, call in enumerate(calls):
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
        got = call(qs[0], stream=side)
        for _ in range(200):
            torch.full((1 << 18,), float("nan"), device=DEV)
        torch.cuda.synchronize()
        assert torch.equal(got[0], refs[j][0][0]) and torch.equal(got[1], refs[j][0][1])


# ---- the calls together ----------------------------------------------------------------------------------
def test_prompts_index_walk_and_decode_over_pages():
    """The set as a serving loop uses it: prompts are normed, rotated and put into pages, an index is built over each sequence's keys, side
    by side for that moment, they get their 8-bit copy for the walk, and from then on the pages are the only cache: decoded tokens take
    new pages as they need them and attend by walk + sparse attention, and by full attention."""
    n_q, n_kv, N, page, sink, window, topk, ef, deg, knn = 4, 2, 600, 16, 4, 50, 16, 48, 12, 12
    g = torch.Generator().manual_seed(11)
    tokens = lambda n: torch.randn((2, n, n_q + 2 * n_kv, 128), generator=g).bfloat16().to(DEV).split((n_q, n_kv, n_kv), dim=2)  # noqa: E731
    w = (1 + 0.2 * torch.randn(128, generator=g)).bfloat16().to(DEV)
    opt = dict(q_weight=w, k_weight=w, inv_freq=torch.from_numpy(_inv_freq(128)).to(DEV))
    per = 45
    free = np.random.default_rng(1).permutation(2 * per).tolist()
    K, V = (torch.full((2 * per, n_kv, page, 128), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    table = np.full((2, per), -1, np.int32)
    for s in range(2):
        for i in range(-(-N // page)):
            table[s, i] = free.pop()
    on_gpu = ints(table)
    cache = ra.PagedCache(K, V, on_gpu)
    Qp = ra.ra_append_tokens_paged(*tokens(N), None, cache, **opt)
    keys = ra.ra_gather_paged(cache, rows=N)
    idx = ra.ra_build_index(keys, Qp, deg, knn)
    k8 = ra.ra_quantize_keys(keys)
    dense = ra.ra_gather_paged(cache, values=True, rows=N)
    pos, indexed = ints([N, N]), ints([N, N])
    for step in range(20):
        if (N + step) % page == 0:
            for s in range(2):
                table[s, (N + step) // page] = free.pop()
            on_gpu.copy_(ints(table))
        qd = ra.ra_append_tokens_paged(*tokens(1), pos, cache, **opt).squeeze(2)
        pos += 1
        n = N + step + 1
        ids, _ = ra.ra_search(qd, idx, None, sink, window, topk, ef, 4, k8=k8)
        out, lse = ra.ra_attend_paged(qd, cache, sink, window, ids, pos, n_indexed=indexed)
        full, full_lse = ra.ra_full_attention_paged(qd, cache, pos)
        if step == 0:          # (before the window slides: the grown decode step's own sparse attention, over a cache without pages)
            Kc, Vc = (ra.ra_gather_paged(cache, values=v, rows=N + 1) for v in (False, True))
            o, m, i8, _ = ra.ra_decode_step(qd, idx, Kc, Vc, sink, window, topk, ef, 4, n_tokens=N + 1)
            a = ra.ra_attend_paged(qd, cache, sink, window, i8, pos, n_indexed=indexed)
            assert torch.allclose(a[0], o, rtol=2e-3, atol=2e-3 * float(o.abs().max())) and torch.allclose(a[1], m, rtol=1e-4)
            assert torch.equal(Kc[:, :, :N], keys) and torch.equal(Vc[:, :, :N], dense)
        if step in (0, 7, 8, 9, 19):
            Kn, Vn = (to_np(x.cpu()).astype(np.float64) for x in (K, V))
            for s in range(2):
                for h in range(n_q):
                    kv = h // (n_q // n_kv)
                    qq, got = to_np(qd[s, h].cpu()), ids[s, h].cpu().numpy()
                    W, om = OP.sets(n, N, sink, window, got.tolist())
                    assert (got >= 0).sum() >= topk // 2 and len(om) >= (got >= 0).sum() - window
                    both = np.concatenate([W, om]).tolist()
                    (Kb, there), (Vb, _) = (OP.rows_of(x, table[s], kv, both) for x in (Kn, Vn))
                    assert there.all()
                    check(out[s, h].cpu().numpy(), float(lse[s, h]), qq, Kb, Vb)
                    (Ka, there), (Va, _) = (OP.rows_of(x, table[s], kv, range(n)) for x in (Kn, Vn))
                    assert there.all()
                    check(full[s, h].cpu().numpy(), float(full_lse[s, h]), qq, Ka, Va)
    idx.free()


def test_captured_tokens_replay_as_positions_and_tables_advance():
    """Append and both attentions in a captured graph, twice, each graph with buffers of its own; positions, lengths and the table's entries
    change between the replays, which take turns with eager work; every replay against the eager calls on a copy of the cache."""
    n_seq, n_q, n_kv, page, per = 2, 8, 2, 16, 25
    f = torch.from_numpy(_inv_freq(128)).to(DEV)
    g = torch.Generator(device=DEV).manual_seed(13)
    pools = [torch.randn((n_seq * per, n_kv, page, 128), generator=g, device=DEV).bfloat16() for _ in range(2)]
    table = torch.full((n_seq, per), -1, dtype=torch.int32, device=DEV)
    perm = torch.randperm(n_seq * per, generator=g, device=DEV).int().view(n_seq, per)
    table[0, :9], table[1, :25] = perm[0, :9], perm[1]
    start = ints([140, 391])

    class Token:
        def __init__(self, seed):
            self.pools = [p.clone() for p in pools]
            self.table, self.pos = table.clone(), start.clone()
            self.cache = ra.PagedCache(*self.pools, self.table)
            self.x = torch.zeros((n_seq, 1, n_q + 2 * n_kv, 128), dtype=torch.bfloat16, device=DEV)
            self.ids = torch.randint(10, 130, (n_seq, n_q, 20), dtype=torch.int32, device=DEV, generator=torch.Generator(device=DEV).manual_seed(seed))
            self.indexed = ints([100, 300])
            self.q = torch.zeros((n_seq, n_q, 1, 128), dtype=torch.bfloat16, device=DEV)
            self.out = [torch.empty((n_seq, n_q, 128), device=DEV) for _ in range(2)]
            self.lse = [torch.empty((n_seq, n_q), device=DEV) for _ in range(2)]
            self.room = [torch.empty(1 << 23, dtype=torch.uint8, device=DEV) for _ in range(2)]

        def step(self):
            q, k, v = self.x.split((n_q, n_kv, n_kv), dim=2)
            ra.ra_append_tokens_paged(q, k, v, self.pos, self.cache, inv_freq=f, q_out=self.q)
            self.pos.add_(1)
            ra.ra_full_attention_paged(self.q.squeeze(2), self.cache, self.pos, workspace=self.room[0], out=self.out[0], lse=self.lse[0])
            ra.ra_attend_paged(self.q.squeeze(2), self.cache, 4, 32, self.ids, self.pos, n_indexed=self.indexed, workspace=self.room[1], out=self.out[1],
                               lse=self.lse[1])

        def state(self):
            return [t.clone() for t in (*self.pools, self.q, *self.out, *self.lse, self.pos)]

    both, graphs = [Token(1), Token(2)], []
    eager = [Token(1), Token(2)]
    for t in both:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            t.step()
    for turn in range(12):                              # (the second sequence runs into the end of its table)
        if turn == 3:
            for t in both + eager:
                t.table[0, 9] = perm[0, 9]              # (and the first one's new page comes late: a token of it is lost)
        for i, (t, e) in enumerate(zip(both, eager)):
            new = torch.randn(t.x.shape, generator=torch.Generator().manual_seed(2 * turn + i)).bfloat16().to(DEV)
            for y in (t, e):
                y.x.copy_(new)
            graphs[i].replay()
        torch.cuda.synchronize()
        for t, e in zip(both, eager):
            e.step()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(t.state(), e.state())), turn
