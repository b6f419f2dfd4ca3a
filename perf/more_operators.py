"""The operators around a key/value cache in pages, as cases that can be timed: what puts tokens into
its pages, what takes rows out of them side by side, and the attention that reads them.

A case is a dict of plain values. Five kinds of call ("op"):

  append    norms of queries and keys per head, position rotation, new rows into the pages
  gather    rows of one cache side by side, as an index is built over them
  full      attention of one query per head over all tokens of every sequence
  attend    the same over retrieved ids and the static tokens
  token     one layer of a decoded token: append, then attention over all of the cache

K and V are [n_pages][n_kv][page][128]; row r of sequence s is slot r % page of page table[s][r // page]
(int32 [n_seq][pages of the longest sequence]). An entry outside [0, n_pages) is no page: its rows are
neither written nor attended, and come as zeroes where rows are gathered. With `own` false, run computes
the operators in their plain form.
"""
import math

import torch

own = False

D = 128
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HEADS = [(32, 8), (32, 8), (8, 2), (16, 2), (8, 8), (32, 4), (4, 1), (6, 2), (16, 1), (1, 1), (28, 4)]
MOST_VALUES = 1 << 28                # most cache values (K or V) of a drawn case: a 128K layer has 2^27


def _case(name, op, **kw):
    c = {"op": op, "dtype": "bf16", "n_seq": 1, "n_q": 32, "n_kv": 8, "page": 16, "N": 131072, "T": 1, "ragged": False, "holes": False,
         "norm": False, "rot": 128, "interleaved": False, "rot_scale": 1.0, "sink": 4, "window": 640, "topk": 100, "grown": 0}
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # a decoded token's rows of one layer into the pages of one sequence: the smallest call, latency
        _case("append_token", "append", N=4096),
        # a 32K prompt: every head's queries as the index build reads them, keys and values into pages of 64 tokens
        _case("append_prompt_32k", "append", T=32768, N=33000, page=64, norm=True),
        # chunks of several sequences of unequal length, one of them with nothing, float32, half of the dimensions rotated
        # in neighbouring pairs, cosines and sines scaled as positions stretched over long contexts have them
        _case("append_chunks_f32", "append", dtype="f32", n_seq=5, n_q=6, n_kv=2, T=1021, N=9001, ragged=True, norm=True,
              rot=64, interleaved=True, rot_scale=1.1386),
        # the keys of a 128K layer side by side (an index is built over them, and they get their 8-bit copy)
        _case("gather_128k", "gather"),
        # few short ragged float32 sequences in small pages, whose ends are missing
        _case("gather_ragged_f32", "gather", dtype="f32", n_seq=3, n_kv=2, N=1003, page=8, ragged=True),
        # one float32 head over 4K tokens: latency
        _case("full_f32_1head_4k", "full", dtype="f32", n_q=1, n_kv=1, N=4096, page=32),
        # exact attention of a 128K layer
        _case("full_128k", "full"),
        # a million tokens, sixteen heads on one KV head, large pages
        _case("full_1m_group16", "full", n_q=16, n_kv=1, N=1 << 20, page=256),
        # a batch of 16 sequences of unequal length up to 32K, one of them empty
        _case("full_batch16_ragged", "full", n_seq=16, N=32768, ragged=True),
        # what follows a walk at 128K: 100 retrieved rows and 644 static ones
        _case("attend_128k", "attend", page=64),
        # a batch of 16 of unequal length in the middle of generation: appended tokens have joined the static rows
        _case("attend_batch16_grown", "attend", n_seq=16, N=32768, ragged=True, grown=301),
        # a decoded token of one layer: its rows into the pages, attention over all of them
        _case("token_batch8_20k", "token", n_seq=8, N=20011, ragged=True, norm=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: operator, type, heads, batch, pages, lengths and options over the ranges that users have."""
    op = rng.choice(["append", "gather", "full", "full", "attend", "attend", "token"])
    c = _case(None, op)
    c["dtype"] = rng.choice(["bf16", "bf16", "f32"])
    c["n_q"], c["n_kv"] = rng.choice(HEADS)
    c["n_seq"] = max(1, int(2 ** rng.uniform(-1.0, 4.9)))
    c["page"] = rng.choice([16, 16, 32, 64, 128, 256, 8, 1])
    c["ragged"], c["holes"] = rng.random() < 0.6, rng.random() < 0.2
    room = MOST_VALUES // (2 if c["dtype"] == "f32" else 1) // (c["n_seq"] * c["n_kv"] * D)
    c["N"] = _log_int(rng, 200, min(room, 1 << 20) if op in ("full", "token") else min(room, 1 << 17))
    c["norm"], c["interleaved"] = rng.random() < 0.5, rng.random() < 0.3
    c["rot"], c["rot_scale"] = rng.choice([128, 128, 64, 32, 96, 16, 0]), rng.choice([1.0, 1.0, 1.25, 0.9])
    if op == "append":
        rows = (1 << 20) // (c["n_seq"] * (c["n_q"] + 2 * c["n_kv"])) or 1
        c["T"] = rng.choice([1, min(rows, _log_int(rng, 2, c["N"])), min(c["N"], rows)])
    if op == "attend":
        c["sink"], c["window"] = rng.choice([0, 4, 128]), rng.choice([0, 64, 640, rng.randrange(1, 1500)])
        c["topk"] = min(max(1, c["N"] // 2), rng.choice([1, 16, 100, 100, rng.randrange(1, 600), 2000]))
        c["grown"] = rng.choice([0, 0, rng.randrange(1, max(2, c["N"] // 3))])
        c["n_seq"] = min(c["n_seq"], max(1, (1 << 24) // (c["n_q"] * c["N"])))
    return c


# ---- inputs -------------------------------------------------------------------------------------------

def _gen(seed, tag):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + tag)


def _randn(shape, seed, tag):
    return torch.randn(shape, generator=_gen(seed, tag), device="cuda", dtype=torch.float32)


def _key_pages(n_pages, n_kv, page, seed):
    """Keys of a head: a common offset and a spread of its own in every dimension."""
    at = _randn((n_kv, 1, D), seed, 1)
    spread = (0.5 * _randn((n_kv, 1, D), seed, 2)).exp()
    return _randn((n_pages, n_kv, page, D), seed, 3).mul_(spread).add_(at * (4.0 / at.norm(dim=-1, keepdim=True)))


def _queries(n_seq, n_q, seed):
    """Queries lie away from the keys, in a direction of their own."""
    at = _randn((n_seq, n_q, D), seed, 4)
    return _randn((n_seq, n_q, D), seed, 5) * (0.5 * _randn((n_seq, n_q, D), seed, 6)).exp() + at * (25.0 / at.norm(dim=-1, keepdim=True))


def _lengths(case, most, seed):
    """Tokens per sequence: all of them, or unequal ones with an empty sequence and one of a single token."""
    n = case["n_seq"]
    if not case["ragged"]:
        return torch.full((n,), most, dtype=torch.int32, device="cuda")
    L = torch.randint(1, most + 1, (n,), generator=_gen(seed, 7), device="cuda", dtype=torch.int32)
    L[0] = most
    if n > 2:
        L[1] = 0
    if n > 3:
        L[2] = 1
    return L


def _table(case, held, seed):
    """Pages of `held` tokens per sequence, in any order from a pool with room for all at their longest, the rest of which belongs to
    nobody -> (table, pages of the pool). With holes every ninth page or so has been given back."""
    page, per = case["page"], -(-case["N"] // case["page"])
    col = torch.arange(per, device="cuda")
    there = col * page < held.view(-1, 1)
    n_pages = case["n_seq"] * per + 3
    order = torch.randperm(n_pages, generator=_gen(seed, 13), device="cuda").int()
    table = torch.where(there, order[:n_pages - 3].view(-1, per), -1)
    if case["holes"]:
        gone = torch.rand(table.shape, generator=_gen(seed, 14), device="cuda") < 1.0 / 9.0
        gone &= col * page < held.view(-1, 1) - page               # (the last one is being written)
        table[gone] = -1
    return table, n_pages


def prepare(case, seed):
    n_seq, n_q, n_kv, N, T = (case[k] for k in ("n_seq", "n_q", "n_kv", "N", "T"))
    op, dtype, page = case["op"], DTYPES[case["dtype"]], case["page"]
    s = {"case": case}
    if op in ("append", "token"):
        s["qkv"] = _randn((n_seq, T, (n_q + 2 * n_kv) * D), seed, 9).to(dtype)    # what the projection has written
        s["weights"] = tuple((1.0 + 0.2 * _randn((D,), seed, 10 + i)).to(dtype) for i in range(2)) if case["norm"] else (None, None)
        i = torch.arange(0, case["rot"], 2, dtype=torch.float64, device="cuda")
        s["inv_freq"] = (500000.0 ** (-i / max(case["rot"], 1))).float() if case["rot"] else None
        s["n_new"] = _lengths(case, T, seed)
        # (a decoded token behind a context of its own, a prompt's or chunk's rows from somewhere)
        behind = torch.rand((n_seq,), generator=_gen(seed, 12), device="cuda", dtype=torch.float64)
        s["first"] = (behind * (N - T + 1)).int().clamp_(max=N - T)
        if not case["ragged"] and T == 1:
            s["first"].fill_(N - 1)
        s["q_out"] = torch.zeros((n_seq, n_q, T, D), dtype=dtype, device="cuda")
        s["n_tokens"] = s["first"] + s["n_new"]
    else:
        s["n_tokens"] = _lengths(case, N, seed)
    s["table"], n_pages = _table(case, s["n_tokens"], seed)
    shape = (n_pages, n_kv, page, D)
    if op == "append":
        s["K"], s["V"] = (torch.zeros(shape, dtype=dtype, device="cuda") for _ in range(2))
    else:
        s["K"] = _key_pages(*shape[:3], seed).to(dtype)
        s["V"] = _randn(shape, seed, 8).to(dtype) if op != "gather" else None
    if op == "gather":
        s["X"] = torch.empty((n_seq, n_kv, N, D), dtype=dtype, device="cuda")
    if op in ("full", "attend"):
        s["q"] = _queries(n_seq, n_q, seed).to(dtype)
    if op == "attend":
        s["n_indexed"] = (s["n_tokens"] - case["grown"]).clamp_(min=0)
        s["ids"] = _retrieved(case, s)
    if op != "append" and op != "gather":
        s["out"] = torch.empty((n_seq, n_q, D), device="cuda")
        s["lse"] = torch.empty((n_seq, n_q), device="cuda")
    if own:
        import paper_2409_10516_amd as ra
        s["cache"] = ra.PagedCache(s["K"], s["V"], s["table"])
    return s


def _static(case, s):
    """Which rows [n_seq][N] are static: the first `sink`, the last `window`, and those that came after the index was built."""
    row, n = torch.arange(case["N"], device="cuda"), s["n_tokens"].view(-1, 1)
    late = torch.minimum(n - case["window"], s["n_indexed"].view(-1, 1))
    return ((row < case["sink"]) | (row >= late)) & (row < n)


def _retrieved(case, s):
    """The indexed rows outside the static set that a head's query likes best, as a walk returns them; every third head's walk
    came back with fewer."""
    topk = case["topk"]
    K, there = _rows_of(case, s, s["K"])
    there = there & (torch.arange(case["N"], device="cuda") < s["n_indexed"].view(-1, 1)) & ~_static(case, s)
    score = (_grouped(s["q"].float(), case["n_kv"]) @ K.transpose(-1, -2)).flatten(1, 2)
    best, ids = score.masked_fill_(~there.unsqueeze(1), -math.inf).topk(topk, dim=-1)
    ids = ids.int().masked_fill_(best == -math.inf, -1)
    ids[:, ::3, topk - topk // 8:] = -1
    return ids.contiguous()


# ---- the plain forms ----------------------------------------------------------------------------------

def _rows_of(case, s, pages):
    """All rows of every sequence side by side, float32 [n_seq][n_kv][N][128], and which there are [n_seq][N]."""
    N, page = case["N"], case["page"]
    table = s["table"].long()
    there = ((table >= 0) & (table < pages.shape[0])).repeat_interleave(page, dim=1)[:, :N]
    x = pages[table.clamp(0, pages.shape[0] - 1)]                                # [n_seq][pages][n_kv][page][128]
    x = x.transpose(1, 2).flatten(2, 3)[:, :, :N]
    return x.float().masked_fill_(~there[:, None, :, None], 0.0), there


def _grouped(q, n_kv):
    return q.unflatten(1, (n_kv, q.shape[1] // n_kv))


def _softmax_out(z, V):
    """Logits [..., rows] (-inf where there is none) and values [..., rows, 128] -> (out, lse); nothing attended: 0, -inf."""
    top = z.amax(dim=-1, keepdim=True)
    p = torch.exp(z - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(dim=-1, keepdim=True)
    return (p @ V) / torch.where(total == 0, 1.0, total), (top + torch.log(total)).squeeze(-1)


def _plain_full(case, s, q):
    K, there = _rows_of(case, s, s["K"])
    there = there & (torch.arange(case["N"], device="cuda") < s["n_tokens"].view(-1, 1))
    z = _grouped(q.float(), case["n_kv"]) @ K.transpose(-1, -2) / math.sqrt(D)
    del K
    out, lse = _softmax_out(z.masked_fill_(~there[:, None, None], -math.inf), _rows_of(case, s, s["V"])[0])
    return out.flatten(1, 2), lse.flatten(1, 2)


def _plain_attend(case, s):
    n_seq, n_q, n_kv, N, page = (case[k] for k in ("n_seq", "n_q", "n_kv", "N", "page"))
    static = _static(case, s)
    order = torch.where(static, torch.arange(N, device="cuda"), N).sort(dim=-1).values
    most = min(N, case["sink"] + max(case["window"], case["grown"]))
    rows = order[:, :most].masked_fill(order[:, :most] == N, -1)
    ids = s["ids"].long()
    at = ids.clamp(0, N - 1)
    free = (ids >= 0) & (ids < s["n_tokens"].view(-1, 1, 1)) & ~static[torch.arange(n_seq, device="cuda").view(-1, 1, 1), at]
    rows = torch.cat((rows.unsqueeze(1).expand(-1, n_q, -1), ids.masked_fill(~free, -1)), dim=-1)      # each head's rows
    seq = torch.arange(n_seq, device="cuda").view(-1, 1, 1)
    kv = (torch.arange(n_q, device="cuda") // (n_q // n_kv)).view(1, -1, 1)
    at = rows.clamp(min=0)
    where = s["table"].long()[seq, at // page]
    there = (rows >= 0) & (where >= 0) & (where < s["K"].shape[0])
    where = where.clamp(0, s["K"].shape[0] - 1)
    K, V = (x[where, kv, at % page].float() for x in (s["K"], s["V"]))
    z = (K @ s["q"].float().unsqueeze(-1)).squeeze(-1) / math.sqrt(D)
    out, lse = _softmax_out(z.masked_fill_(~there, -math.inf).unsqueeze(-2), V)
    return out.squeeze(-2), lse.squeeze(-1)


def _plain_head_rows(case, x, weight, s):
    """Projected rows [n_seq][T][heads][128] -> normed and rotated ones, in the type of x."""
    dtype, rot = x.dtype, case["rot"]
    x = x.float()
    if weight is not None:
        r = 1.0 / torch.sqrt(x.double().square().mean(dim=-1, keepdim=True) + 1e-6)
        x = x * r.float() * weight.float()
    if rot:
        pos = s["first"].double().view(-1, 1) + torch.arange(case["T"], device="cuda", dtype=torch.float64)
        angle = (pos.unsqueeze(-1) * s["inv_freq"].double()).unsqueeze(2)
        c, si = ((case["rot_scale"] * f(angle)).float() for f in (torch.cos, torch.sin))
        a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if case["interleaved"] else (x[..., :rot // 2], x[..., rot // 2:rot])
        turned = a * c - b * si, b * c + a * si
        turned = torch.stack(turned, dim=-1).flatten(-2) if case["interleaved"] else torch.cat(turned, dim=-1)
        x = torch.cat((turned, x[..., rot:]), dim=-1)
    return x.to(dtype)


def _split(case, qkv):
    n_q, n_kv = case["n_q"], case["n_kv"]
    return qkv.unflatten(-1, (n_q + 2 * n_kv, D)).split((n_q, n_kv, n_kv), dim=2)


def _plain_append(case, s):
    T, page = case["T"], case["page"]
    q, k, v = _split(case, s["qkv"])
    new = torch.arange(T, device="cuda") < s["n_new"].view(-1, 1)                  # [n_seq][T]
    rows = _plain_head_rows(case, q, s["weights"][0], s).transpose(1, 2)
    s["q_out"].copy_(torch.where(new[:, None, :, None], rows, s["q_out"]))
    seq, t = torch.nonzero(new, as_tuple=True)
    at = s["first"].long()[seq] + t
    where = s["table"].long()[seq, at // page]
    keep = (where >= 0) & (where < s["K"].shape[0])
    seq, t, at, where = seq[keep], t[keep], at[keep], where[keep]
    s["K"][where, :, at % page] = _plain_head_rows(case, k, s["weights"][1], s)[seq, t]
    s["V"][where, :, at % page] = v[seq, t]
    return {"q": s["q_out"], "K": s["K"], "V": s["V"]}


def _plain(s):
    case = s["case"]
    op = case["op"]
    if op == "gather":
        return s["X"].copy_(_rows_of(case, s, s["K"])[0])
    if op == "full":
        return _plain_full(case, s, s["q"])
    if op == "attend":
        return _plain_attend(case, s)
    got = _plain_append(case, s)
    if op == "token":
        got["out"], got["lse"] = _plain_full(case, s, s["q_out"].squeeze(2))
    return got


# ---- the framework's calls ----------------------------------------------------------------------------

def _own(s):
    import paper_2409_10516_amd as ra
    case = s["case"]
    op, cache = case["op"], s["cache"]
    if op == "gather":
        return ra.ra_gather_paged(cache, rows=case["N"], out=s["X"])
    if op == "full":
        return ra.ra_full_attention_paged(s["q"], cache, s["n_tokens"], N=case["N"], out=s["out"], lse=s["lse"])
    if op == "attend":
        return ra.ra_attend_paged(s["q"], cache, case["sink"], case["window"], s["ids"], s["n_tokens"], n_indexed=s["n_indexed"], N=case["N"],
                                  out=s["out"], lse=s["lse"])
    q, k, v = _split(case, s["qkv"])
    ra.ra_append_tokens_paged(q, k, v, s["first"], cache, n_new=s["n_new"], q_weight=s["weights"][0], k_weight=s["weights"][1], eps=1e-6,
                              inv_freq=s["inv_freq"], interleaved=case["interleaved"], rot_scale=case["rot_scale"], q_out=s["q_out"])
    got = {"q": s["q_out"], "K": s["K"], "V": s["V"]}
    if op == "token":
        got["out"], got["lse"] = ra.ra_full_attention_paged(s["q_out"].squeeze(2), cache, s["n_tokens"], N=case["N"], out=s["out"], lse=s["lse"])
    return got


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without --------------------------------------------------------------------

def _mean_share(case):
    """Share of the rows that are there: unequal lengths are spread evenly."""
    return 0.5 + 0.5 / case["n_seq"] if case["ragged"] else 1.0


def work(case):
    n_seq, n_q, n_kv, N, T = (case[k] for k in ("n_seq", "n_q", "n_kv", "N", "T"))
    row, op = D * (2 if case["dtype"] == "bf16" else 4), case["op"]
    rows = n_seq * N * _mean_share(case)
    if op == "gather":
        return {"bytes": rows * n_kv * row + n_seq * n_kv * N * row + 4 * rows / case["page"], "flops": 0}
    todo = {"bytes": 0, "flops": 0}
    if op in ("append", "token"):
        tokens = n_seq * T * _mean_share(case)
        todo["bytes"] += tokens * 2 * row * (n_q + 2 * n_kv)
        todo["flops"] += tokens * (n_q + n_kv) * D * (3 + (4 if case["norm"] else 0))
    if op in ("full", "token"):
        if op == "token" and case["ragged"]:
            rows = n_seq * N * 0.5                                                 # (behind contexts of any length)
        todo["bytes"] += rows * n_kv * 2 * row + 4 * rows / case["page"] + n_seq * n_q * (row + 4 * D + 4)
        todo["flops"] += rows * n_q * 4 * D
    if op == "attend":
        static = min(N, case["sink"] + max(case["window"], case["grown"]))
        todo["bytes"] += n_seq * ((static * n_kv + case["topk"] * n_q) * 2 * row + n_q * (4 * case["topk"] + row + 4 * D + 4))
        todo["flops"] += n_seq * n_q * (static + case["topk"]) * 4 * D
    return todo


# ---- the definition in 64 bits ------------------------------------------------------------------------

def _exact_slots(s, seq, rows):
    """Pages and slots of some rows of a sequence, those that have a page."""
    page = s["case"]["page"]
    where = s["table"][seq].long()[torch.div(rows, page, rounding_mode="floor")]
    ok = (where > -1) & (where < s["K"].size(0))
    return where[ok], torch.remainder(rows, page)[ok]


def _exact_attention(s, q, rows_of):
    n_seq, n_q = q.shape[:2]
    group = n_q // s["case"]["n_kv"]
    out = torch.zeros((n_seq, n_q, D), dtype=torch.float64, device="cuda")
    lse = torch.full((n_seq, n_q), -math.inf, dtype=torch.float64, device="cuda")
    for i in range(n_seq):
        for h in range(n_q):
            where, slot = _exact_slots(s, i, rows_of(i, h))
            if where.numel():
                K, V = (x[where, h // group, slot].double() for x in (s["K"], s["V"]))
                z = K.mv(q[i, h].double()) / D ** 0.5
                lse[i, h] = torch.logsumexp(z, dim=0)
                out[i, h] = torch.softmax(z, dim=0) @ V
    return out, lse


def _exact_turned(case, s, x, weight):
    """Norm and rotation of [n_seq][T][heads][128] in 64 bits, as products of complex numbers."""
    x, rot = x.double(), case["rot"]
    if weight is not None:
        x = x * weight.double() / (x.pow(2).sum(-1, keepdim=True) / D + 1e-6).sqrt()
    if not rot:
        return x
    t = torch.arange(case["T"], device="cuda").view(1, -1, 1, 1) + s["first"].view(-1, 1, 1, 1)
    size = torch.full((), case["rot_scale"], dtype=torch.float64, device="cuda")
    spin = torch.polar(size, t.double() * s["inv_freq"].double())
    pairs = x[..., :rot].reshape(*x.shape[:-1], rot // 2, 2) if case["interleaved"] else x[..., :rot].reshape(*x.shape[:-1], 2, rot // 2).transpose(-1, -2)
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * spin)
    z = z if case["interleaved"] else z.transpose(-1, -2)
    return torch.cat((z.reshape(*x.shape[:-1], rot), x[..., rot:]), dim=-1)


def exact(case, seed):
    s = prepare(case, seed)
    op, n_kv = case["op"], case["n_kv"]
    if op == "gather":
        X = torch.zeros(s["X"].shape, dtype=torch.float64, device="cuda")
        for i in range(case["n_seq"]):
            rows = torch.arange(case["N"], device="cuda")
            where, slot = _exact_slots(s, i, rows)
            at = s["table"][i].long()[rows // case["page"]]
            X[i, :, rows[(at > -1) & (at < s["K"].size(0))]] = s["K"][where, :, slot].double().transpose(0, 1)
        return X
    if op == "full":
        if case["n_seq"] * case["n_q"] * case["N"] > 1 << 26:
            return None
        n = s["n_tokens"].tolist()
        return _exact_attention(s, s["q"], lambda i, h: torch.arange(n[i], device="cuda"))
    if op == "attend":
        n, indexed, ids = s["n_tokens"].tolist(), s["n_indexed"].tolist(), s["ids"].long()

        def rows_of(i, h):
            late = max(0, min(n[i] - case["window"], indexed[i]))
            sink = min(case["sink"], n[i])
            near = torch.cat((torch.arange(sink, device="cuda"), torch.arange(max(late, sink), n[i], device="cuda")))
            far = ids[i, h]
            return torch.cat((near, far[(far >= sink) & (far < late)]))
        return _exact_attention(s, s["q"], rows_of)
    q, k, v = _split(case, s["qkv"])
    q, k, v = _exact_turned(case, s, q, s["weights"][0]), _exact_turned(case, s, k, s["weights"][1]), v.double()
    got = {"q": torch.zeros(s["q_out"].shape, dtype=torch.float64, device="cuda"), "K": s["K"].double(), "V": s["V"].double()}
    n_new, first = s["n_new"].tolist(), s["first"].tolist()
    for i, (n, at) in enumerate(zip(n_new, first)):
        got["q"][i, :, :n] = q[i, :n].transpose(0, 1)
        rows = torch.arange(at, at + n, device="cuda")
        page = s["table"][i].long()[rows // case["page"]]
        ok = (page > -1) & (page < s["K"].size(0))
        got["K"][page[ok], :, rows[ok] % case["page"]] = k[i, :n][ok]
        got["V"][page[ok], :, rows[ok] % case["page"]] = v[i, :n][ok]
    if op == "token":
        got["out"] = got["lse"] = None       # (they go by the rows that the same pass has rounded)
    return got
