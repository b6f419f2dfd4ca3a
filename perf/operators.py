"""The operators around a key/value cache held in 4 bits, as cases that can be timed: what puts tokens
into a cache, what turns rows into 4 bits and back, and the attention that reads them.

A case is a dict of plain values. Five kinds of call ("op"):

  append    norms of queries and keys per head, position rotation, new rows into the caches
  quantize  rows into 4 bits and back into the type they came from
  full      attention of one query per head over the whole 4-bit cache
  attend    the same over retrieved ids and the static tokens
  token     one layer of a decoded token: append into the 4-bit cache, attention over all of it

Caches are [n_seq][n_kv][capacity][128]. A row in 4 bits is 64 bytes of codes (sign and one of 0, 0.5,
1, 1.5, 2, 3, 4, 6; even dimensions in the low halves) and a scale byte for each block of 32 dimensions
(2^(byte - 127), the least power of two with which nothing exceeds 6). With `own` false, run computes
the operators in their plain form.
"""
import math

import torch

own = False

D, BLOCK = 128, 32
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HEADS = [(32, 8), (32, 8), (8, 2), (16, 2), (8, 8), (32, 4), (4, 1), (6, 2), (16, 1), (1, 1), (28, 4)]
MOST_VALUES = 1 << 28                # most cache values (K or V) of a drawn case: a 128K layer has 2^27
CODES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0)


def _case(name, op, **kw):
    c = {"op": op, "dtype": "bf16", "n_seq": 1, "n_q": 32, "n_kv": 8, "N": 131072, "T": 1, "ragged": False,
         "norm": False, "rot": 128, "interleaved": False, "q4": False, "sink": 4, "window": 640, "topk": 100, "grown": 0}
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # a decoded token's rows of one layer into the caches of one sequence: the smallest call, latency
        _case("append_token", "append", N=4096),
        # a 32K prompt: every head's queries as the index build reads them, keys and values into the cache
        _case("append_prompt_32k", "append", T=32768, N=33000, norm=True),
        # chunks of several sequences of unequal length, one of them with nothing, float32, half of the
        # dimensions rotated in neighbouring pairs, rows in 4 bits beside the cache
        _case("append_chunks_f32", "append", dtype="f32", n_seq=5, n_q=6, n_kv=2, T=1021, N=9001, ragged=True, norm=True,
              rot=64, interleaved=True, q4=True),
        # the keys of a 128K layer into 4 bits and back (an index is built again from what the cache stands for)
        _case("quantize_128k", "quantize"),
        # few short ragged float32 rows
        _case("quantize_ragged_f32", "quantize", dtype="f32", n_seq=3, n_kv=2, N=1003),
        # one float32 head over 4K tokens: latency
        _case("full_f32_1head_4k", "full", dtype="f32", n_q=1, n_kv=1, N=4096),
        # exact attention of a 128K layer
        _case("full_128k", "full"),
        # a million tokens, sixteen heads on one KV head
        _case("full_1m_group16", "full", n_q=16, n_kv=1, N=1 << 20),
        # a batch of 16 sequences of unequal length up to 32K, one of them empty
        _case("full_batch16_ragged", "full", n_seq=16, N=32768, ragged=True),
        # what follows a walk at 128K: 100 retrieved rows and 644 static ones
        _case("attend_128k", "attend"),
        # a batch of 16 in the middle of generation: appended tokens have joined the static rows
        _case("attend_batch16_grown", "attend", n_seq=16, N=32768, grown=301),
        # a decoded token of one layer that keeps its cache in 4 bits only
        _case("token_batch8_20k", "token", n_seq=8, N=20011, ragged=True, norm=True, q4=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: operator, type, heads, batch, lengths and options over the ranges that users have."""
    op = rng.choice(["append", "quantize", "full", "full", "attend", "token"])
    c = _case(None, op)
    c["dtype"] = rng.choice(["bf16", "bf16", "f32"])
    c["n_q"], c["n_kv"] = rng.choice(HEADS)
    c["n_seq"] = max(1, int(2 ** rng.uniform(-1.0, 4.9)))
    c["ragged"] = rng.random() < 0.5
    room = MOST_VALUES // (2 if c["dtype"] == "f32" else 1) // (c["n_seq"] * c["n_kv"] * D)
    c["N"] = _log_int(rng, 200, min(room, 1 << 20) if op in ("full", "token") else min(room, 1 << 17))
    c["norm"], c["interleaved"] = rng.random() < 0.5, rng.random() < 0.3
    c["rot"] = rng.choice([128, 128, 64, 32, 96, 16, 0])
    c["q4"] = op == "token" or rng.random() < 0.5
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


def _keys(n_seq, n_kv, rows, seed):
    """Keys of a head: a common offset and a spread of its own in every dimension."""
    at = _randn((n_seq, n_kv, 1, D), seed, 1)
    spread = (0.5 * _randn((n_seq, n_kv, 1, D), seed, 2)).exp()
    return _randn((n_seq, n_kv, rows, D), seed, 3).mul_(spread).add_(at * (4.0 / at.norm(dim=-1, keepdim=True)))


def _queries(n_seq, n_q, seed):
    """Queries lie away from the keys: an offset of three times a key's length in a direction of their own."""
    at = _randn((n_seq, n_q, D), seed, 4)
    return _randn((n_seq, n_q, D), seed, 5) * (0.5 * _randn((n_seq, n_q, D), seed, 6)).exp() + at * (45.0 / at.norm(dim=-1, keepdim=True))


def _pack(x):
    """float32 rows [..., 128] -> (codes uint8 [..., 64], scale bytes uint8 [..., 4])."""
    value, scale = _quantized(x)
    y = value.unflatten(-1, (D // BLOCK, BLOCK)).abs() / _unit(scale).unsqueeze(-1)
    code = torch.where(y <= 2.0, 2.0 * y, torch.where(y <= 4.0, y + 2.0, 0.5 * y + 4.0)).flatten(-2).to(torch.uint8)
    code = code | ((x < 0).to(torch.uint8) << 3)
    return code[..., 0::2] | (code[..., 1::2] << 4), scale


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


def prepare(case, seed):
    n_seq, n_q, n_kv, N, T = (case[k] for k in ("n_seq", "n_q", "n_kv", "N", "T"))
    op, dtype = case["op"], DTYPES[case["dtype"]]
    s = {"case": case}
    if op == "quantize":
        s["X"] = _keys(n_seq, n_kv, N, seed).to(dtype)
        s["buffers"] = (torch.zeros((n_seq, n_kv, N, D // 2), dtype=torch.uint8, device="cuda"),
                        torch.zeros((n_seq, n_kv, N, D // BLOCK), dtype=torch.uint8, device="cuda"), torch.empty_like(s["X"]))
        return s
    if op in ("full", "attend", "token") or case["q4"]:
        s["k4"] = _pack(_keys(n_seq, n_kv, N, seed))
        s["v4"] = _pack(_randn((n_seq, n_kv, N, D), seed, 8))
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
        if op == "append":
            s["K"], s["V"] = (torch.zeros((n_seq, n_kv, N, D), dtype=dtype, device="cuda") for _ in range(2))
    if op in ("full", "attend"):
        s["q"] = _queries(n_seq, n_q, seed).to(dtype)
        s["n_tokens"] = _lengths(case, N, seed)
    if op == "token":
        s["n_tokens"] = s["first"] + s["n_new"]
    if op in ("full", "token"):
        s["out"] = torch.empty((n_seq, n_q, D), device="cuda")
        s["lse"] = torch.empty((n_seq, n_q), device="cuda")
    if op == "attend":
        s["ids"] = _retrieved(case, s)
        s["index"] = _index(case)
    return s


def _static(case):
    """Which rows are static: the first `sink`, the last `window`, and those that came after the index was built."""
    row, N = torch.arange(case["N"], device="cuda"), case["N"]
    return (row < case["sink"]) | (row >= min(N - case["window"], N - case["grown"]))


def _retrieved(case, s):
    """The rows outside the static set that a head's query likes best, as a walk returns them; every third
    head's walk came back with fewer."""
    n_seq, n_q, n_kv, topk = (case[k] for k in ("n_seq", "n_q", "n_kv", "topk"))
    score = _grouped(s["q"].float(), n_kv) @ _values(*s["k4"]).transpose(-1, -2)
    score = score.flatten(1, 2).masked_fill_(_static(case), -math.inf)
    best, ids = score.topk(topk, dim=-1)
    ids = ids.int().masked_fill_(best == -math.inf, -1)
    ids[:, ::3, topk - topk // 8:] = -1
    return ids.contiguous()


def _index(case):
    """The handle of the walk's index (attention takes its sizes, and its workspace, from it). The graph is
    one that no walk of these cases reads."""
    import paper_2409_10516_amd as ra
    graphs, rows = case["n_seq"] * case["n_q"], case["N"] - case["grown"]
    return ra.ra_index_import(torch.full((graphs, rows, 1), -1, dtype=torch.int32), torch.zeros(graphs, dtype=torch.int32),
                              case["n_seq"], case["n_q"], case["n_kv"])


# ---- the plain forms ----------------------------------------------------------------------------------

def _unit(byte):
    """2^(byte - 127), from its bits; NaN for 255."""
    return torch.where(byte == 255, math.nan, (byte.int() << 23).view(torch.float32))


def _quantized(x):
    """float32 rows -> (the values that their 4-bit rows stand for, scale bytes)."""
    x = x.unflatten(-1, (D // BLOCK, BLOCK))
    top = x.abs().amax(dim=-1)
    m, e = torch.frexp(torch.where(top < 2.0 ** 127, top, 1.0))      # top = m 2^e, m in [0.5, 1), and 6 = 0.75 2^3
    k = (e - 2 - (m <= 0.75).int()).clamp_(min=-125)
    k = torch.where(top == 0, -125, k)
    unit = _unit(k + 127).unsqueeze(-1)
    y = x / unit
    step = 0.5 + 0.5 * (y.abs() >= 2.0) + (y.abs() >= 4.0)
    value = torch.round(y / step) * step * unit
    bad = ~(top < 2.0 ** 127)
    value = torch.where(bad.unsqueeze(-1), math.nan, value)
    return value.flatten(-2), torch.where(bad, 255, k + 127).to(torch.uint8)


def _values(codes, scale):
    """The float32 values that 4-bit rows stand for."""
    table = torch.tensor(CODES, device=codes.device)
    v = torch.stack((table[(codes & 15).int()], table[(codes >> 4).int()]), dim=-1).flatten(-2)
    return (v.unflatten(-1, (D // BLOCK, BLOCK)) * _unit(scale).unsqueeze(-1)).flatten(-2)


def _grouped(q, n_kv):
    return q.unflatten(1, (n_kv, q.shape[1] // n_kv))


def _softmax_out(z, V):
    """Logits [..., rows] (-inf where there is none) and values [..., rows, 128] -> (out, lse); nothing attended: 0, -inf."""
    top = z.amax(dim=-1, keepdim=True)
    p = torch.exp(z - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(dim=-1, keepdim=True)
    return (p @ V) / torch.where(total == 0, 1.0, total), (top + torch.log(total)).squeeze(-1)


def _plain_full(q, k4, v4, n_tokens):
    n_kv, N = k4[0].shape[1], k4[0].shape[2]
    z = _grouped(q.float(), n_kv) @ _values(*k4).transpose(-1, -2) / math.sqrt(D)
    there = torch.arange(N, device="cuda") < n_tokens.view(-1, 1, 1, 1)
    out, lse = _softmax_out(z.masked_fill_(~there, -math.inf), _values(*v4))
    return out.flatten(1, 2), lse.flatten(1, 2)


def _plain_attend(case, q, k4, v4, ids):
    n_seq, n_q, n_kv = case["n_seq"], case["n_q"], case["n_kv"]
    rows = torch.nonzero(_static(case)).squeeze(-1).int()
    all_rows = torch.cat((rows.expand(n_seq, n_q, -1), ids), dim=-1)           # each head's rows
    seq = torch.arange(n_seq, device="cuda").view(-1, 1, 1)
    kv = (torch.arange(n_q, device="cuda") // (n_q // n_kv)).view(1, -1, 1)
    at = all_rows.clamp(min=0).long()
    K, V = (_values(codes[seq, kv, at], scale[seq, kv, at]) for codes, scale in (k4, v4))
    z = (K @ q.float().unsqueeze(-1)).squeeze(-1) / math.sqrt(D)
    out, lse = _softmax_out(z.masked_fill_(all_rows < 0, -math.inf).unsqueeze(-2), V)
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
        c, si = torch.cos(angle).float(), torch.sin(angle).float()
        a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if case["interleaved"] else (x[..., :rot // 2], x[..., rot // 2:rot])
        turned = a * c - b * si, b * c + a * si
        turned = torch.stack(turned, dim=-1).flatten(-2) if case["interleaved"] else torch.cat(turned, dim=-1)
        x = torch.cat((turned, x[..., rot:]), dim=-1)
    return x.to(dtype)


def _split(case, qkv):
    n_q, n_kv = case["n_q"], case["n_kv"]
    return qkv.unflatten(-1, (n_q + 2 * n_kv, D)).split((n_q, n_kv, n_kv), dim=2)


def _plain_append(case, s):
    T, N = case["T"], case["N"]
    q, k, v = _split(case, s["qkv"])
    new = torch.arange(T, device="cuda") < s["n_new"].view(-1, 1)                  # [n_seq][T]
    rows = _plain_head_rows(case, q, s["weights"][0], s).transpose(1, 2)
    s["q_out"].copy_(torch.where(new[:, None, :, None], rows, s["q_out"]))
    seq, t = torch.nonzero(new, as_tuple=True)
    at = s["first"].long()[seq] + t
    k = _plain_head_rows(case, k, s["weights"][1], s)[seq, t]                      # [new tokens][n_kv][128]
    v = v[seq, t]
    if "K" in s:
        s["K"][seq, :, at] = k
        s["V"][seq, :, at] = v
    if "k4" in s:
        for cache, x in ((s["k4"], k), (s["v4"], v)):
            codes, scale = _pack(x.float())
            cache[0][seq, :, at] = codes
            cache[1][seq, :, at] = scale
    return s["q_out"]


def _new_rows(case, s):
    """What the 4-bit rows [first, first + T) stand for, in the cache's type."""
    dtype = DTYPES[case["dtype"]]
    seq = torch.arange(case["n_seq"], device="cuda").view(-1, 1)
    at = s["first"].long().view(-1, 1) + torch.arange(case["T"], device="cuda")
    return [_values(codes[seq, :, at], scale[seq, :, at]).transpose(1, 2).to(dtype) for codes, scale in (s["k4"], s["v4"])]


def _plain(s):
    case = s["case"]
    op = case["op"]
    if op == "quantize":
        return _quantized(s["X"].float())[0].to(s["X"].dtype)
    if op == "full":
        return _plain_full(s["q"], s["k4"], s["v4"], s["n_tokens"])
    if op == "attend":
        return _plain_attend(case, s["q"], s["k4"], s["v4"], s["ids"])
    q = _plain_append(case, s)
    got = {"q": q}
    if op == "append":
        got["K"], got["V"] = s["K"], s["V"]
    if case["q4"]:
        got["k4"], got["v4"] = _new_rows(case, s)
    if op == "token":
        got["out"], got["lse"] = _plain_full(q.squeeze(2), s["k4"], s["v4"], s["n_tokens"])
    return got


# ---- the framework's calls ----------------------------------------------------------------------------

def _own(s):
    import paper_2409_10516_amd as ra
    case = s["case"]
    op, T = case["op"], case["T"]
    if op == "quantize":
        codes, scale, back = s["buffers"]
        x4 = ra.ra_quantize_kv4(s["X"], out=(codes, scale))
        return ra.ra_dequantize_kv4(x4, s["X"].dtype, out=back)
    if op == "full":
        return ra.ra_full_attention_q4(s["q"], s["k4"], s["v4"], s["n_tokens"], out=s["out"], lse=s["lse"])
    if op == "attend":
        return ra.ra_attend_q4(s["q"], s["index"], s["k4"], s["v4"], case["sink"], case["window"], s["ids"])
    q, k, v = _split(case, s["qkv"])
    ra.ra_append_tokens(q, k, v, s["first"], n_new=s["n_new"], q_weight=s["weights"][0], k_weight=s["weights"][1], eps=1e-6,
                        inv_freq=s["inv_freq"], interleaved=case["interleaved"], q_out=s["q_out"], K=s.get("K"), V=s.get("V"),
                        k4=s.get("k4"), v4=s.get("v4"))
    got = {"q": s["q_out"]}
    if op == "append":
        got["K"], got["V"] = s["K"], s["V"]
    if case["q4"]:
        got["k4"], got["v4"] = (ra.ra_dequantize_kv4(x4, s["qkv"].dtype, first=s["first"], rows=T) for x4 in (s["k4"], s["v4"]))
    if op == "token":
        got["out"], got["lse"] = ra.ra_full_attention_q4(s["q_out"].squeeze(2), s["k4"], s["v4"], s["n_tokens"], out=s["out"],
                                                         lse=s["lse"])
    return got


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without --------------------------------------------------------------------

def _mean_share(case):
    """Share of the rows that are there: unequal lengths are spread evenly."""
    return 0.5 + 0.5 / case["n_seq"] if case["ragged"] else 1.0


def work(case):
    n_seq, n_q, n_kv, N, T = (case[k] for k in ("n_seq", "n_q", "n_kv", "N", "T"))
    row, row4 = D * (2 if case["dtype"] == "bf16" else 4), D // 2 + D // BLOCK
    op = case["op"]
    if op == "quantize":
        rows = n_seq * n_kv * N
        return {"bytes": 2 * rows * (row + row4), "flops": 4 * rows * D}
    todo = {"bytes": 0, "flops": 0}
    if op in ("append", "token"):
        tokens = n_seq * T * _mean_share(case)
        todo["bytes"] += tokens * (row * (n_q + 2 * n_kv) + row * n_q)
        todo["bytes"] += tokens * 2 * n_kv * ((row if op == "append" else 0) + (row + 2 * row4 if case["q4"] else 0))
        todo["flops"] += tokens * (n_q + n_kv) * D * (3 + (4 if case["norm"] else 0))
    if op in ("full", "token"):
        rows = n_seq * N * _mean_share(case)
        todo["bytes"] += rows * n_kv * 2 * row4 + n_seq * n_q * (row + 4 * D + 4)
        todo["flops"] += rows * n_q * 4 * D
    if op == "attend":
        static = min(N, case["sink"] + max(case["window"], case["grown"]))
        rows = static * n_kv + case["topk"] * n_q
        todo["bytes"] += n_seq * (rows * 2 * row4 + n_q * (4 * case["topk"] + row + 4 * D + 4))
        todo["flops"] += n_seq * n_q * (static + case["topk"]) * 4 * D
    return todo


# ---- the definition in 64 bits ------------------------------------------------------------------------

def _exact_rows(x4, seq, head, rows):
    """Float64 values of some rows of one head, from the definition of a code: (-1)^s 2^(e - 1) (1 + m / 2), or s m / 2 for e = 0."""
    b = x4[0][seq, head, rows].to(torch.int32)
    code = torch.stack((b % 16, b // 16), dim=-1).reshape(b.shape[0], D)
    e, m = (code // 2) % 4, (code % 2).double()
    size = torch.where(e == 0, 0.5 * m, 2.0 ** (e.double() - 1.0) * (1.0 + 0.5 * m))
    unit = 2.0 ** (x4[1][seq, head, rows].double() - 127.0)
    return torch.where(code >= 8, -size, size) * unit.repeat_interleave(BLOCK, dim=-1)


def _exact_attention(q, k4, v4, rows_of):
    n_seq, n_q = q.shape[:2]
    group = n_q // k4[0].shape[1]
    out = torch.zeros((n_seq, n_q, D), dtype=torch.float64, device="cuda")
    lse = torch.full((n_seq, n_q), -math.inf, dtype=torch.float64, device="cuda")
    for i in range(n_seq):
        for h in range(n_q):
            rows = rows_of(i, h)
            if rows.numel():
                K, V = (_exact_rows(x4, i, h // group, rows) for x4 in (k4, v4))
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
    spin = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), t.double() * s["inv_freq"].double())
    pairs = x[..., :rot].reshape(*x.shape[:-1], rot // 2, 2) if case["interleaved"] else x[..., :rot].reshape(*x.shape[:-1], 2, rot // 2).transpose(-1, -2)
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * spin)
    z = z if case["interleaved"] else z.transpose(-1, -2)
    return torch.cat((z.reshape(*x.shape[:-1], rot), x[..., rot:]), dim=-1)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "quantize":
        x = s["X"].double().reshape(-1, BLOCK)
        k = torch.ceil(torch.log2(x.abs().amax(-1, keepdim=True).clamp_min(2.0 ** -130) / 6.0)).clamp_min(-125.0)
        k = torch.where(6.0 * 2.0 ** (k - 1) >= x.abs().amax(-1, keepdim=True), k - 1, k).clamp_min(-125.0)
        grid = torch.tensor(CODES[:8], dtype=torch.float64, device="cuda")
        y = (x / 2.0 ** k).abs()
        up = torch.bucketize(y, grid).clamp_(1, 7)                               # grid[up - 1] < y <= grid[up]
        low, high = grid[up - 1], grid[up]
        nearer = torch.where(y - low == high - y, up % 2 == 0, high - y < y - low)
        return (torch.where(nearer, high, low) * x.sign() * 2.0 ** k).reshape(s["X"].shape)
    if op == "full":
        if case["n_seq"] * case["n_q"] * case["N"] > 1 << 26:
            return None
        n = s["n_tokens"].tolist()
        return _exact_attention(s["q"], s["k4"], s["v4"], lambda i, h: torch.arange(n[i], device="cuda"))
    if op == "attend":
        static, ids = torch.nonzero(_static(case)).squeeze(-1), s["ids"].long()
        return _exact_attention(s["q"], s["k4"], s["v4"], lambda i, h: torch.cat((static, ids[i, h][ids[i, h] >= 0])))
    q, k, v = _split(case, s["qkv"])
    q, k, v = _exact_turned(case, s, q, s["weights"][0]), _exact_turned(case, s, k, s["weights"][1]), v.double()
    got = {"q": torch.zeros(s["q_out"].shape, dtype=torch.float64, device="cuda")}
    if op == "append":
        got["K"], got["V"] = (torch.zeros(s["K"].shape, dtype=torch.float64, device="cuda") for _ in range(2))
    n_new, first = s["n_new"].tolist(), s["first"].tolist()
    for i, (n, at) in enumerate(zip(n_new, first)):
        got["q"][i, :, :n] = q[i, :n].transpose(0, 1)
        if op == "append":
            got["K"][i, :, at:at + n], got["V"][i, :, at:at + n] = k[i, :n].transpose(0, 1), v[i, :n].transpose(0, 1)
    if case["q4"]:
        got["k4"] = got["v4"] = None         # (a value in 4 bits goes by the rounded row: no number of 64 bits is its result)
    if op == "token":
        got["out"] = got["lse"] = None       # (they go by the cache's 4-bit rows, which the same pass has written)
    return got
