"""Position rotation on the way into a cache, and attention over latent vectors, as timed cases.

    append         rows of keys rotated to their positions and quantised with their
                   values into the slots of a `KVCache`, the query rows rotated in the
                   same call; the values that the cache now stands for read back
    latent_append  the same for a `LatentCache`: one latent vector and one rotated key a
                   token, shared by all heads, rounded into their slots
    absorbed       attention over a latent cache whose query heads have been taken
                   into the latent space: keys [latent | rotated], values the latent
    expanded       attention over a latent cache through per-head keys and values,
                   w_k and w_v applied to the latent vectors

Rotation.  Of a row's first r values pair i, (x[i], x[i + r/2]) or interleaved
(x[2i], x[2i + 1]), becomes (a c - b s, b c + a s), c and s the entries [position, i] of
the given tables; products and sums in 32 bits, each rounded.

Quantised format.  A row x is one token's key or value of one head, D values.
4 bits: a = max|x|, T = clamp(floor(log2(a / 7)), -100, 125); per 16 values
r = max|x| / (7 2^T) is rounded to e = (1 + m/16) 2^(E-15), E and m in 0..15
(ties to even, saturating); c = clamp(round(x / (e 2^T)), -7, 7), ties to even; the value
is c e 2^T.  8 bits: s = max(bf16(a / 127), 2^-100), c = clamp(round(x / s), -127, 127),
the value is c s.

Attention of row i of a sequence's nq query rows, whose context is the first kv_len
tokens of its listed blocks: pos_i = kv_len - nq + i; with c_j the latent and r_j the
rotated part of token j,
    absorbed  z = scale (q[:R].c_j + q[R:].r_j),               out = sum_j p_j c_j
    expanded  z = scale (q[:N].(w_k c_j) + q[N:].r_j),         out = sum_j p_j (w_v c_j)
p the softmax over the keys that the row sees: those of listed blocks (not -1) with
(not causal, or j <= pos_i, or j < prefix) and (no tags, or the tag of its slot is the
row's).  A row that sees nothing gives 0, its log-sum-exp -inf.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}


# ------------------------------------------------------------------ the cases
def _append(name, n, q_heads, heads, dim, bits, dtype, rotary, pairs=False, block=64, far=8192,
            holes=False):
    return dict(name=name, kind="append", n=n, q_heads=q_heads, heads=heads, dim=dim, bits=bits,
                dtype=dtype, rotary=rotary, pairs=pairs, block=block, far=far, holes=holes)


def _latent_append(name, n, q_heads, latent, rope, dtype, stored, pairs=True, block=64, far=8192,
                   holes=False):
    return dict(name=name, kind="latent_append", n=n, q_heads=q_heads, latent=latent, rope=rope,
                rotary=rope, dtype=dtype, stored=stored, pairs=pairs, block=block, far=far,
                holes=holes)


def _attend(name, kind, seqs, kv, q, heads, latent, rope, dtype, block=64, ragged=0.0, causal=True,
            prefix=0.0, docs=0, retrieved=False, nope=0, value=0):
    return dict(name=name, kind=kind, seqs=seqs, kv=kv, q=q, heads=heads, latent=latent, rope=rope,
                dtype=dtype, block=block, ragged=ragged, causal=causal, prefix=prefix, docs=docs,
                retrieved=retrieved, nope=nope, value=value)


def listed():
    return [
        # one request's decoding step: a single token's query, key and value
        _append("append_1", 1, 32, 8, 128, 4, "bf16", 128, block=16),
        # a request's prompt on its way into the cache
        _append("append_8192", 8192, 32, 8, 128, 4, "bf16", 128),
        # a ragged batch whose padding is skipped, half of each head rotated, adjacent
        # pairs, master values in 32 bits, far positions
        _append("append_1531_int8", 1531, 5, 5, 64, 8, "fp32", 32, pairs=True, block=16,
                far=200_000, holes=True),
        # a decoding step of 48 requests
        _latent_append("latent_append_48", 48, 64, 512, 64, "bf16", "bf16", block=16),
        # the memory of a request: 16 chunks of 1024 tokens
        _latent_append("latent_append_16384", 16384, 16, 512, 64, "bf16", "bf16"),
        # one interactive user's decoding step over a short context
        _attend("latent_decode_1x700", "absorbed", 1, 700, 1, 16, 256, 32, "bf16", block=16),
        # a serving step: 64 requests of very different lengths
        _attend("latent_decode_64_ragged", "absorbed", 64, 8192, 1, 32, 512, 64, "bf16", ragged=0.9),
        # one request over a very long context
        _attend("latent_decode_1x200k", "absorbed", 1, 200_000, 1, 64, 512, 64, "bf16", block=128),
        # drafted tokens checked, many heads
        _attend("latent_draft_16x5", "absorbed", 16, 5000, 5, 40, 512, 64, "fp16", block=32, ragged=0.5),
        # a batch of 256 queries, each over the 32 chunks that its retrieval returned: the
        # namespaces keep tenants apart
        _attend("latent_retrieved_256x32", "absorbed", 256, 2048, 1, 12, 128, 32, "bf16", causal=False,
                docs=16, retrieved=True),
        # requests behind the memory prepended to them, which all their rows see
        _attend("latent_prompt_behind_memory", "expanded", 2, 10_240, 2048, 32, 512, 64, "bf16",
                ragged=0.3, prefix=0.8, nope=128, value=128),
        # several documents packed into one prompt, processed at once
        _attend("latent_prompt_packed", "expanded", 1, 6007, 6007, 16, 256, 32, "fp16", docs=7, nope=64,
                value=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "latent_append"] + ["absorbed"] * 3 + ["expanded"] * 2)
    block = rng.choice([16, 32, 48, 64, 64, 128])
    latent, rope = rng.choice([128, 256, 512, 512]), rng.choice([32, 64, 64])
    if kind == "append":
        heads, dim = rng.choice([1, 2, 3, 4, 5, 8]), rng.choice([64, 128, 128, 256])
        group = rng.choice([1, 2, 4, 7])
        rotary = rng.choice([dim, dim, dim // 2])
        return _strip(_append("", _log_int(rng, 1, 8192 * 48 * 128 // ((2 + group) * heads * dim)),
                              heads * group, heads, dim, rng.choice([4, 4, 8]),
                              rng.choice(["bf16", "bf16", "fp16", "fp32"]), rotary, rng.random() < 0.4, block,
                              rng.choice([4096, 200_000]), rng.random() < 0.3))
    if kind == "latent_append":
        stored = rng.choice(["bf16", "bf16", "fp16"])
        return _strip(_latent_append("", _log_int(rng, 1, 16384), rng.choice([1, 5, 16, 32]), latent, rope,
                                     rng.choice([stored, stored, "fp32"]), stored, rng.random() < 0.5,
                                     block, rng.choice([4096, 200_000]), rng.random() < 0.3))
    while True:
        heads = rng.choice([1, 4, 8, 12, 16, 32, 40, 64, 128])
        q = _log_int(rng, 16, 4096) if kind == "expanded" else \
            1 if rng.random() < 0.6 else _log_int(rng, 2, 64)
        kv = max(q, _log_int(rng, 1, 200_000))
        seqs = _log_int(rng, 1, 256)
        # no more pairs than the largest prompt, no more tokens than the longest
        # contexts, and a plain form that fits the card
        if seqs * q * kv * heads <= 2 * 2048 * 10_240 * 32 and seqs * kv <= 64 * 8192 and \
                (kind == "absorbed" or seqs * kv * heads <= 2 * 10_240 * 32 * 4):
            break
    retrieved = q == 1 and kv >= 256 and rng.random() < 0.3
    return _strip(_attend("", kind, seqs, kv, q, heads, latent, rope, rng.choice(["bf16", "bf16", "fp16"]), block,
                          rng.choice([0.0, 0.5, 0.9]), not retrieved and rng.random() < 0.8,
                          rng.choice([0.0, 0.0, 0.5, 0.9]),
                          rng.choice([4, 16]) if retrieved else rng.choice([0, 0, 3, 9]), retrieved,
                          rng.choice([64, 128]) if kind == "expanded" else 0,
                          rng.choice([64, 128]) if kind == "expanded" else 0))


def _strip(case):
    del case["name"]
    return case


# ------------------------------------------------------------------ the inputs
def _lengths(c):
    """Each sequence's context length and number of query rows, from the case."""
    kv, nq = [], []
    for i in range(c["seqs"]):
        f = 1.0 - c["ragged"] * math.modf(i * 0.6180339887)[0]
        nq.append(max(1, round(c["q"] * f)) if c["q"] > 8 else c["q"])
        kv.append(max(nq[-1], round(c["kv"] * f)))
    return kv, nq


def _prefixes(c):
    return [int(c["prefix"] * n) for n in _lengths(c)[0]]


def _documents(n, docs):
    """The document of each of n tokens: unequal runs."""
    cuts = sorted(int(n * math.modf((j + 1) * 0.6180339887)[0]) for j in range(docs - 1))
    at = [0] + cuts + [n]
    return [(at[j], at[j + 1]) for j in range(docs)]


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _randn(g, *shape):
    return torch.randn(*shape, device=DEV, generator=g)


def _table(c):
    """cos and sin of position x frequency, from 64 bits."""
    half = c["rotary"] // 2
    freq = 10_000.0 ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half)
    angle = torch.arange(c["far"], device=DEV, dtype=torch.float64)[:, None] * freq
    return torch.cos(angle).float(), torch.sin(angle).float()


def _rows_in(c, g):
    """Slots in the order of blocks handed out at random, as an allocator gives them (a
    quarter of the rows are padding where `holes`), consecutive positions, the tables."""
    T, n = c["block"], c["n"]
    per = -(-n // T)
    blocks = torch.randperm(2 * per + 1, device=DEV, generator=g)[:per]
    slots = (blocks[:, None] * T + torch.arange(T, device=DEV)).reshape(-1)[:n]
    if c["holes"]:
        slots = torch.where(torch.arange(n, device=DEV) % 4 == 3, -1, slots)
    first = torch.randint(c["far"], (1,), device=DEV, generator=g)
    cos, sin = _table(c)
    return dict(n_blocks=2 * per + 1, slots=slots.contiguous(), cos=cos, sin=sin,
                positions=(first + torch.arange(n, device=DEV)) % c["far"])


def _inputs(c, seed):
    g = _gen(seed)
    dt = DTYPES[c["dtype"]]
    if c["kind"] == "append":
        s = _rows_in(c, g)
        # keys: a few channels are much larger than the others; values: tokens of
        # different size
        gain = 1.0 + 3.0 * (torch.rand(c["heads"], c["dim"], device=DEV, generator=g) < 1 / 16).float()
        s["k"] = (_randn(g, c["n"], c["heads"], c["dim"]) * gain).to(dt)
        s["v"] = (_randn(g, c["n"], c["heads"], c["dim"]) *
                  (0.25 + torch.rand(c["n"], c["heads"], 1, device=DEV, generator=g))).to(dt)
        s["q"] = _randn(g, c["n"], c["q_heads"], c["dim"]).to(dt)
        return s
    if c["kind"] == "latent_append":
        s = _rows_in(c, g)
        s["latent"] = _randn(g, c["n"], c["latent"]).to(dt)
        s["k"] = _randn(g, c["n"], c["rope"]).to(dt)
        s["q"] = _randn(g, c["n"], c["q_heads"], c["rope"]).to(dt)
        return s
    s = {}
    T = c["block"]
    kv, nq = _lengths(c)
    S, width = c["seqs"], -(-max(kv) // T)
    need = [-(-n // T) for n in kv]
    j = torch.arange(width, device=DEV)
    if c["retrieved"]:
        # a store of chunks with a namespace each; a query's list: chunks of its own
        # namespace and, every fourth, of another; a few lists end early
        ns = c["docs"]
        per = max(64, width)
        s["n_blocks"] = ns * per
        b = torch.arange(S, device=DEV)[:, None]
        start = torch.randint(per, (S, 1), device=DEV, generator=g)
        tag = (b + (j % 4 == 3).long()) % ns
        s["blocks"] = ((start + j) % per * ns + tag)
        s["blocks"][(b % 5 == 0) & (j >= width - width // 4)] = -1
        s["tags"] = (torch.arange(s["n_blocks"] * T, device=DEV) // T % ns).int()
        s["q_tags"] = (torch.arange(S, device=DEV) % ns).int()
        kv, nq = [width * T] * S, [1] * S
    else:
        s["n_blocks"] = sum(need) + 3
        order = torch.randperm(s["n_blocks"], device=DEV, generator=g)
        first = torch.tensor([0] + need[:-1], device=DEV).cumsum(0)[:, None]
        nb = torch.tensor(need, device=DEV)[:, None]
        at = torch.clamp(first + j, max=s["n_blocks"] - 1)
        s["blocks"] = torch.where(j < nb, order[at], -1)
        if c["docs"]:
            s["tags"] = torch.full((s["n_blocks"] * T,), -1, dtype=torch.int32, device=DEV)
            qt = []
            for i in range(S):
                t = torch.empty(kv[i], dtype=torch.int32, device=DEV)
                for d, (a, e) in enumerate(_documents(kv[i], c["docs"])):
                    t[a:e] = d
                p = torch.arange(kv[i], device=DEV)
                s["tags"][s["blocks"][i][p // T] * T + p % T] = t
                qt.append(t[kv[i] - nq[i]:])
            s["q_tags"] = torch.cat(qt)
    s["kv_len"] = torch.tensor(kv, dtype=torch.int32, device=DEV)
    s["q_start"] = torch.tensor([0] + nq, device=DEV).cumsum(0).int()
    s["prefix"] = torch.tensor(_prefixes(c), dtype=torch.int32, device=DEV) if c["prefix"] else None
    s["q_rows"], s["even"] = max(nq), min(nq) == max(nq)
    R, P, H = c["latent"], c["rope"], c["heads"]
    s["rows"] = _randn(g, s["n_blocks"] * T, R + P).to(dt)
    if c["kind"] == "absorbed":
        # as the products with w_k leave them: scores of a few units
        s["q"] = (1.5 * _randn(g, sum(nq), H, R + P)).to(dt)
        s["scale"] = (R + P) ** -0.5
    else:
        s["q"] = (1.5 * _randn(g, sum(nq), H, c["nope"] + P)).to(dt)
        # one projection's rows, head by head: keys' before values'
        w = (_randn(g, H, c["nope"] + c["value"], R) * R ** -0.5).to(dt)
        s["w_k"], s["w_v"] = w[:, :c["nope"]], w[:, c["nope"]:]
        s["scale"] = (c["nope"] + P) ** -0.5
    return s


# ------------------------------------------------------------------ the plain form
def _pow2(e):
    """2^e in 64 bits, exact (e: whole numbers from -1022 to 1023)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _over(a, d):
    """a / d, rounded once (by a scalar the GPU would multiply by 1 / d)."""
    return a / torch.full_like(a, d)


def _to_sig(x, bits):
    """x rounded to so many significant bits, ties to even."""
    unit = _pow2(torch.frexp(x)[1] - bits)
    return torch.round(x / unit) * unit


def _quantise(x, bits):
    """What the cache stands for, as codes and the scale of each code (64 bits: half steps
    are told from their neighbours)."""
    x = x.double()
    n, h, d = x.shape
    a = x.abs().amax(-1, keepdim=True)
    if bits == 8:
        s = torch.clamp(_to_sig(_over(a, 127.0), 8), min=2.0 ** -100)
        code = torch.clamp(torch.round(x / s), -127, 127)
        return code.to(torch.int8), s.float()
    t = torch.clamp(torch.frexp(_over(a, 7.0))[1] - 1, -100, 125)
    t = torch.where(a == 0, -100, t)
    x = x.view(n, h, d // 16, 16)
    r = _over(x.abs().amax(-1), 7.0) / _pow2(t)
    e = torch.clamp(_to_sig(r, 5), 2.0 ** -15, 1.9375)
    s = e * _pow2(t)
    code = torch.clamp(torch.round(x / s[..., None]), -7, 7) + 8
    code = code.to(torch.uint8).view(n, h, d)
    return code[..., 0::2] | code[..., 1::2] << 4, s.float()


def _dequantise(code, scale, bits):
    if bits == 8:
        return code.float() * scale
    code = torch.stack((code & 15, code >> 4), -1).float() - 8.0
    return (code.view(*scale.shape, 16) * scale[..., None]).flatten(-2)


def _rotate(x, s, c, wide=False):
    """x [n, heads, d] with its first `rotary` values turned."""
    up = torch.float64 if wide else torch.float32
    x, r = x.to(up), c["rotary"]
    co, si = (s[t][s["positions"]].to(up)[:, None] for t in ("cos", "sin"))
    if c["pairs"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack((a * co - b * si, b * co + a * si), -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat((a * co - b * si, b * co + a * si), -1)
    return torch.cat((y, x[..., r:]), -1)


def _plain_append(s, c):
    at = torch.where(s["slots"] < 0, s["n_blocks"] * c["block"], s["slots"])
    real = (s["slots"] >= 0)[:, None, None]
    k = _rotate(s["k"], s, c)
    q = (_rotate(s["q"], s, c) * real).to(s["q"].dtype)
    (kc, ks), (vc, vs) = s["cache"]
    kc[at], ks[at] = _quantise(k, c["bits"])
    vc[at], vs[at] = _quantise(s["v"].float(), c["bits"])
    k = (_dequantise(kc[at], ks[at], c["bits"]) * real).to(torch.bfloat16)
    v = (_dequantise(vc[at], vs[at], c["bits"]) * real).to(torch.bfloat16)
    return q, k, v


def _plain_latent_append(s, c):
    at = torch.where(s["slots"] < 0, s["n_blocks"] * c["block"], s["slots"])
    q = (_rotate(s["q"], s, c) * (s["slots"] >= 0)[:, None, None]).to(s["q"].dtype)
    rows = torch.cat((s["latent"].float(), _rotate(s["k"][:, None], s, c)[:, 0]), -1)
    s["cache"][at] = rows.to(s["cache"].dtype)
    return q, s["cache"][:-1]


def _plain_attend(s, c):
    """All sequences at once, padded to the longest."""
    T, H, R, P = c["block"], c["heads"], c["latent"], c["rope"]
    blocks = s["blocks"]
    S, L, Q = blocks.shape[0], blocks.shape[1] * T, s["q_rows"]
    j = torch.arange(L, device=DEV)
    at = blocks.repeat_interleave(T, 1) * T + j % T
    listed_ = (at >= 0) & (j < s["kv_len"][:, None])
    at = torch.where(listed_, at, 0)
    nq = (s["q_start"][1:] - s["q_start"][:-1])[:, None]
    i = torch.arange(Q, device=DEV)
    row = torch.where(i < nq, s["q_start"][:-1, None] + i, 0)                # [S, Q]
    pos = s["kv_len"][:, None] - nq + i
    tok = s["rows"][at].float()                                              # [S, L, R + P]
    q = s["q"][row].float() * s["scale"]                                     # [S, Q, H, ...]
    if c["kind"] == "absorbed":
        z = (q.reshape(S, Q * H, R + P) @ tok.transpose(1, 2)).view(S, Q, H, L).transpose(1, 2)
    else:
        N = c["nope"]
        lat = tok[:, None, :, :R]
        k = lat @ s["w_k"].float().transpose(1, 2)                           # [S, H, L, N]
        q = q.transpose(1, 2)
        z = q[..., :N] @ k.transpose(2, 3) + q[..., N:] @ tok[:, None, :, R:].transpose(2, 3)
    seen = listed_[:, None, :].expand(S, Q, L)
    if c["causal"]:
        near = j <= pos[..., None]
        if s["prefix"] is not None:
            near = near | (j < s["prefix"][:, None, None])
        seen = seen & near
    if c["docs"]:
        seen = seen & (s["tags"][at][:, None, :] == s["q_tags"][row][..., None])
    z = z.masked_fill(~seen[:, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(z - top)
    total = p.sum(-1, keepdim=True)                                          # [S, H, Q, 1]
    real = i < nq
    if c["kind"] == "absorbed":
        o = (p.transpose(1, 2).reshape(S, Q * H, L) @ tok[..., :R]).view(S, Q, H, R)
        o = torch.where(total.transpose(1, 2) > 0, o / total.transpose(1, 2), 0.0)
        lse = (top + torch.log(total))[..., 0].transpose(1, 2)
        return o[real].to(s["q"].dtype), lse[real].contiguous()
    o = p @ (lat @ s["w_v"].float().transpose(1, 2))
    o = torch.where(total > 0, o / total, 0.0)
    return o.transpose(1, 2)[real].to(s["q"].dtype)


# ------------------------------------------------------------------ the calls
def prepare(case, seed):
    c = case
    s = _inputs(c, seed)
    s["case"] = c
    if own:
        from paper_2607_05708_gb300 import KVCache, LatentCache
        if c["kind"] == "append":
            s["handle"] = KVCache(s["n_blocks"], c["heads"], c["dim"], block_tokens=c["block"], bits=c["bits"])
        else:
            s["handle"] = LatentCache(s["n_blocks"], c["latent"], c["rope"], block_tokens=c["block"],
                                      dtype=DTYPES[c.get("stored", c["dtype"])], tagged="tags" in s)
        if "rows" in s:
            rows = s.pop("rows")
            s["handle"].append(rows[:, :c["latent"]], rows[:, c["latent"]:], torch.arange(len(rows), device=DEV),
                               tags=s.get("tags"))
    elif c["kind"] == "append":
        n, h, d = s["n_blocks"] * c["block"] + 1, c["heads"], c["dim"]
        code = ((n, h, d // 2), torch.uint8) if c["bits"] == 4 else ((n, h, d), torch.int8)
        s["cache"] = [(torch.zeros(code[0], dtype=code[1], device=DEV),
                       torch.zeros(n, h, d // 16 if c["bits"] == 4 else 1, device=DEV)) for _ in range(2)]
    elif c["kind"] == "latent_append":
        s["cache"] = torch.zeros(s["n_blocks"] * c["block"] + 1, c["latent"] + c["rope"],
                                 dtype=DTYPES[c["stored"]], device=DEV)
    return s


def run(state):
    s, c = state, state["case"]
    if not own:
        return {"append": _plain_append, "latent_append": _plain_latent_append}.get(c["kind"], _plain_attend)(s, c)
    h = s["handle"]
    if c["kind"] == "append":
        q = h.append(s["k"], s["v"], s["slots"], s["positions"], s["cos"], s["sin"], q=s["q"],
                     interleaved=c["pairs"])
        return (q, *h.read(s["slots"]))
    if c["kind"] == "latent_append":
        q = h.append(s["latent"], s["k"], s["slots"], s["positions"], s["cos"], s["sin"], q=s["q"],
                     interleaved=c["pairs"])
        return q, h.data
    q_start = None if s["even"] else s["q_start"]
    if c["kind"] == "absorbed":
        return h.attend(s["q"], s["blocks"], s["scale"], kv_len=s["kv_len"], q_start=q_start, causal=c["causal"],
                        prefix_len=s["prefix"], q_tags=s.get("q_tags"))
    return h.attend_expanded(s["q"], s["w_k"], s["w_v"], s["blocks"], kv_len=s["kv_len"], q_start=q_start,
                             causal=c["causal"], prefix_len=s["prefix"], q_tags=s.get("q_tags"))


def _pairs(c):
    """Visible (row, key) pairs of one head, and the tokens that some row sees."""
    kv, nq = _lengths(c)
    if c["retrieved"]:
        T = c["block"]
        width = -(-max(kv) // T)
        seen = 0
        for b in range(c["seqs"]):
            most = width - width // 4 if b % 5 == 0 else width
            seen += T * sum(1 for j in range(most) if j % 4 != 3)
        return seen, seen
    pairs = tokens = 0
    for n, r, pre in zip(kv, nq, _prefixes(c)):
        first = n - r                       # position of the first row
        for a, e in _documents(n, c["docs"]) if c["docs"] else [(0, n)]:
            if not c["causal"]:
                rows = max(0, e - max(a, first)) if c["docs"] else r
                pairs += rows * (e - a)
                tokens += (e - a) if rows else 0
                continue
            i0, i1 = (max(a, first), e) if c["docs"] else (first, n)
            if i1 <= i0:
                continue
            tokens += e - a
            p = min(max(pre, a), e) - a     # the prefix's part of the document
            # row at position x sees max(p, x - a + 1) keys
            low = max(0, min(i1, a + p) - i0)
            pairs += low * p
            x0, x1 = i0 + low, i1
            pairs += (x1 - x0) * ((x0 - a + 1) + (x1 - a)) // 2
    return pairs, tokens


def work(case):
    c = case
    if c["kind"] in ("append", "latent_append"):
        real = c["n"] - (c["n"] // 4 if c["holes"] else 0)
        size = SIZE[c["dtype"]]
        # tables' rows, query rows read and written
        moved = real * c["rotary"] * 4
        if c["kind"] == "append":
            d = c["dim"]
            stored = d + d // 8 + 2 if c["bits"] == 4 else 2 * d + 4
            moved += (real + c["n"]) * c["q_heads"] * d * size
            moved += real * c["heads"] * (2 * d * size + 2 * stored) + c["n"] * c["heads"] * d * 4
        else:
            moved += (real + c["n"]) * c["q_heads"] * c["rope"] * size
            moved += real * (c["latent"] + c["rope"]) * (size + 2)
        return {"bytes": moved, "flops": 0}
    pairs, tokens = _pairs(c)
    rows, H, R, P = sum(_lengths(c)[1]), c["heads"], c["latent"], c["rope"]
    if c["kind"] == "absorbed":
        return {"bytes": tokens * (R + P) * 2 + rows * H * (2 * (2 * R + P) + 4),
                "flops": 2 * pairs * H * (2 * R + P)}
    N, V = c["nope"], c["value"]
    return {"bytes": tokens * (R + P) * 2 + rows * H * 2 * (N + P + V) + H * (N + V) * R * 2,
            "flops": 2 * pairs * H * (N + P + V) + 2 * tokens * H * (N + V) * R}


# ------------------------------------------------------------------ in 64 bits
def _exact_values(x, bits):
    """What the cache stands for after x is written: the nearest of the levels that the
    format has, from tables of the midpoints between them."""
    x = x.double()
    n, h, d = x.shape
    a = x.abs().amax(-1, keepdim=True)
    power = torch.tensor([2.0 ** i for i in range(-160, 131)], dtype=torch.float64, device=DEV)
    if bits == 8:
        # p <= a / 127 < 2 p
        p = power[torch.bucketize(a, 127 * power, right=True).sub(1).clamp(min=0)]
        y = a * 128 / (127 * p)
        f = torch.floor(y)
        f = f + ((y - f > 0.5) | ((y - f == 0.5) & (f % 2 == 1))).double()
        s = (f * p / 128).clamp(min=2.0 ** -100)
        top, y = 127, x / s
    else:
        p = power[torch.bucketize(a, 7 * power, right=True).sub(1).clamp(min=0)]
        p = p.clamp(2.0 ** -100, 2.0 ** 125)
        level = torch.tensor([(1 + b % 16 / 16) * 2.0 ** (b // 16 - 15) for b in range(256)],
                             dtype=torch.float64, device=DEV)
        mid = 7 * (level[1:] + level[:-1]) / 2
        r = x.view(n, h, d // 16, 16).abs().amax(-1) / p
        i = torch.bucketize(r, mid)                      # mid[i-1] < r <= mid[i]
        tie = (i < 255) & (r == mid[i.clamp(max=254)])
        i = torch.where(tie & (i % 2 == 1), i + 1, i)
        s = (level[i] * p).repeat_interleave(16, -1)
        top, y = 7, x / s
    f = torch.floor(y)
    rest = y - f
    c = f + ((rest > 0.5) | ((rest == 0.5) & (f % 2 != 0))).double()
    return c.clamp(-top, top) * s


def _exact_rotation(x, s, c):
    """Each pair as a complex number, times that of its angle."""
    x, r = x.double(), c["rotary"]
    turn = torch.complex(s["cos"].double(), s["sin"].double())[s["positions"]][:, None]
    head = x[..., :r].unflatten(-1, (r // 2, 2) if c["pairs"] else (2, r // 2))
    if not c["pairs"]:
        head = head.transpose(-1, -2)
    y = torch.view_as_real(torch.view_as_complex(head.contiguous()) * turn)
    if not c["pairs"]:
        y = y.transpose(-1, -2)
    out = x.clone()
    out[..., :r] = y.flatten(-2)
    return out


def exact(case, seed):
    c = case
    s = _inputs(c, seed)
    T = c["block"]
    if c["kind"] in ("append", "latent_append"):
        real = s["slots"] >= 0
        q = _exact_rotation(s["q"], s, c)
        q[~real] = 0
        if c["kind"] == "append":
            # (keys are quantised from the rotation's 32-bit result)
            k = _exact_values(_exact_rotation(s["k"], s, c).float(), c["bits"])
            v = _exact_values(s["v"], c["bits"])
            k[~real], v[~real] = 0, 0
            return q, k, v
        data = torch.zeros(s["n_blocks"] * T, c["latent"] + c["rope"], dtype=torch.float64, device=DEV)
        data[s["slots"][real], :c["latent"]] = s["latent"][real].double()
        data[s["slots"][real], c["latent"]:] = _exact_rotation(s["k"][:, None], s, c)[real, 0]
        return q, data
    R, H = c["latent"], c["heads"]
    wide = R if c["kind"] == "absorbed" else c["value"]
    rows = s["q_start"].tolist()
    out = torch.zeros(rows[-1], H, wide, dtype=torch.float64, device=DEV)
    lse = torch.full((rows[-1], H), -math.inf, dtype=torch.float64, device=DEV)
    for b, n in enumerate(s["kv_len"].tolist()):
        r0, r1 = rows[b], rows[b + 1]
        tok = torch.arange(n, device=DEV)
        blk = s["blocks"][b][tok // T]
        tok = tok[blk >= 0]
        at = blk[blk >= 0] * T + tok % T
        if not len(tok):
            continue
        X = s["rows"][at].double()
        pos = n - (r1 - r0) + torch.arange(r1 - r0, device=DEV)
        step = max(1, (1 << 27) // len(tok))
        for i0 in range(0, r1 - r0, step):
            i1 = min(r1 - r0, i0 + step)
            m = torch.ones(i1 - i0, len(tok), dtype=torch.bool, device=DEV)
            if c["causal"]:
                last = pos[i0:i1]
                if s["prefix"] is not None:
                    last = torch.maximum(last, s["prefix"][b].long() - 1)
                m &= tok[None] <= last[:, None]
            if c["docs"]:
                m &= s["q_tags"][r0 + i0:r0 + i1][:, None] == s["tags"][at][None]
            for h in range(H):
                q = s["q"][r0 + i0:r0 + i1, h].double()
                K, V = X, X[:, :R]
                if c["kind"] == "expanded":
                    K = torch.cat((X[:, :R] @ s["w_k"][h].double().T, X[:, R:]), -1)
                    V = X[:, :R] @ s["w_v"][h].double().T
                z = torch.where(m, q @ K.T * s["scale"], -math.inf)
                total = torch.logsumexp(z, -1)
                w = torch.where(m, torch.exp(z - total[:, None]), 0.0)
                out[r0 + i0:r0 + i1, h] = w @ V
                lse[r0 + i0:r0 + i1, h] = total
    return (out, lse) if c["kind"] == "absorbed" else out
