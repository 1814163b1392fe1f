"""Cases of latent attention and its cache: attention whose keys and values come from one shared latent vector a token.

A cached token is a row of R latent values c and P rotary values r, the same for all H query heads.  `op` says which operator a
case measures:

  append    rows written into the pool; with the 8-bit pool they are read back too, so that the values they stand for come out
  gather    cached rows read back, decoded
  absorbed  queries [T, H, R + P] against rows (c, r); the values are c itself; out [T, H, R]
  expanded  queries [T, H, N + P] against keys (W_k c, r) and values W_v c of every head; out [T, H, N]

A batch of the attention operators: `docs` shared cached prefixes of `doc_lo..doc_hi` tokens, a request sits behind one of them
drawn uniformly, has `own_lo..own_hi` cached tokens of its own and brings `ext_lo..ext_hi` new ones.  Lengths and places are drawn
from `lens`, so that a case is the same work for every seed; page order and all values come from the seed.

The pool: rows by slot.  fp32 and bf16: R + P elements a row.  8 bits: a row is R one-byte codes (4 exponent bits, 3 mantissa bits,
largest 448) and P bf16 values; behind all rows lies one int8 exponent k a slot, c = code * 2^k, the smallest k with
max|c| 2^-k <= 448.
"""
import random

import torch

own = False

_DEFAULTS = dict(op="absorbed", dtype="bf16", H=16, R=512, P=64, N=128, num_slots=65536, page=16, B=1, docs=1, doc_lo=0, doc_hi=0,
                 own_lo=0, own_hi=0, ext_lo=1, ext_hi=1, rows=0, lens=0)


def listed():
    return [
        # a decode batch of 48 requests writes one new row each: the smallest call, a launch and its latency
        dict(name="append_decode", op="append", rows=48, num_slots=16384),
        # a prefill chunk is written into the 8-bit pool and read back as stored
        dict(name="append_fp8_read_back", op="append", dtype="bf16_kv8", rows=16384, num_slots=65536),
        # cached documents are read back from the 8-bit pool, to be moved or expanded elsewhere
        dict(name="gather_fp8", op="gather", dtype="bf16_kv8", rows=100003, num_slots=131072),
        # fp32 rows of the smaller latent, an odd number of them, page size 1
        dict(name="gather_fp32", op="gather", dtype="f32", R=256, rows=5001, num_slots=8192, page=1),
        # one request being decoded on a shard of 16 heads: latency
        dict(name="decode_one", B=1, doc_lo=1800, doc_hi=1800, own_lo=333, own_hi=333),
        # a full decode batch with all 128 heads on one card, ragged lengths: matrix units and memory about equally busy
        dict(name="decode_batch", H=128, B=128, docs=4, doc_lo=500, doc_hi=1800, own_lo=200, own_hi=6000, num_slots=524288),
        # decoding on a shard of 16 heads over long conversations in the 8-bit pool: memory
        dict(name="decode_long_fp8", dtype="bf16_kv8", H=16, B=48, own_lo=2000, own_hi=24000, num_slots=1048576),
        # short questions to long shared documents, a chunk of new tokens each; the most arithmetic
        dict(name="extend_doc_qa", H=64, B=16, docs=4, doc_lo=16384, doc_hi=16384, ext_lo=20, ext_hi=80, num_slots=131072),
        # fp32, the smaller latent, a few heads and new tokens behind a short prefix
        dict(name="extend_fp32", dtype="f32", H=4, R=256, B=4, doc_lo=96, doc_hi=96, ext_lo=16, ext_hi=32, num_slots=512, page=1),
        # new prompts behind a short system prompt, expanded keys and values on a shard of 16 heads
        dict(name="expanded_prefill", op="expanded", H=16, B=8, doc_lo=57, doc_hi=57, ext_lo=300, ext_hi=3500),
        # agents behind shared histories with long extends: every shared token is expanded once
        dict(name="expanded_agents", op="expanded", H=32, B=24, docs=4, doc_lo=1500, doc_hi=2000, ext_lo=200, ext_hi=1000),
        # one chunk of a long prompt over its cached part in the 8-bit pool: few rows, a long key axis
        dict(name="expanded_chunk_fp8", op="expanded", dtype="bf16_kv8", H=16, B=1, doc_lo=12000, doc_hi=12000, ext_lo=500, ext_hi=500),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def _range(rng, lo, hi):
    a, b = sorted((_log(rng, lo, hi), _log(rng, lo, hi)))
    return a, b


def draw(rng):
    while True:
        c = _draw(rng)
        w = work(c)
        # no more than the largest listed ones, in arithmetic, in bytes and in what the plain form holds (padded scores and rows)
        p = _plan(dict(_DEFAULTS, **c))
        if w["flops"] > (2e9 if c["dtype"] == "f32" else 4e11 if c["op"] == "absorbed" else 9e11) or w["bytes"] > 6e8:
            continue
        if c["op"] in ("append", "gather"):
            return c
        k = max(a + e for a, e in zip(p["prefix"], p["ext"]))
        pad = c["B"] * k * (c["H"] * max(p["ext"]) + c["R"] + (2 * c["H"] * 128 if c["op"] == "expanded" else 0))
        if pad <= 3e9 and 2 * p["slots"] <= c["num_slots"]:
            return c


def _draw(rng):
    op = rng.choice(["append", "gather", "absorbed", "absorbed", "absorbed", "expanded", "expanded"])
    c = dict(op=op, lens=rng.randrange(1 << 30), dtype=rng.choice(["bf16", "bf16", "bf16_kv8", "bf16_kv8", "f32"]),
             R=rng.choice([512, 512, 512, 256]), page=rng.choice([16, 16, 1, 64]), num_slots=524288)
    if op in ("append", "gather"):
        c["rows"] = _log(rng, 1, 120000)
        c["num_slots"] = 131072
        return c
    c["H"] = rng.choice([8, 16, 16, 20, 32, 64, 128]) if c["dtype"] != "f32" else rng.choice([1, 2, 4, 5, 8])
    c["docs"] = _log(rng, 1, 6)
    if c["dtype"] == "f32":
        c.update(B=rng.randint(1, 8))
        c["doc_lo"], c["doc_hi"] = _range(rng, 1, 400)
        c["ext_lo"], c["ext_hi"] = _range(rng, 1, 40)
    elif op == "expanded":
        c.update(B=_log(rng, 1, 24), N=rng.choice([128, 128, 64]))
        c["doc_lo"], c["doc_hi"] = _range(rng, 1, 8000)
        c["ext_lo"], c["ext_hi"] = _range(rng, 100, 3500)
    elif rng.random() < 0.6:
        c.update(B=_log(rng, 1, 128))
        c["doc_lo"], c["doc_hi"] = _range(rng, 100, 4000)
        c["own_lo"], c["own_hi"] = _range(rng, 1, 16000)
    else:
        c.update(B=_log(rng, 1, 32))
        c["doc_lo"], c["doc_hi"] = _range(rng, 100, 16000)
        c["ext_lo"], c["ext_hi"] = _range(rng, 2, 200)
    return c


# ---- the batch of a case: lengths and places, from the case alone --------------------------------------------------------
def _plan(c):
    rng = random.Random("lengths %d" % c.get("lens", 0))
    c = dict(_DEFAULTS, **c)
    doc_len = [rng.randint(c["doc_lo"], c["doc_hi"]) for _ in range(c["docs"])]
    doc = [rng.randrange(c["docs"]) for _ in range(c["B"])]
    mine = [rng.randint(c["own_lo"], c["own_hi"]) for _ in range(c["B"])]
    ext = [rng.randint(c["ext_lo"], c["ext_hi"]) for _ in range(c["B"])]
    page = c["page"]
    slots = sum(-(-n // page) * page for n in doc_len + mine)
    return dict(doc_len=doc_len, doc=doc, mine=mine, ext=ext, prefix=[doc_len[d] + o for d, o in zip(doc, mine)], slots=slots)


def _row_bytes(c):
    return 4 * (c["R"] + c["P"]) if c["dtype"] == "f32" else c["R"] + 2 * c["P"] + 1 if c["dtype"] == "bf16_kv8" else 2 * (c["R"] + c["P"])


def work(case):
    c = dict(_DEFAULTS, **case)
    el, width, row = 4 if c["dtype"] == "f32" else 2, c["R"] + c["P"], _row_bytes(c)
    if c["op"] in ("append", "gather"):
        by = c["rows"] * (4 + row + el * width)
        if c["op"] == "append" and c["dtype"] == "bf16_kv8":
            by *= 2
        return {"bytes": float(by), "flops": 0.0}
    p = _plan(c)
    t, keys = sum(p["ext"]), sum(p["doc_len"][d] for d in set(p["doc"])) + sum(p["mine"])
    pairs = sum(e * q + e * (e + 1) / 2 for q, e in zip(p["prefix"], p["ext"]))
    by = keys * row + 4 * sum(p["prefix"]) + t * width * el
    if c["op"] == "absorbed":
        return {"bytes": float(by + t * c["H"] * (width + c["R"]) * el), "flops": 2.0 * c["H"] * pairs * (width + c["R"])}
    by += t * c["H"] * (2 * c["N"] + c["P"]) * el + 2 * c["H"] * c["N"] * c["R"] * el
    return {"bytes": float(by), "flops": 2.0 * c["H"] * (pairs * (2 * c["N"] + c["P"]) + (keys + t) * 2 * c["N"] * c["R"])}


# ---- inputs ----------------------------------------------------------------------------------------------------------------
def _type(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _power(k):
    """2^k in 32 bits, exactly (torch's exp2 and ldexp on a GPU are off in the last place)."""
    return ((k.int() + 127) << 23).view(torch.float32)


def _stored(rows, c):
    """Rows [n, R + P] as the pool's bytes: [n, row bytes] and, for the 8-bit pool, the exponents [n]."""
    if c["dtype"] != "bf16_kv8":
        return rows.contiguous().view(torch.uint8), None
    lat = rows[:, :c["R"]].float()
    m, e = torch.frexp(lat.abs().amax(1))                 # max = m 2^e, m in [0.5, 1); 448 = 0.875 2^9
    k = torch.where(m > 0, e - 9 + (m > 0.875).int(), torch.zeros_like(e))
    codes = (lat * _power(-k)[:, None]).to(torch.float8_e4m3fn)
    return torch.cat([codes.view(torch.uint8), rows[:, c["R"]:].contiguous().view(torch.uint8)], 1), k.to(torch.int8)


def prepare(case, seed):
    c = dict(_DEFAULTS, **case)
    dev, dt = torch.device("cuda"), _type(c)
    gen = torch.Generator(device=dev).manual_seed(int(seed) * 7919 + c["lens"] % 7919)
    width, n = c["R"] + c["P"], c["num_slots"]

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=gen, device=dev) * std).to(dt)

    pages = torch.randperm(n // c["page"], generator=gen, device=dev)
    order = (pages[:, None] * c["page"] + torch.arange(c["page"], device=dev)).view(-1).int()
    s = dict(c=c, kw=dict(num_slots=n, kv8=c["dtype"] == "bf16_kv8"))
    row = _row_bytes(c) - (c["dtype"] == "bf16_kv8")
    pool = torch.zeros(n * _row_bytes(c), dtype=torch.uint8, device=dev)
    s["pool"] = pool

    def fill(slots):
        for at in range(0, len(slots), 65536):
            part = slots[at:at + 65536].long()
            by, exps = _stored(normal(len(part), width), c)
            pool[:n * row].view(n, row)[part] = by
            if exps is not None:
                pool[n * row:].view(torch.int8)[part] = exps

    if c["op"] in ("append", "gather"):
        s["slots"] = order[:c["rows"]].contiguous()
        if c["op"] == "gather":
            s["slots"] = s["slots"][torch.randperm(c["rows"], generator=gen, device=dev)].contiguous()
            fill(s["slots"])
        else:
            s["rows"] = normal(c["rows"], width)
        return s

    p = _plan(c)
    taken = 0

    def take(k):
        nonlocal taken
        at, taken = taken, taken + -(-k // c["page"]) * c["page"]
        return order[at:at + k]

    docs = [take(k) for k in p["doc_len"]]
    mine = [take(k) for k in p["mine"]]
    fill(order[:taken])
    t = sum(p["ext"])
    none = torch.full((max(p["ext"]),), -1, dtype=torch.int32, device=dev)
    s["slot_idx"] = torch.cat([x for r in range(c["B"]) for x in (docs[p["doc"][r]], mine[r], none[:p["ext"][r]])])
    total = [a + e for a, e in zip(p["prefix"], p["ext"])]

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device=dev)

    def starts(x):
        return ints([sum(x[:i]) for i in range(len(x) + 1)])

    s["offsets"], s["prefix_len"], s["ext_len"], s["ext_offsets"] = starts(total), ints(p["prefix"]), ints(p["ext"]), starts(p["ext"])
    s["max_kv_len"], s["max_ext_len"] = max(total), max(p["ext"])
    s["rows"] = normal(t, width)
    s["scale"] = (128 + c["P"]) ** -0.5
    if c["op"] == "absorbed":
        s["q"] = normal(t, c["H"], width)
    else:
        s["q"] = normal(t, c["H"], c["N"] + c["P"])
        s["w_k"] = normal(c["H"], c["N"], c["R"], std=c["R"] ** -0.5)
        s["w_v"] = normal(c["H"], c["N"], c["R"], std=c["R"] ** -0.5)
    return s


# ---- one pass --------------------------------------------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2407_00023_amd import binding as pa
    c, kw = s["c"], s["kw"]
    if c["op"] == "append":
        pa.append_latent(s["pool"], s["slots"], s["rows"], rope_dim=c["P"], **kw)
        if not kw["kv8"]:
            return s["pool"].view(_type(c))
    if c["op"] in ("append", "gather"):
        return pa.gather_latent(s["pool"], s["slots"], latent_dim=c["R"], rope_dim=c["P"], dtype=_type(c), **kw)
    batch = (s["slot_idx"], s["offsets"], s["prefix_len"], s["ext_len"], s["ext_offsets"], s["scale"])
    if c["op"] == "absorbed":
        return pa.latent_attention(s["q"], s["rows"], s["pool"], *batch, rope_dim=c["P"], max_kv_len=s["max_kv_len"], **kw)
    return pa.latent_attention_expanded(s["q"], s["rows"], s["w_k"], s["w_v"], s["pool"], *batch, max_kv_len=s["max_kv_len"], **kw)


def _read(s, slots):
    """The rows of these slots, in 32 bits."""
    c, pool, n = s["c"], s["pool"], s["c"]["num_slots"]
    if c["dtype"] != "bf16_kv8":
        return pool.view(_type(c)).view(n, -1)[slots].float()
    row = c["R"] + 2 * c["P"]
    by = pool[:n * row].view(n, row)[slots]
    k = pool[n * row:].view(torch.int8)[slots].int()
    lat = by[..., :c["R"]].contiguous().view(torch.float8_e4m3fn).float() * _power(k)[..., None]
    return torch.cat([lat, by[..., c["R"]:].contiguous().view(torch.bfloat16).float()], -1)


def _run_plain(s):
    c = s["c"]
    if c["op"] == "append":
        n, at = c["num_slots"], s["slots"].long()
        by, exps = _stored(s["rows"], c)
        row = by.shape[1]
        s["pool"][:n * row].view(n, row)[at] = by
        if exps is None:
            return s["pool"].view(_type(c))
        s["pool"][n * row:].view(torch.int8)[at] = exps
    if c["op"] in ("append", "gather"):
        return _read(s, s["slots"].long()).to(_type(c))

    # requests padded to the longest: key rows [B, K, R + P], queries [B, E, H, ...]
    dev, K, E, H, R = s["pool"].device, s["max_kv_len"], s["max_ext_len"], c["H"], c["R"]
    pre, ext, first = s["prefix_len"].long()[:, None], s["ext_len"].long()[:, None], s["ext_offsets"].long()[:-1, None]
    j, i = torch.arange(K, device=dev)[None], torch.arange(E, device=dev)[None]
    slots = s["slot_idx"][(s["offsets"].long()[:-1, None] + j).clamp(max=len(s["slot_idx"]) - 1)].long()
    cached, fresh = j < pre, (j >= pre) & (j < pre + ext)
    rows = _read(s, torch.where(cached, slots, torch.zeros_like(slots)))
    new = s["rows"].float()[torch.where(fresh, first + j - pre, torch.zeros_like(j))]
    rows = torch.where(cached[..., None], rows, torch.where(fresh[..., None], new, torch.zeros_like(new)))
    there = i < ext
    q = s["q"].float()[torch.where(there, first + i, torch.zeros_like(i))]
    seen = (j[:, None, :] <= pre[:, :, None] + i[..., None]) & (j[:, None, :] < (pre + ext)[:, :, None])     # [B, E, K]
    if c["op"] == "absorbed":
        score = torch.matmul(q.flatten(1, 2), rows.transpose(1, 2)).view(-1, E, H, K)
        score = score.mul_(s["scale"]).masked_fill_(~seen[:, :, None], -torch.inf)
        score = torch.exp(score.sub_(score.amax(-1, keepdim=True)))
        out = torch.matmul(score.flatten(1, 2), rows[..., :R]).view(-1, E, H, R) / score.sum(-1, keepdim=True)
    else:
        N = c["N"]
        lat, q = rows[..., :R], q.transpose(1, 2)                                       # [B, K, R], [B, H, E, N + P]
        k = torch.matmul(lat[:, None], s["w_k"].float().transpose(1, 2)[None])          # [B, H, K, N]
        v = torch.matmul(lat[:, None], s["w_v"].float().transpose(1, 2)[None])
        score = torch.matmul(q[..., :N], k.transpose(2, 3)) + torch.matmul(q[..., N:], rows[:, None, :, R:].transpose(2, 3))
        score = score.mul_(s["scale"]).masked_fill_(~seen[:, None], -torch.inf)
        score = torch.exp(score.sub_(score.amax(-1, keepdim=True)))
        out = (torch.matmul(score, v) / score.sum(-1, keepdim=True)).transpose(1, 2)
    return out[there].to(_type(c))


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    n, R, P = c["num_slots"], c["R"], c["P"]
    row = R + 2 * P

    def two(e):
        return ((e.long() + 1023) << 52).view(torch.float64)

    def quantised(x):
        """A row's latent values rounded to 1 + 3 bits above 2^-6 2^k and to multiples of 2^-9 2^k below."""
        top = x.abs().amax(1, keepdim=True)
        k = torch.frexp(top / 448).exponent          # top / 448 <= 2^k, equal at most where it is 2^(k - 1)
        k = torch.where(top == 0, 0, torch.where(top <= 448 * two(k - 1), k - 1, k))
        y = x / two(k)
        step = two(torch.frexp(y.abs().clamp(min=2.0 ** -6)).exponent - 4)
        return torch.round(y / step) * step * two(k)

    def pool_rows(at):
        if c["dtype"] != "bf16_kv8":
            return s["pool"].view(_type(c)).view(n, R + P)[at].double()
        by = s["pool"][:n * row].view(n, row)[at].int()
        code, k = by[:, :R], s["pool"][n * row:].view(torch.int8)[at]
        e, m = (code >> 3) & 15, (code & 7).double()
        size = torch.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * two(e - 7))
        lat = torch.where(code >= 128, -size, size) * two(k)[:, None]
        bits = by[:, R::2] | (by[:, R + 1::2] << 8)
        return torch.cat([lat, (bits << 16).view(torch.float32).double()], 1)

    if c["op"] == "append":
        x = s["rows"].double()
        if c["dtype"] == "bf16_kv8":
            return torch.cat([quantised(x[:, :R]), x[:, R:]], 1)
        pool = torch.zeros(n, R + P, dtype=torch.float64, device=x.device)
        pool[s["slots"].long()] = x
        return pool.view(-1)
    if c["op"] == "gather":
        return pool_rows(s["slots"].long())
    p, H, outs = _plan(c), c["H"], []
    at, t = 0, 0
    for a, e in zip(p["prefix"], p["ext"]):
        keys = torch.cat([pool_rows(s["slot_idx"][at:at + a].long()), s["rows"][t:t + e].double()])
        q = s["q"][t:t + e].double()
        hidden = torch.arange(a + e, device=q.device)[None] > a + torch.arange(e, device=q.device)[:, None]
        for h in range(H):
            if c["op"] == "absorbed":
                k, v = keys, keys[:, :R]
            else:
                k = torch.cat([keys[:, :R] @ s["w_k"][h].double().T, keys[:, R:]], 1)
                v = keys[:, :R] @ s["w_v"][h].double().T
            z = (q[:, h] @ k.T * s["scale"]).masked_fill(hidden, -torch.inf)
            outs.append(torch.softmax(z, 1) @ v)
        at, t = at + a + e, t + e
    sizes = [e for e in p["ext"] for _ in range(H)]
    width = outs[0].shape[1]
    out = torch.empty(t, H, width, dtype=torch.float64, device=outs[0].device)
    first = 0
    for n_out, (o, e) in enumerate(zip(outs, sizes)):
        h = n_out % H
        out[first:first + e, h] = o
        first += e if h == H - 1 else 0
    return out
