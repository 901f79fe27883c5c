"""Operators of serving tokens to many tenants: what is timed of them, and their plain forms.

* ``append`` and ``read``: rows of keys and values written to a paged cache, and read from it. A cache is a pool of
  pages of ``page`` tokens; a table names each sequence's pages in order. Values are bf16, or e4m3 with an
  exponent per token and head (``s`` = 2^(exponent - 127), the smallest one with max |x| / s <= 448).
* ``attention``: new tokens (one for each sequence, or a few drafted ones) over such a cache, in causal order, with a
  sliding window and first keys that stay visible (sinks).
* ``lora``: low-rank adapters of many requests at once beside a shared projection,
  ``y[m] = act(base[m] + s_a B_a A_a x[m])`` with ``a = adapter[m]`` (negative: none).

Functions: ``listed`` and ``draw`` give cases, ``prepare`` what a program has in hand before a call, ``run`` one
call (of the library where ``own`` is true, else in plain torch operations), ``work`` what it cannot do without and
``exact`` its result in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

SPARE = 10            # a pool holds this share (percent) more pages than its sequences use


# ------------------------------------------------------------------ cases

def _rows(op, batch, q_len, kv_len, kv_heads, dim, page, e4m3, ragged):
    """q_len: rows written or read, the last ones of a sequence of kv_len tokens."""
    return {"op": op, "batch": batch, "q_len": q_len, "kv_len": kv_len, "kv_heads": kv_heads, "dim": dim, "page": page, "e4m3": e4m3,
            "ragged": ragged}


def _attention(batch, heads, kv_heads, dim, q_len, kv_len, page, e4m3, window, sinks, ragged):
    """window: keys to the left of a token that it sees, 0 for all of them."""
    return {**_rows("attention", batch, q_len, kv_len, kv_heads, dim, page, e4m3, ragged), "heads": heads, "window": window,
            "sinks": sinks}


def _lora(m, k, n, rank, adapters, mixed, ragged, act="none", f32=False):
    """mixed: rows of different adapters one after the other (single tokens of many requests), else each adapter's rows
    together (prompts); ragged: adapters of smaller ranks among them."""
    return {"op": "lora", "m": m, "k": k, "n": n, "rank": rank, "adapters": adapters, "mixed": mixed, "ragged": ragged, "act": act,
            "f32": f32}


def listed():
    return [
        # one new token for each of a serving batch's sequences
        {"name": "append_token_24x500", **_rows("append", 24, 1, 500, 8, 128, 16, False, True)},
        # two prompts put into an 8-bit cache
        {"name": "append_prompt_2x3001_e4m3", **_rows("append", 2, 3001, 3001, 8, 128, 64, True, True)},
        # a few short sequences read back, as when they move to another place
        {"name": "read_5x100", **_rows("read", 5, 100, 100, 12, 64, 16, False, True)},
        # a long prompt's 8-bit rows read back for attention over contiguous keys
        {"name": "read_1x8191_e4m3", **_rows("read", 1, 8191, 8191, 8, 128, 64, True, False)},
        # one new token of three short sequences: all launch and latency
        {"name": "attn_token_3x300", **_attention(3, 12, 12, 64, 1, 300, 16, False, 0, 0, True)},
        # one new token for each of a serving batch's sequences
        {"name": "attn_token_24x4096", **_attention(24, 32, 8, 128, 1, 4096, 16, False, 0, 0, True)},
        # one new token of one very long sequence in an 8-bit cache
        {"name": "attn_token_1x100001_e4m3", **_attention(1, 32, 8, 128, 1, 100001, 64, True, 0, 0, False)},
        # five drafted tokens for each of sixteen sequences, a window and sinks
        {"name": "attn_drafts_16x5_w1024", **_attention(16, 32, 8, 128, 5, 8191, 32, False, 1024, 4, True)},
        # one request's token through an encoder-wide layer
        {"name": "lora_1x768x768_r8", **_lora(1, 768, 768, 8, 4, True, False)},
        # a token of each of 64 requests, every few of another tenant
        {"name": "lora_64x4096x4096_r16", **_lora(64, 4096, 4096, 16, 24, True, True)},
        # class scores in fp32 for a batch that fills no tile
        {"name": "lora_100x2048x1000_r32", **_lora(100, 2048, 1000, 32, 7, False, True, f32=True)},
        # prompts of five tenants through a hidden layer
        {"name": "lora_8192x4096x4096_r64", **_lora(8192, 4096, 4096, 64, 5, False, True, act="gelu")},
    ]


def _log(rng, lo, hi):
    """An integer of [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    while True:
        kind = rng.randrange(5)
        if kind < 2:
            case = _lora(_log(rng, 1, 8192), 8 * _log(rng, 8, 1024), _log(rng, 64, 8192), rng.choice((8, 16, 24, 32, 64, 128)),
                         _log(rng, 1, 32), rng.random() < 0.5, rng.random() < 0.5, rng.choice(("none", "relu", "gelu")), rng.random() < 0.3)
            if case["m"] * case["k"] * case["adapters"] * case["rank"] > 8192 * 4096 * 1024:      # the plain form takes every adapter
                continue
        else:
            dim, page, e4m3 = rng.choice((64, 128)), rng.choice((16, 32, 64, 128, 256)), rng.random() < 0.5
            kv_heads, ragged = rng.choice((1, 2, 3, 4, 8, 12)), rng.random() < 0.7
            batch, kv = _log(rng, 1, 64), _log(rng, 1, 100001)
            if kind < 4:
                q = rng.choice((1, 1, rng.randint(2, 8)))
                window = rng.choice((0, _log(rng, 16, 2048)))
                case = _attention(batch, kv_heads * rng.choice((1, 2, 3, 4, 8)), kv_heads, dim, min(q, kv), kv, page, e4m3, window,
                                  rng.choice((0, rng.randint(1, 64))) if window else 0, ragged)
            else:
                case = _rows(rng.choice(("append", "read")), batch, rng.choice((1, _log(rng, 1, kv), kv)), kv, kv_heads, dim, page, e4m3,
                             ragged)
            if batch * kv * kv_heads * dim > 1.1e8:
                continue
        w = work(case)
        if w["flops"] <= 2 * 8192 * 128 * 8192 and w["bytes"] <= 4.2e8:       # no more than the largest listed
            return case


def _lens(c):
    """(new tokens, tokens in all) of each sequence: ragged ones get shorter down to half."""
    out = []
    for b in range(c["batch"]):
        cut = (b * 2 + 1) * c["kv_len"] // (4 * c["batch"]) if c["ragged"] else 0
        kv = max(1, c["kv_len"] - cut)
        out.append((min(c["q_len"], kv), kv))
    return out


def _ranks(c):
    return [max(1, c["rank"] - (a % 3) * c["rank"] // 4) if c["ragged"] else c["rank"] for a in range(c["adapters"])]


def _adapters(c):
    """The adapter of each row; some rows have none."""
    rows = range(c["m"])
    if c["mixed"]:
        return [(7 * r + r // 5) % c["adapters"] if r % 16 != 11 else -1 for r in rows]
    return [r * c["adapters"] // c["m"] if r % 1024 != 1000 else -1 for r in rows]


def work(case):
    c = case
    if c["op"] == "lora":
        m, k, n = c["m"], c["k"], c["n"]
        ranks, ids = _ranks(c), [a for a in _adapters(c) if a >= 0]
        return {"bytes": 2.0 * m * k + 2.0 * m * n * (4 if c["f32"] else 2) + sum(2.0 * ranks[a] * (k + n) for a in set(ids)),
                "flops": sum(2.0 * ranks[a] * (k + n) for a in ids)}
    d, hk = c["dim"], c["kv_heads"]
    held = d + 1 if c["e4m3"] else 2 * d                 # bytes of a token's head in the cache
    lens = _lens(c)
    if c["op"] != "attention":
        rows = sum(q for q, _ in lens)
        return {"bytes": 2.0 * rows * hk * (2 * d + held), "flops": float(rows * hk * d)}
    pairs = keys = rows = 0
    for qn, kn in lens:
        p0 = kn - qn                                     # the first new token's position
        for p in range(p0, kn):
            lo = max(0, p - c["window"]) if c["window"] else 0
            pairs += p + 1 - lo + min(c["sinks"], lo)
        start = max(0, p0 - c["window"]) if c["window"] else 0
        keys += kn - start + min(c["sinks"], start)
        rows += qn
    return {"bytes": 4.0 * d * c["heads"] * rows + 2.0 * keys * hk * held, "flops": 4.0 * d * c["heads"] * pairs}


# ------------------------------------------------------------------ a program's state

def prepare(case, seed):
    c = case
    dev = torch.device("cuda", 0)
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed) * 1000003 + 29)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device=dev, dtype=torch.float32).mul_(std).to(torch.bfloat16)

    # scratch that a serving program keeps for its calls
    s = {"case": c, "work": torch.empty(32 << 20, device=dev, dtype=torch.uint8)}
    if c["op"] == "lora":
        m, k, n, rank = c["m"], c["k"], c["n"], c["rank"]
        dtype = torch.float32 if c["f32"] else torch.bfloat16
        s["x"], s["base"] = normal(m, k), normal(m, n).to(dtype)
        s["a"], s["b"] = normal(c["adapters"], rank, k, std=k ** -0.5), normal(c["adapters"], n, rank, std=rank ** -0.5)
        s["adapter"] = torch.tensor(_adapters(c), dtype=torch.int32).to(dev)
        s["ranks"] = torch.tensor(_ranks(c), dtype=torch.int32).to(dev)
        s["scales"] = torch.rand(c["adapters"], generator=g, device=dev).add_(0.5)
        s["out"] = torch.zeros(m, n, device=dev, dtype=dtype)
        return s
    b, q, hk, d, page = (c[x] for x in ("batch", "q_len", "kv_heads", "dim", "page"))
    lens = _lens(c)
    columns = (c["kv_len"] + page - 1) // page
    used = [(kn + page - 1) // page for _, kn in lens]
    pages = sum(used) + max(1, sum(used) * SPARE // 100)
    order = torch.randperm(pages, generator=g, device=dev, dtype=torch.int32)
    first = torch.tensor([sum(used[:i]) for i in range(b)]).to(dev).view(b, 1)
    col = torch.arange(columns, device=dev).view(1, columns)
    there = col < torch.tensor(used).to(dev).view(b, 1)
    s["table"] = order[(first + col).clamp(max=pages - 1)].masked_fill(~there, -1)
    lens = torch.tensor(lens, dtype=torch.int32)
    s["q_lens"], s["kv_lens"] = lens[:, 0].to(dev), lens[:, 1].to(dev)
    if c["e4m3"]:
        # what rounded normal values look like: the top of e4m3's range is used, and scales vary by token
        s["k"], s["v"] = (normal(pages, page, hk, d, std=110.0).float().clamp_(-448, 448).to(torch.float8_e4m3fn) for _ in "kv")
        s["exps"] = torch.randint(118, 122, (pages, 2, hk, page), generator=g, device=dev, dtype=torch.int32).to(torch.uint8)
    else:
        s["k"], s["v"], s["exps"] = normal(pages, page, hk, d), normal(pages, page, hk, d), None
    if c["op"] == "append":
        spread = torch.randint(-3, 3, (b, q, hk, 1), generator=g, device=dev).float().exp2_()
        s["new_k"], s["new_v"] = ((normal(b, q, hk, d).float() * spread).to(torch.bfloat16) for _ in "kv")
    elif c["op"] == "read":
        # rows behind a sequence's last are not written
        s["out_k"], s["out_v"] = (torch.zeros(b, q, hk, d, device=dev, dtype=torch.bfloat16) for _ in "kv")
    else:
        s["q"] = normal(b, q, c["heads"], d)
        s["out"] = torch.zeros(b, q, c["heads"], d, device=dev, dtype=torch.bfloat16)
    return s


# ------------------------------------------------------------------ one call

def run(state):
    op = state["case"]["op"]
    if own:
        return _own(state)
    return {"append": _plain_append, "read": _plain_read, "attention": _plain_attention, "lora": _plain_lora}[op](state)


def _own(s):
    import paper_2306_03622_amd as tp
    c = s["case"]
    if c["op"] == "lora":
        tp.tps_lora(s["x"], s["a"], s["b"], s["adapter"], s["out"], base=s["base"], ranks=s["ranks"] if c["ragged"] else None,
                    scales=s["scales"], act=c["act"], work=s["work"])
        return s["out"]
    cache = s.get("cache")
    if cache is None:
        cache = s["cache"] = tp.PagedCache(s["k"], s["v"], s["exps"])
    q_lens = s["q_lens"] if c["ragged"] else None
    if c["op"] == "append":
        tp.tps_cache_append(cache, s["table"], s["kv_lens"], s["new_k"], s["new_v"], q_lens=q_lens)
        return _pool(s)
    if c["op"] == "read":
        tp.tps_cache_read(cache, s["table"], s["kv_lens"], s["out_k"], s["out_v"], q_lens=q_lens)
        return {"k": s["out_k"], "v": s["out_v"]}
    tp.tps_cache_attention(cache, s["table"], s["kv_lens"], s["q"], s["out"], q_lens=q_lens, kv_len=c["kv_len"],
                           window=c["window"] if c["window"] else -1, sinks=c["sinks"], work=s["work"])
    return s["out"]


def _pool(s):
    return {"k": s["k"], "v": s["v"], "exps": s["exps"]} if s["case"]["e4m3"] else {"k": s["k"], "v": s["v"]}


def _power(byte):
    """2^(byte - 127) exactly: the number whose exponent bits those are."""
    return (byte.to(torch.int32) << 23).view(torch.float32)


def _places(s):
    """(sequence, row, page, token in the page) of every row that a sequence really has."""
    c = s["case"]
    i = torch.arange(c["q_len"], device=s["table"].device).view(1, -1)
    here = i < s["q_lens"].view(-1, 1)
    seq, row = here.nonzero(as_tuple=True)
    pos = (s["kv_lens"] - s["q_lens"]).long()[seq] + row
    return seq, row, s["table"].long()[seq, pos // c["page"]], pos % c["page"]


def _plain_append(s):
    seq, row, page, at = _places(s)
    if not s["case"]["e4m3"]:
        s["k"][page, at] = s["new_k"][seq, row]
        s["v"][page, at] = s["new_v"][seq, row]
        return _pool(s)
    x = torch.stack((s["new_k"][seq, row], s["new_v"][seq, row])).float()                  # [2, rows, heads, dim]
    part, power = torch.frexp(x.abs().amax(-1))                                             # part in [0.5, 1), 448 = 0.875 2^9
    e = (power - 9 + (part > 0.875).int()).masked_fill(part == 0, -126).clamp(-126, 127)
    codes = (x * _power(127 - e)[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
    s["k"].view(torch.uint8)[page, at] = codes[0]
    s["v"].view(torch.uint8)[page, at] = codes[1]
    s["exps"].transpose(2, 3).transpose(1, 2)[page, at] = (e + 127).to(torch.uint8).transpose(0, 1).contiguous()
    return _pool(s)


def _plain_read(s):
    c = s["case"]
    seq, row, page, at = _places(s)
    k, v = s["k"][page, at].float(), s["v"][page, at].float()
    if c["e4m3"]:
        scale = _power(s["exps"].transpose(2, 3).transpose(1, 2)[page, at])
        k, v = k * scale[:, 0, :, None], v * scale[:, 1, :, None]
    s["out_k"][seq, row], s["out_v"][seq, row] = k.to(torch.bfloat16), v.to(torch.bfloat16)
    return {"k": s["out_k"], "v": s["out_v"]}


def _plain_attention(s):
    c = s["case"]
    b, h, hk, d, nq, page = (c[x] for x in ("batch", "heads", "kv_heads", "dim", "q_len", "page"))
    dev, nk = s["q"].device, s["table"].shape[1] * c["page"]
    i, j = torch.arange(nq, device=dev).view(1, nq, 1), torch.arange(nk, device=dev).view(1, 1, nk)
    ql, kl = s["q_lens"].long().view(b, 1, 1), s["kv_lens"].long().view(b, 1, 1)
    back = kl - ql + i - j                                                     # how far a key is to the left
    see = (back >= 0) & (j < kl)
    if c["window"]:
        see = see & ((back <= c["window"]) | (j < c["sinks"]))
    at = s["table"].long().clamp(min=0)
    k, v = s["k"][at].float(), s["v"][at].float()                              # [b, columns, page, heads, dim]
    if c["e4m3"]:
        scale = _power(s["exps"][at]).transpose(3, 4)           # [b, columns, 2, page, heads]
        k, v = k * scale[:, :, 0, :, :, None], v * scale[:, :, 1, :, :, None]
    there = (j < kl).view(b, nk, 1, 1)
    k = k.view(b, nk, hk, d).masked_fill(~there, 0).permute(0, 2, 3, 1).contiguous()       # [b, hk, d, nk]
    v = v.view(b, nk, hk, d).masked_fill(~there, 0).permute(0, 2, 1, 3).contiguous()       # [b, hk, nk, d]
    q = s["q"].float().view(b, nq, hk, h // hk, d).permute(0, 2, 3, 1, 4).reshape(b, hk, -1, d).contiguous()
    p = torch.matmul(q, k).view(b, hk, h // hk, nq, nk) * d ** -0.5
    p = p.masked_fill_(~see.view(b, 1, 1, nq, nk), -math.inf)
    top = p.amax(-1, keepdim=True)
    p = p.sub_(top.masked_fill(top == -math.inf, 0)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(b, hk, -1, nk), v).view(b, hk, h // hk, nq, d) / total.masked_fill(total == 0, 1)
    o = o.permute(0, 3, 1, 2, 4).reshape(b, nq, h, d)
    row = torch.arange(nq, device=dev).view(1, nq) < s["q_lens"].view(b, 1)
    return torch.where(row.view(b, nq, 1, 1), o, 0.0).to(torch.bfloat16)


def _plain_lora(s):
    c = s["case"]
    m, rank, slots = c["m"], c["rank"], c["adapters"]
    dev = s["x"].device
    # every row through every adapter, of which its own is kept
    t = (s["x"].float() @ s["a"].float().view(slots * rank, -1).t()).view(m, slots, rank)
    mine = s["adapter"].view(m, 1, 1) == torch.arange(slots, device=dev).view(1, slots, 1)
    held = torch.arange(rank, device=dev).view(1, 1, rank) < s["ranks"].view(1, slots, 1)
    t = torch.where(mine & held, t * s["scales"].view(1, slots, 1), 0.0).view(m, slots * rank)
    y = s["base"].float() + t @ s["b"].float().permute(0, 2, 1).reshape(slots * rank, -1)
    if c["act"] == "relu":
        y = y.clamp(min=0)
    elif c["act"] == "gelu":
        y = 0.5 * y * (1 + torch.erf(y * 0.5 ** 0.5))
    return y.to(s["out"].dtype)


# ------------------------------------------------------------------ the same in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "read": _exact_read, "attention": _exact_attention, "lora": _exact_lora}[case["op"]](case, s)


def _power64(e):
    """2^e in 64 bits, without a power function's rounding."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _to_e4m3(x):
    """[.., dim] in 64 bits: (what each value's code stands for, exponent): three bits behind the first one, steps of 2^-9 at least."""
    top = x.abs().amax(-1, keepdim=True)
    e = torch.full_like(top, -126.0)
    for power in range(-126, 128):                       # the last exponent that is too small, plus one
        e = torch.where(top > 448.0 * 2.0 ** (power - 1), float(power), e)
    y = x * _power64(-e)
    step = _power64(torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4)
    return torch.round(y / step) * step, (e[..., 0] + 127).to(torch.uint8)


def _exact_append(c, s):
    k, v = s["k"].double(), s["v"].double()
    exps = s["exps"]
    nk, nv = s["new_k"].double(), s["new_v"].double()
    if c["e4m3"]:
        (nk, ke), (nv, ve) = _to_e4m3(nk), _to_e4m3(nv)
    table = s["table"].long()
    for b, (qn, kn) in enumerate(_lens(c)):
        pos = torch.arange(kn - qn, kn, device=k.device)
        page, at = table[b, torch.div(pos, c["page"], rounding_mode="floor")], pos % c["page"]
        k[page, at], v[page, at] = nk[b, :qn], nv[b, :qn]
        if c["e4m3"]:
            for h in range(c["kv_heads"]):
                exps[page, 0, h, at], exps[page, 1, h, at] = ke[b, :qn, h], ve[b, :qn, h]
    return {"k": k, "v": v, "exps": exps} if c["e4m3"] else {"k": k, "v": v}


def _sequence(c, s, b, kn):
    """Keys and values [kn, heads, dim] of a sequence in 64 bits."""
    page = s["table"][b].long()[: (kn + c["page"] - 1) // c["page"]]
    out = []
    for n, pool in enumerate((s["k"], s["v"])):
        x = pool[page].double()
        if c["e4m3"]:
            x = x * _power64(s["exps"][page, n].long() - 127).permute(0, 2, 1)[..., None]
        out.append(x.reshape(-1, c["kv_heads"], c["dim"])[:kn])
    return out


def _exact_read(c, s):
    k, v = (torch.zeros(t.shape, dtype=torch.float64, device=t.device) for t in (s["out_k"], s["out_v"]))
    for b, (qn, kn) in enumerate(_lens(c)):
        sk, sv = _sequence(c, s, b, kn)
        k[b, :qn], v[b, :qn] = sk[kn - qn:], sv[kn - qn:]
    return {"k": k, "v": v}


def _exact_attention(c, s):
    """One sequence and one head at a time, softmax in 64 bits over the keys each query sees."""
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=s["out"].device)
    share = c["heads"] // c["kv_heads"]
    for b, (qn, kn) in enumerate(_lens(c)):
        k, v = _sequence(c, s, b, kn)
        pos, key = torch.arange(kn - qn, kn, device=out.device)[:, None], torch.arange(kn, device=out.device)[None]
        hidden = key > pos
        if c["window"]:
            hidden = hidden | ((pos - key > c["window"]) & (key >= c["sinks"]))
        for h in range(c["heads"]):
            score = s["q"][b, :qn, h].double() @ k[:, h // share].t().contiguous() / math.sqrt(c["dim"])
            out[b, :qn, h] = torch.softmax(score.masked_fill(hidden, -math.inf), -1) @ v[:, h // share].contiguous()
    return out


def _exact_lora(c, s):
    """One adapter's rows at a time."""
    y = s["base"].double()
    ids, ranks = torch.tensor(_adapters(c)), _ranks(c)
    for a in range(c["adapters"]):
        rows = (ids == a).nonzero().view(-1).to(y.device)
        if not len(rows):
            continue
        down, up = s["a"][a, :ranks[a]].double(), s["b"][a, :, :ranks[a]].double()
        t = s["x"][rows].double() @ down.t().contiguous()
        y[rows] += float(s["scales"][a]) * (t @ up.t().contiguous())
    if c["act"] == "relu":
        y = torch.relu(y)
    elif c["act"] == "gelu":
        y = y * torch.special.ndtr(y)
    return y
