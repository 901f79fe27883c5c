"""The operators this repository offers beside its models: what is timed of them, and their plain forms.

* ``linear_w4``: a linear layer with 4-bit weights and a bf16 scale per group of inputs,
  ``y = act(x W^T + bias)``, from one row (a matrix-vector product) to thousands.
* ``attention``: softmax attention with a sliding window, first keys that stay visible (sinks),
  a causal order, lengths per sequence, shared key/value heads and chunks of new tokens.

Functions: ``listed`` and ``draw`` give cases, ``prepare`` what a program has in hand before a
call, ``run`` one call (of the library where ``own`` is true, else in plain torch operations),
``work`` what it cannot do without and ``exact`` its result in 64 bits.

The 4-bit format (``tp.W4Weight``): rows padded to whole 16, columns to whole 128; the block of
rows 16 n.. and columns 128 k.. is 1024 bytes, blocks row by row; inside it the 32-bit word
4 (16 q + r) + j holds row r, columns 32 j + 8 q + 0..7, column i in the 4 bits at 4 (i / 2) + 16 (i % 2). A code
is the value plus 8. Scales are ordered [row / 16][group][row % 16]; padding has code 8 and scale 0.
"""
from __future__ import annotations

import math

import torch

own = False

HEADROOM = 5          # a key/value cache holds this share (percent) more tokens than its longest sequence


# ------------------------------------------------------------------ cases

def _linear(m, n, k, group, act="none", f32=False):
    return {"op": "linear_w4", "m": m, "n": n, "k": k, "group": group, "act": act, "f32": f32}


def _attention(batch, heads, kv_heads, dim, q_len, kv_len, causal, window, sinks, ragged, fused=False):
    """window: keys to the left (and, when not causal, to the right) that a query sees, 0 for all of them; fused:
    q, k and v are slices of one projection's output, as in an encoder layer, else a cache is read."""
    return {"op": "attention", "batch": batch, "heads": heads, "kv_heads": kv_heads, "dim": dim, "q_len": q_len,
            "kv_len": kv_len, "causal": causal, "window": window, "sinks": sinks, "ragged": ragged, "fused": fused}


def listed():
    return [
        # one request of one row through an encoder-wide layer: all launch and latency
        {"name": "w4_1x768x768_g32", **_linear(1, 768, 768, 32)},
        # the benchmark's layer and batch, quantised: a hidden layer of the heavy model
        {"name": "w4_8x4096x4096_g128", **_linear(8, 4096, 4096, 128, act="gelu")},
        # one row through a layer wider than the caches: the weights come from memory
        {"name": "w4_1x32768x8192_g128", **_linear(1, 32768, 8192, 128)},
        # class scores of a batch that fills no tile, in fp32
        {"name": "w4_100x1000x2048_g64", **_linear(100, 1000, 2048, 64, f32=True)},
        # an encoder's fused projection at the benchmark's larger batch (8 sequences of 128)
        {"name": "w4_1024x2304x768_g64", **_linear(1024, 2304, 768, 64)},
        # offline scoring: a hidden layer over a large batch
        {"name": "w4_8192x4096x4096_g128", **_linear(8192, 4096, 4096, 128, act="gelu")},
        # an encoder layer on a few short padded sequences
        {"name": "attn_encoder_5x96", **_attention(5, 12, 12, 64, 96, 96, False, 0, 0, True, fused=True)},
        # an encoder layer on long padded documents, each token seeing its neighbours and the first one
        {"name": "attn_encoder_8x2048_w128", **_attention(8, 12, 12, 64, 2048, 2048, False, 128, 1, True, fused=True)},
        # one new token for each of sixteen running sequences, a window and sinks over their caches
        {"name": "attn_token_16x4096_w1024", **_attention(16, 32, 8, 128, 1, 4096, True, 1024, 4, True)},
        # one new token of one very long sequence: its whole cache is read
        {"name": "attn_token_1x100001", **_attention(1, 32, 8, 128, 1, 100001, True, 0, 0, False)},
        # a chunk of a prompt behind what is cached already
        {"name": "attn_chunk_2x500_6000_w1024", **_attention(2, 32, 8, 128, 500, 6000, True, 1024, 4, True)},
        # a whole prompt at once
        {"name": "attn_prompt_1x8191", **_attention(1, 32, 8, 128, 8191, 8191, True, 0, 0, False)},
    ]


def _log(rng, lo, hi):
    """An integer of [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    while True:
        if rng.random() < 0.5:
            group = rng.choice((32, 64, 128))
            case = _linear(_log(rng, 1, 8192), _log(rng, 64, 32768), group * _log(rng, 1, 8192 // group), group,
                           rng.choice(("none", "relu", "gelu")), rng.random() < 0.3)
        else:
            dim = rng.choice((64, 128))
            window = rng.choice((0, _log(rng, 16, 2048)))
            sinks = rng.choice((0, rng.randint(1, 64))) if window else 0
            kind = rng.randrange(3)
            if kind == 0:                       # an encoder layer
                heads, s = rng.randint(1, 16), _log(rng, 1, 4096)
                case = _attention(_log(rng, 1, 32), heads, heads, dim, s, s, False, window, sinks, rng.random() < 0.7, True)
            else:
                kv_heads, share = rng.choice((1, 2, 4, 8)), rng.choice((1, 2, 3, 4, 8))
                kv = _log(rng, 1, 100001)
                q = rng.choice((1, rng.randint(1, 8))) if kind == 1 else _log(rng, 2, 8192)
                case = _attention(_log(rng, 1, 32), kv_heads * share, kv_heads, dim, min(q, kv), kv, True, window, sinks,
                                  rng.random() < 0.7)
            c = case
            # the plain form writes every score down
            if c["batch"] * c["heads"] * c["q_len"] * c["kv_len"] > 32 * 8191 * 8191:
                continue
            if c["batch"] * c["kv_heads"] * c["kv_len"] * dim > 32 * 4096 * 8 * 128:
                continue
        w = work(case)
        if w["flops"] <= 2 * 8192 * 4096 * 4096 and w["bytes"] <= 4.5e8:      # no more than the largest listed
            return case


def _lens(c):
    """(new tokens, tokens in all) of each sequence: ragged ones get shorter down to half."""
    out = []
    for b in range(c["batch"]):
        cut = (b * 2 + 1) * c["kv_len"] // (4 * c["batch"]) if c["ragged"] else 0
        kv = max(1, c["kv_len"] - cut)
        out.append((min(c["q_len"], kv), kv))
    return out


def _blocks(c):
    return (c["n"] + 15) // 16, (c["k"] + 127) // 128


def work(case):
    c = case
    if c["op"] == "linear_w4":
        m, n, k = c["m"], c["n"], c["k"]
        return {"bytes": n * k / 2 + 2 * n * (k // c["group"]) + 2 * m * k + 2 * n + m * n * (4 if c["f32"] else 2),
                "flops": 2.0 * m * n * k}
    pairs = keys = rows = 0
    for qn, kn in _lens(c):
        p0 = kn - qn                            # the first new token's position
        pos = torch.arange(p0, kn, dtype=torch.int64)
        hi = pos if c["causal"] or not c["window"] else (pos + c["window"]).clamp(max=kn - 1)
        if not c["causal"] and not c["window"]:
            hi = torch.full_like(pos, kn - 1)
        lo = (pos - c["window"]).clamp(min=0) if c["window"] else torch.zeros_like(pos)
        first = lo.clamp(max=c["sinks"])        # sinks in front of the window
        pairs += int((hi - lo + 1 + first).sum())
        start = max(0, p0 - c["window"]) if c["window"] else 0
        keys += kn - start + min(c["sinks"], start)
        rows += qn
    d, h = c["dim"], c["heads"]
    return {"bytes": 2.0 * d * (2 * h * rows + 2 * c["kv_heads"] * keys), "flops": 4.0 * d * h * pairs}


# ------------------------------------------------------------------ a program's state

def prepare(case, seed):
    dev = torch.device("cuda", 0)
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed) * 1000003 + 17)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device=dev, dtype=torch.float32).mul_(std).to(torch.bfloat16)

    s = {"case": case}
    if case["op"] == "linear_w4":
        m, n, k, group = case["m"], case["n"], case["k"], case["group"]
        nb, kb = _blocks(case)
        codes = torch.randint(0, 16, (nb, kb, 4, 16, 4, 8), generator=g, device=dev, dtype=torch.int32)
        # middle values are the frequent ones, as in weights rounded to 16 steps
        codes = (codes + torch.randint(0, 16, codes.shape, generator=g, device=dev, dtype=torch.int32) + 1) // 2
        codes.clamp_(max=15)
        row = torch.arange(nb * 16, device=dev).view(nb, 1, 1, 16, 1, 1)
        col = (torch.arange(kb, device=dev).view(kb, 1, 1, 1, 1) * 128 + torch.arange(4, device=dev).view(4, 1, 1, 1) * 8 +
               torch.arange(4, device=dev).view(4, 1) * 32 + torch.arange(8, device=dev))
        codes.masked_fill_((row >= n) | (col >= k), 8)
        words = torch.zeros(codes.shape[:-1], device=dev, dtype=torch.int32)
        for i in range(8):
            words |= codes[..., i] << (4 * (i // 2) + 16 * (i % 2))
        groups = kb * 128 // group
        scales = torch.rand(nb, groups, 16, generator=g, device=dev).add_(0.5).mul_(k ** -0.5 / 4)
        scales.masked_fill_((torch.arange(nb * 16, device=dev).view(nb, 1, 16) >= n) |
                            (torch.arange(groups, device=dev).view(groups, 1) >= k // group), 0.0)
        s["codes"] = words.view(torch.uint8).view(nb, kb, 1024)
        s["scales"] = scales.to(torch.bfloat16)
        s["x"] = normal(m, k)
        s["bias"] = normal(n, std=0.02)
        s["out"] = torch.zeros(m, n, device=dev, dtype=torch.float32 if case["f32"] else torch.bfloat16)
    else:
        b, h, hk, d, q, kv = (case[x] for x in ("batch", "heads", "kv_heads", "dim", "q_len", "kv_len"))
        if case["fused"]:
            qkv = normal(b, q, 3 * h, d)
            s["q"], s["k"], s["v"] = qkv[:, :, :h], qkv[:, :, h:2 * h], qkv[:, :, 2 * h:]
        else:
            room = kv + kv * HEADROOM // 100
            s["q"] = normal(b, q, h, d)
            s["k"], s["v"] = normal(b, room, hk, d)[:, :kv], normal(b, room, hk, d)[:, :kv]
        lens = torch.tensor(_lens(case), dtype=torch.int32)
        s["q_lens"], s["kv_lens"] = lens[:, 0].to(dev), lens[:, 1].to(dev)
        # rows behind a sequence's last are not written
        s["out"] = torch.zeros(b, q, h, d, device=dev, dtype=torch.bfloat16)
    # scratch that a serving program keeps for its calls
    s["work"] = torch.empty(32 << 20, device=dev, dtype=torch.uint8)
    return s


# ------------------------------------------------------------------ one call

def run(state):
    if state["case"]["op"] == "linear_w4":
        return _own_linear(state) if own else _plain_linear(state)
    return _own_attention(state) if own else _plain_attention(state)


def _own_linear(s):
    import paper_2306_03622_amd as tp
    c = s["case"]
    w = s.get("w")
    if w is None:
        w = s["w"] = tp.W4Weight(s["codes"], s["scales"], c["n"], c["k"], c["group"])
    tp.tpo_linear_w4(s["x"], w, s["out"], bias=s["bias"], act=c["act"], work=s["work"])
    return s["out"]


def _own_attention(s):
    import paper_2306_03622_amd as tp
    c = s["case"]
    window = (c["window"], 0 if c["causal"] else c["window"]) if c["window"] else (-1, -1)
    tp.tpo_attention(s["q"], s["k"], s["v"], s["out"], q_lens=s["q_lens"] if c["ragged"] else None,
                     kv_lens=s["kv_lens"] if c["ragged"] else None, causal=c["causal"], window=window, sinks=c["sinks"],
                     work=s["work"])
    return s["out"]


def _plain_linear(s):
    c = s["case"]
    n, k, group = c["n"], c["k"], c["group"]
    nb, kb = _blocks(c)
    words = s["codes"].view(torch.int32).view(nb, kb, 4, 16, 4, 1)            # [.., q, r, j]
    shift = torch.tensor([0, 16, 4, 20, 8, 24, 12, 28], dtype=torch.int32, device=words.device)
    codes = (words >> shift) & 15
    codes = codes.permute(0, 3, 1, 4, 2, 5).reshape(nb * 16, kb * 128)        # [row][kb, j, q, i]
    scale = s["scales"].float().transpose(1, 2).reshape(nb * 16, -1)
    w = ((codes - 8).float().view(nb * 16, -1, group) * scale[:, :, None]).view(nb * 16, kb * 128)[:n, :k]
    y = s["x"].float() @ w.t() + s["bias"].float()
    if c["act"] == "relu":
        y = y.clamp(min=0)
    elif c["act"] == "gelu":
        y = 0.5 * y * (1 + torch.erf(y * 0.5 ** 0.5))
    return y.to(s["out"].dtype)


def _plain_attention(s):
    c = s["case"]
    b, h, hk, d, nq, nk = (c[x] for x in ("batch", "heads", "kv_heads", "dim", "q_len", "kv_len"))
    dev = s["q"].device
    ql, kl = s["q_lens"].long().view(b, 1, 1), s["kv_lens"].long().view(b, 1, 1)
    i, j = torch.arange(nq, device=dev).view(1, nq, 1), torch.arange(nk, device=dev).view(1, 1, nk)
    off = j - (kl - ql + i)                                                   # how far a key is to the right
    see = (j < kl).expand(b, nq, nk)
    if c["causal"]:
        see = see & (off <= 0)
    if c["window"]:
        see = see & ((off.abs() <= c["window"]) | (j < c["sinks"]))
    there = (torch.arange(nk, device=dev).view(1, nk) < kl.view(b, 1)).view(b, nk, 1, 1)
    k = s["k"].float().masked_fill(~there, 0).permute(0, 2, 3, 1).contiguous()            # [b, hk, d, nk]
    v = s["v"].float().masked_fill(~there, 0).permute(0, 2, 1, 3).contiguous()            # [b, hk, nk, d]
    q = s["q"].float().view(b, nq, hk, h // hk, d).permute(0, 2, 3, 1, 4).reshape(b, hk, -1, d).contiguous()
    p = torch.matmul(q, k).view(b, hk, h // hk, nq, nk) * d ** -0.5
    p = p.masked_fill_(~see.view(b, 1, 1, nq, nk), -math.inf)
    top = p.amax(-1, keepdim=True)
    top = top.masked_fill(top == -math.inf, 0)
    p = p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(b, hk, -1, nk), v).view(b, hk, h // hk, nq, d) / total.masked_fill(total == 0, 1)
    o = o.permute(0, 3, 1, 2, 4).reshape(b, nq, h, d)
    row = torch.arange(nq, device=dev).view(1, nq) < s["q_lens"].view(b, 1)
    return torch.where(row.view(b, nq, 1, 1), o, 0.0).to(torch.bfloat16)


# ------------------------------------------------------------------ the same in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return _exact_linear(case, s) if case["op"] == "linear_w4" else _exact_attention(case, s)


def _exact_linear(c, s):
    """Every weight is looked up at its own place: byte and half byte from (row, column)."""
    n, k = c["n"], c["k"]
    dev = s["x"].device
    flat, groups = s["codes"].reshape(-1), s["scales"].shape[1]
    kb = (k + 127) // 128
    col = torch.arange(k, device=dev)
    i = col % 8
    bit = 4 * (i // 2) + 16 * (i % 2)
    out = torch.empty(c["m"], n, dtype=torch.float64, device=dev)
    x = s["x"].double()
    for r0 in range(0, n, 2048):
        row = torch.arange(r0, min(n, r0 + 2048), device=dev)[:, None]
        word = ((row // 16) * kb + col // 128) * 256 + 4 * (16 * ((col // 8) % 4) + row % 16) + (col // 32) % 4
        byte = flat[word * 4 + bit // 8].long()
        code = torch.where(bit % 8 == 4, byte // 16, byte % 16)
        scale = s["scales"].reshape(-1).double()[((row // 16) * groups + col // c["group"]) * 16 + row % 16]
        out[:, r0:r0 + row.shape[0]] = x @ ((code.double() - 8) * scale).t().contiguous()
    out += s["bias"].double()
    if c["act"] == "relu":
        out = torch.relu(out)
    elif c["act"] == "gelu":
        out = out * torch.special.ndtr(out)
    return out


def _exact_attention(c, s):
    """One sequence, one head and a block of queries at a time, softmax in 64 bits over the keys each query sees."""
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=s["out"].device)
    share = c["heads"] // c["kv_heads"]
    for b, (qn, kn) in enumerate(_lens(c)):
        key = torch.arange(kn, device=out.device)[None]
        for r0 in range(0, qn, 2048):
            r1 = min(qn, r0 + 2048)
            pos = torch.arange(r0, r1, device=out.device)[:, None] + (kn - qn)
            hidden = torch.zeros(r1 - r0, kn, dtype=torch.bool, device=out.device)
            if c["window"]:
                hidden = ((pos - key > c["window"]) | (key - pos > c["window"])) & (key >= c["sinks"])
            if c["causal"]:
                hidden = hidden | (key > pos)
            for h in range(c["heads"]):
                k, v = s["k"][b, :kn, h // share].double(), s["v"][b, :kn, h // share].double()
                score = s["q"][b, r0:r1, h].double() @ k.t().contiguous() / math.sqrt(c["dim"])
                out[b, r0:r1, h] = torch.softmax(score.masked_fill(hidden, -math.inf), -1) @ v
    return out
