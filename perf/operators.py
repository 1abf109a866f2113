"""The paged key-value cache and the attention over it, as they are timed: the cache written and read back, one new token of every
sequence attending, the rows of prompts attending.

Each case is one pass through the public entry points (`own`), or the same thing in elementary torch operations on the same buffers.
Head counts and sizes are those of the paper's models (1024 = 16 x 64, 2048 = 32 x 64 or 16 x 128, 2880 = 32 x 90), of the packed
decode product's width (4096 = 32 x 128), and grouped forms of them (fewer key-value heads than query heads).
"""
import math
import random

import torch

own = False


def listed():
    return [
        # four sequences generate a token each through one layer of the smallest model: nothing but launches
        dict(name="cache_append", kind="cache", cache="int8", io="bf16", heads=16, kv_heads=16, d=64, page=16, batch=4, rows=1, len=777,
             ragged=True, window=0),
        # four prompts of 2048 tokens enter the cache of a 1.3B-shaped layer
        dict(name="cache_prompts", kind="cache", cache="int8", io="bf16", heads=32, kv_heads=32, d=64, page=64, batch=4, rows=2048,
             len=2048, ragged=False, window=0),
        # ragged continuations of cached prompts, heads of 90 (the 2.6B shape), full-precision activations into a 16-bit cache
        dict(name="cache_ragged_f32", kind="cache", cache="bf16", io="f32", heads=32, kv_heads=32, d=90, page=32, batch=9, rows=700,
             len=1531, ragged=True, window=0),
        # a short 16-bit history is read back, as before a sequence moves to other pages
        dict(name="read_short", kind="read", cache="bf16", io="bf16", heads=16, kv_heads=16, d=128, page=16, batch=2, rows=300, len=300,
             ragged=True, window=0),
        # the whole INT8 history of a ragged batch is read back in 16 bits
        dict(name="read_history", kind="read", cache="int8", io="bf16", heads=32, kv_heads=8, d=128, page=64, batch=16, rows=8192,
             len=8192, ragged=True, window=0),
        # one sequence, token by token, early on
        dict(name="decode_one", kind="decode", cache="int8", io="bf16", heads=16, kv_heads=16, d=128, page=16, batch=1, rows=1, len=517,
             ragged=False, window=0),
        # eight sequences of a 1.3B-shaped layer decoded together
        dict(name="decode_batch", kind="decode", cache="int8", io="bf16", heads=32, kv_heads=32, d=64, page=32, batch=8, rows=1, len=2048,
             ragged=False, window=0),
        # a full batch of very different lengths, eight key-value heads for 32 query heads, 16-bit cache
        dict(name="decode_ragged", kind="decode", cache="bf16", io="bf16", heads=32, kv_heads=8, d=128, page=64, batch=64, rows=1,
             len=8192, ragged=True, window=0),
        # few sequences with long histories: the split over the length carries it
        dict(name="decode_long", kind="decode", cache="int8", io="bf16", heads=32, kv_heads=8, d=128, page=128, batch=4, rows=1,
             len=131072, ragged=False, window=0),
        # one short prompt
        dict(name="prefill_short", kind="prefill", cache="bf16", io="bf16", heads=16, kv_heads=16, d=128, page=16, batch=1, rows=130,
             len=130, ragged=False, window=0),
        # ragged prompts behind cached beginnings, heads of 90, a sliding window
        dict(name="prefill_ragged", kind="prefill", cache="int8", io="bf16", heads=32, kv_heads=32, d=90, page=32, batch=7, rows=1500,
             len=2200, ragged=True, window=1024),
        # one long prompt, grouped heads
        dict(name="prefill_long", kind="prefill", cache="int8", io="bf16", heads=32, kv_heads=8, d=128, page=64, batch=1, rows=8192,
             len=8192, ragged=False, window=0),
    ]


# ---------------------------------------------------------------------------------------------------------------------
# more cases of the same ranges
# ---------------------------------------------------------------------------------------------------------------------
def _spread(rng, lo, hi):
    """A whole number in [lo, hi], even over the logarithm."""
    return min(max(int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))), lo), hi)


def draw(rng):
    """Caches of 1 to 131072 tokens a sequence, 1 to 64 sequences, prompts of 16 to 8192 rows, 1 to 16 query heads a key-value head."""
    most = [work(c) for c in listed()]
    most_bytes, most_flops = max(w["bytes"] for w in most), max(w["flops"] for w in most)
    while True:
        kind = rng.choice(["cache", "read", "decode", "decode", "prefill", "prefill"])
        kv_heads, group = rng.choice([1, 2, 4, 8, 16, 32]), rng.choice([1, 1, 2, 4, 5, 8, 16])
        c = dict(kind=kind, cache=rng.choice(["int8", "int8", "bf16"]), io="bf16", heads=kv_heads * group, kv_heads=kv_heads,
                 d=rng.choice([32, 64, 64, 80, 90, 96, 128, 128]), page=rng.choice([16, 32, 64, 128]), ragged=rng.random() < 0.6, window=0)
        if kind in ("cache", "read") and rng.random() < 0.3:
            c["io"] = "f32"
        if kind == "decode":
            c.update(batch=_spread(rng, 1, 64), rows=1, len=_spread(rng, 1, 131072))
        elif kind == "prefill":
            c.update(batch=_spread(rng, 1, 12), rows=_spread(rng, 16, 8192))
            c["len"] = c["rows"] + rng.choice([0, 0, _spread(rng, 1, 4096)])
        elif kind == "read":
            c.update(batch=_spread(rng, 1, 32), rows=_spread(rng, 1, 16384))
            c["len"] = c["rows"] + rng.choice([0, _spread(rng, 1, 2000)])
        else:
            c.update(batch=_spread(rng, 1, 32), rows=rng.choice([1, _spread(rng, 2, 8192)]))
            c["len"] = c["rows"] + rng.choice([0, _spread(rng, 1, 4096)])
        if kind in ("decode", "prefill") and rng.random() < 0.2:
            c["window"] = _spread(rng, 16, 4096)
        w = work(c)
        # (the plain form holds all the keys of a batch, as long as its longest sequence, and all the scores at once)
        keys, scores = c["batch"] * c["len"] * c["kv_heads"] * _padded(c["d"]), c["batch"] * c["heads"] * c["rows"] * c["len"]
        if c["heads"] <= 64 and w["bytes"] <= most_bytes and w["flops"] <= most_flops and max(keys * 4, scores) <= 2.2e9:
            return c


# ---------------------------------------------------------------------------------------------------------------------
# sizes
# ---------------------------------------------------------------------------------------------------------------------
def _sizes(c):
    """(rows, lengths) of the sequences: new rows of each, and its tokens in the cache with them.  Fixed by the case."""
    rng = random.Random(1000003 * c["len"] + 1009 * c["rows"] + c["batch"])
    rows, lens = [], []
    for b in range(c["batch"]):
        n = c["rows"] if b == 0 or not c["ragged"] else _spread(rng, max(1, c["rows"] // 32), c["rows"])
        before = c["len"] - c["rows"]
        if b > 0 and c["ragged"] and before:
            before = _spread(rng, max(1, before // 64), before)
        rows.append(n)
        lens.append(n + before)
    return rows, lens


def _padded(d):
    return -(-d // 32) * 32


def work(c):
    rows, lens = _sizes(c)
    T, d, es, io = sum(rows), c["d"], 1 if c["cache"] == "int8" else 2, 2 if c["io"] == "bf16" else 4
    token = 2 * c["kv_heads"] * (d * es + (4 if c["cache"] == "int8" else 0))          # keys and values of a token in the cache
    window = c["window"] or 1 << 40
    if c["kind"] == "cache":       # rows in, the cache written, the cache read, rows out
        return dict(bytes=2 * T * (2 * c["kv_heads"] * d * io + token), flops=8 * T * c["kv_heads"] * d)
    if c["kind"] == "read":
        return dict(bytes=T * (2 * c["kv_heads"] * d * io + token), flops=2 * T * c["kv_heads"] * d)
    own_rows = T * c["heads"] * (2 * d * io + 4)
    seen = pairs = 0
    for n, length in zip(rows, lens):
        first = length - n
        pairs += sum(min(p + 1, window) for p in range(first, length))
        seen += length - max(0, first + 1 - window)
    return dict(bytes=seen * token + own_rows, flops=4 * d * c["heads"] * pairs)


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _views(c, cache, n_pages):
    """Keys [page][head][token][Dp], values [page][head][token / 16][Dp][token % 16] and, for INT8, the steps of both [page][head][token]."""
    dp, page, es = _padded(c["d"]), c["page"], 1 if c["cache"] == "int8" else 2
    part = page * dp * es
    head = 2 * part + (8 * page if c["cache"] == "int8" else 0)
    v = cache.view(n_pages, c["kv_heads"], head)
    dtype = torch.int8 if c["cache"] == "int8" else torch.bfloat16
    keys = v[..., :part].view(dtype).unflatten(-1, (page, dp))
    values = v[..., part:2 * part].view(dtype).unflatten(-1, (page // 16, dp, 16))
    if c["cache"] != "int8":
        return keys, values, None, None
    return keys, values, v[..., 2 * part:2 * part + 4 * page].view(torch.float32), v[..., 2 * part + 4 * page:].view(torch.float32)


def _steps(x):
    """AbsMax INT8 of the last axis in 32 bits: codes (as 32-bit values) and what one step of them stands for."""
    top = x.abs().amax(-1, keepdim=True).clamp_min(1e-5)
    return torch.round(x * (128.0 / top)).clamp(-128, 127), top / 128.0


def _activations(g, shape, dtype):
    """N(0, 1) with one channel of a head in sixty-four eight times larger, as keys have them."""
    x = torch.randn(shape, generator=g, device="cuda")
    x[..., 5::64] *= 8.0
    return x.to(dtype)


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    rows, lens = _sizes(c)
    T, B, Hk, H, d, page = sum(rows), c["batch"], c["kv_heads"], c["heads"], c["d"], c["page"]
    io = torch.bfloat16 if c["io"] == "bf16" else torch.float32
    pages = [-(-n // page) for n in lens]
    n_pages, max_pages = sum(pages) + 3, max(pages) + 1
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32).cpu()
    table = torch.full((B, max_pages), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = order[at:at + n]
        at += n
    es = 1 if c["cache"] == "int8" else 2
    cache = torch.zeros(n_pages * Hk * (2 * page * _padded(d) * es + (8 * page if es == 1 else 0)), dtype=torch.uint8, device="cuda")
    s = dict(case=c, T=T, n_pages=n_pages, max_pages=max_pages, max_len=max(lens), cache=cache, table=table.cuda(),
             lens=torch.tensor(lens, dtype=torch.int32).cuda(),
             row_start=torch.tensor([sum(rows[:b]) for b in range(B + 1)], dtype=torch.int32).cuda())
    if c["kind"] == "cache":
        # the rows of a fused q/k/v projection where its parts are aligned, tensors of their own otherwise
        item = 2 if c["io"] == "bf16" else 4
        if H * d * item % 16 == 0 and Hk * d * item % 16 == 0:
            qkv = _activations(g, (T, H + 2 * Hk, d), io)
            s["K"], s["V"] = qkv[:, H:H + Hk], qkv[:, H + Hk:]
        else:
            s["K"], s["V"] = _activations(g, (T, Hk, d), io), _activations(g, (T, Hk, d), io)
    else:
        keys, values, key_steps, value_steps = _views(c, cache, n_pages)
        for to, steps, turned in ((keys, key_steps, False), (values, value_steps, True)):
            x = _activations(g, (n_pages, Hk, page, d), torch.bfloat16)
            if es == 1:
                x, step = _steps(x.float())
                steps.copy_(step.squeeze(-1))
            if turned:
                to[..., :d, :].copy_(x.unflatten(2, (page // 16, 16)).transpose(-1, -2))
            else:
                to[..., :d].copy_(x)
    if c["kind"] in ("cache", "read"):
        s["out"] = [torch.empty((T, Hk, d), dtype=io, device="cuda") for _ in range(2)]
    else:
        s["Q"] = _activations(g, (T, H, d), io)
        s["O"] = torch.empty((T, H, d), dtype=io, device="cuda")
        s["lse"] = torch.empty((T, H), dtype=torch.float32, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------
def _own(s):
    from paper_2602_22592_amd import binding as pq
    c = s["case"]
    if "plan" not in s:
        kv = pq.make_kv_desc(pq.PQ_KV_INT8 if c["cache"] == "int8" else pq.PQ_KV_BF16, c["kv_heads"], c["d"], c["page"], s["n_pages"],
                             c["batch"], s["max_pages"])
        at = pq.make_attn_desc(kv, c["heads"], window=c["window"], max_len=s["max_len"])
        s["plan"] = kv, at, pq.attn_decode_workspace(at) if c["kind"] == "decode" else None
    kv, at, ws = s["plan"]
    if c["kind"] == "cache":
        pq.kv_write(kv, s["K"], s["V"], s["cache"], s["lens"], s["table"], row_start=s["row_start"])
    if c["kind"] in ("cache", "read"):
        pq.kv_read(kv, s["cache"], s["lens"], s["table"], s["out"][0], s["out"][1], row_start=s["row_start"])
        return s["out"]
    if c["kind"] == "decode":
        pq.attn_decode(at, s["Q"], s["cache"], s["lens"], s["table"], s["O"], ws, lse=s["lse"])
    else:
        pq.attn_prefill(at, s["Q"], s["cache"], s["lens"], s["table"], s["row_start"], s["O"], lse=s["lse"])
    return s["O"], s["lse"]


def _places(s):
    """Of every row: its sequence, its number in it, and its position in the cache."""
    t = torch.arange(s["T"], device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(s["row_start"][1:].contiguous(), t, right=True)
    number = t.long() - s["row_start"][seq].long()
    n = (s["row_start"][1:] - s["row_start"][:-1]).long()
    return seq, number, s["lens"].long()[seq] - n[seq] + number


def _dense(s, page, slot):
    """Keys and values of the given places of the cache in 32 bits, [...][head][d]."""
    c = s["case"]
    keys, values, key_steps, value_steps = _views(c, s["cache"], s["n_pages"])
    k = keys[page, :, slot, :].float()[..., :c["d"]]
    v = values[page, :, slot // 16, :, slot % 16].float()[..., :c["d"]]
    if key_steps is not None:
        k, v = k * key_steps[page, :, slot].unsqueeze(-1), v * value_steps[page, :, slot].unsqueeze(-1)
    return k, v


def _plain_write(s):
    c = s["case"]
    seq, _, pos = _places(s)
    page, slot = s["table"][seq, pos // c["page"]].long(), pos % c["page"]
    keys, values, key_steps, value_steps = _views(c, s["cache"], s["n_pages"])
    k, v = s["K"].float(), s["V"].float()
    if key_steps is not None:
        (k, k_step), (v, v_step) = _steps(k), _steps(v)
        key_steps[page, :, slot] = k_step.squeeze(-1)
        value_steps[page, :, slot] = v_step.squeeze(-1)
    pad = torch.nn.functional.pad
    keys[page, :, slot, :] = pad(k, (0, _padded(c["d"]) - c["d"])).to(keys.dtype)
    values[page, :, slot // 16, :, slot % 16] = pad(v, (0, _padded(c["d"]) - c["d"])).to(values.dtype)


def _plain_read(s):
    c = s["case"]
    seq, _, pos = _places(s)
    k, v = _dense(s, s["table"][seq, pos // c["page"]].long(), pos % c["page"])
    return [k.to(s["out"][0].dtype), v.to(s["out"][1].dtype)]


def _plain_attention(s):
    c = s["case"]
    B, Hk, H, d, G = c["batch"], c["kv_heads"], c["heads"], c["d"], c["heads"] // c["kv_heads"]
    L, n = s["max_len"], c["rows"]
    p = torch.arange(L, device="cuda")
    page = s["table"][:, p // c["page"]].long().clamp_min(0)                            # [B][L]
    k, v = _dense(s, page, (p % c["page"]).expand(B, L))                                # [B][L][Hk][d]
    seq, number, pos = _places(s)
    q = torch.zeros((B, n, H, d), device="cuda")
    q[seq, number] = s["Q"].float()
    row_pos = torch.full((B, n), -1, dtype=torch.long, device="cuda")
    row_pos[seq, number] = pos
    q = q.view(B, n, Hk, G, d).permute(0, 2, 3, 1, 4).reshape(B, Hk, G * n, d)
    kt = k.permute(0, 2, 3, 1).contiguous()                                             # [B][Hk][d][L]
    scores = torch.matmul(q, kt).mul_(1.0 / math.sqrt(d)).view(B, Hk, G, n, L)
    hidden = p > row_pos.unsqueeze(-1)                                                  # [B][n][L]
    if c["window"]:
        hidden |= p <= row_pos.unsqueeze(-1) - c["window"]
    scores.masked_fill_(hidden.view(B, 1, 1, n, L), -math.inf)
    top = scores.amax(-1, keepdim=True).clamp_min(-3e38)
    scores.sub_(top).exp_()
    total = scores.sum(-1, keepdim=True)
    o = torch.matmul(scores.view(B, Hk, G * n, L), v.permute(0, 2, 1, 3).contiguous()).view(B, Hk, G, n, d)
    o = (o / total.clamp_min(1e-38)).permute(0, 3, 1, 2, 4).reshape(B, n, H, d)
    lse = (top + total.log()).squeeze(-1).permute(0, 3, 1, 2).reshape(B, n, H)
    return o[seq, number].to(s["O"].dtype), lse[seq, number]


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    if kind == "cache":
        _plain_write(state)
    if kind in ("cache", "read"):
        return _plain_read(state)
    return _plain_attention(state)


# ---------------------------------------------------------------------------------------------------------------------
# the same in 64 bits, sequence by sequence
# ---------------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    c, rows, lens = case, *_sizes(case)
    d, page, G = c["d"], c["page"], c["heads"] // c["kv_heads"]
    if c["kind"] == "cache":
        out = []
        for x in (s["K"], s["V"]):
            if c["cache"] == "int8":     # the codes are defined by a quotient and a product in 32 bits
                most = x.float().abs().max(-1, keepdim=True).values.clamp(min=1e-5)
                x = (x.float() * (128.0 / most)).round().clamp(-128, 127).double() * most.double() / 128
            else:                        # and a 16-bit cache holds 16 bits
                x = x.to(torch.bfloat16).double()
            out.append(x)
        return out
    keys, values, key_steps, value_steps = _views(c, s["cache"], s["n_pages"])
    table, outs = s["table"].cpu(), ([], [])
    at = 0
    for b, (n, length) in enumerate(zip(rows, lens)):
        used = table[b, :-(-length // page)].long().cuda()
        k = keys[used].double().transpose(1, 2).flatten(0, 1)[:length, :, :d]                               # [L][Hk][d]
        v = values[used].double().permute(0, 2, 4, 1, 3).flatten(0, 2)[:length, :, :d]
        if key_steps is not None:
            k = k * key_steps[used].double().transpose(1, 2).flatten(0, 1)[:length, :, None]
            v = v * value_steps[used].double().transpose(1, 2).flatten(0, 1)[:length, :, None]
        if c["kind"] == "read":
            outs[0].append(k[length - n:])
            outs[1].append(v[length - n:])
            continue
        place = torch.arange(length, device="cuda")
        mine = place[length - n:, None]
        seen = place[None] <= mine
        if c["window"]:
            seen &= place[None] > mine - c["window"]
        o = torch.empty((n, c["heads"], d), dtype=torch.float64, device="cuda")
        lse = torch.empty((n, c["heads"]), dtype=torch.float64, device="cuda")
        for h in range(c["heads"]):
            a = s["Q"][at:at + n, h].double() @ k[:, h // G].t().contiguous() / math.sqrt(d)
            a = torch.where(seen, a, -math.inf)
            lse[:, h] = torch.logsumexp(a, -1)
            o[:, h] = torch.exp(a - lse[:, h, None]) @ v[:, h // G].contiguous()
        outs[0].append(o)
        outs[1].append(lse)
        at += n
    return torch.cat(outs[0]), torch.cat(outs[1])
