"""What a training step of a layer's attention half needs beside its projections, as it is timed: rotary positions (also of single tokens), attention
over the rows of packed sequences with its gradient, and the AdamW step over many tensors.

Each case is one pass through the public entry points (`own`), or the same thing in elementary torch operations on the same buffers.
Head counts and sizes are those of the paper's models (2048 = 32 x 64 or 16 x 128, 2880 = 32 x 90, 4096 = 32 x 128), and grouped forms of them (fewer
key-value heads than query heads); the optimizer's tensors are those of a decoupled layer, or a mixed bag of sizes.
"""
import math
import random

import torch

own = False

BLOCK = 256                    # elements of a tensor that share the steps of their 8-bit states


def listed():
    return [
        # four sequences generate a token each: positions of the new queries and keys, nothing but a launch
        dict(name="rope_token", kind="rope", io="bf16", heads=16, kv_heads=16, d=64, rot=64, layout="half", inverse=False, parts=False, batch=4,
             rows=1, len=777, ragged=True),
        # ragged prompts behind cached beginnings, heads of 90 turned in part and pairs of neighbours, full precision
        dict(name="rope_ragged_f32", kind="rope", io="f32", heads=32, kv_heads=32, d=90, rot=46, layout="pairs", inverse=False, parts=False,
             batch=9, rows=700, len=1531, ragged=True),
        # the gradient of one long sequence's queries and keys, frequencies stretched for it
        dict(name="rope_long_grad", kind="rope", io="bf16", heads=32, kv_heads=8, d=128, rot=128, layout="half", inverse=True, parts=True, batch=1,
             rows=32768, len=32768, ragged=False),
        # one short sequence
        dict(name="attn_short", kind="attn", grad=False, heads=16, kv_heads=16, d=128, batch=1, rows=130, ragged=False, causal=True, window=0),
        # one long sequence, grouped heads
        dict(name="attn_long", kind="attn", grad=False, heads=32, kv_heads=8, d=128, batch=1, rows=8192, ragged=False, causal=True, window=0),
        # gradients: one short sequence ..
        dict(name="grad_short", kind="attn", grad=True, heads=16, kv_heads=16, d=128, batch=1, rows=130, ragged=False, causal=True, window=0),
        # .. packed ragged documents, heads of 90 (the 2.6B shape), a sliding window
        dict(name="grad_ragged", kind="attn", grad=True, heads=32, kv_heads=32, d=90, batch=7, rows=1500, ragged=True, causal=True, window=500),
        # .. four sequences of 2048 tokens through a 1.3B-shaped layer
        dict(name="grad_batch", kind="attn", grad=True, heads=32, kv_heads=32, d=64, batch=4, rows=2048, ragged=False, causal=True, window=0),
        # .. and one long sequence with grouped heads
        dict(name="grad_long", kind="attn", grad=True, heads=32, kv_heads=8, d=128, batch=1, rows=8192, ragged=False, causal=True, window=0),
        # the gains and scales of a small model: fifty tensors of up to 1500 elements
        dict(name="adamw_small", kind="adamw", layers=0, d=0, ffn=0, experts=0, rank=0, count=50, largest=1500, param="f32", grad="f32", state="f32"),
        # a mixed bag of odd sizes, 16-bit weights with 32-bit masters, 16-bit gradients, 32-bit states
        dict(name="adamw_masters", kind="adamw", layers=0, d=0, ffn=0, experts=0, rank=0, count=70, largest=1500001, param="bf16+f32", grad="bf16",
             state="f32"),
        # two layers of the 1.3B shape with their experts, 16-bit weights, 8-bit states
        dict(name="adamw_layers", kind="adamw", layers=2, d=2048, ffn=5504, experts=8, rank=32, count=0, largest=0, param="bf16", grad="f32",
             state="8bit"),
    ]


# ---------------------------------------------------------------------------------------------------------------------
# more cases of the same ranges
# ---------------------------------------------------------------------------------------------------------------------
def _spread(rng, lo, hi):
    """A whole number in [lo, hi], even over the logarithm."""
    return min(max(int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))), lo), hi)


def draw(rng):
    """1 to 8192 rows a sequence of attention and 32768 of positions, 1 to 64 sequences, 1 to 16 query heads a key-value head, 1 to 90 tensors."""
    most = [work(c) for c in listed()]
    most_bytes, most_flops = max(w["bytes"] for w in most), max(w["flops"] for w in most)
    while True:
        kind = rng.choice(["rope", "attn", "attn", "grad", "grad", "grad", "adamw", "adamw"])
        if kind == "adamw":
            c = dict(kind="adamw", layers=0, d=0, ffn=0, experts=0, rank=0, count=0, largest=0, param=rng.choice(["f32", "bf16", "bf16+f32"]),
                     grad=rng.choice(["f32", "f32", "bf16"]), state=rng.choice(["f32", "8bit"]))
            if rng.random() < 0.4:
                d = 32 * _spread(rng, 4, 70)
                c.update(layers=_spread(rng, 1, 6), d=d, ffn=4 * _spread(rng, d // 4, d), experts=rng.choice([1, 2, 8]), rank=8 * _spread(rng, 1, 16))
            else:
                c.update(count=_spread(rng, 1, 90), largest=_spread(rng, 1, 2000000))
        else:
            kv_heads, group = rng.choice([1, 2, 4, 8, 16, 32]), rng.choice([1, 1, 2, 4, 5, 8, 16])
            c = dict(kind="rope" if kind == "rope" else "attn", heads=kv_heads * group, kv_heads=kv_heads,
                     d=rng.choice([32, 64, 64, 80, 90, 96, 128, 128]), ragged=rng.random() < 0.6)
            if kind == "rope":
                c.update(io=rng.choice(["bf16", "bf16", "f32"]), rot=c["d"] if rng.random() < 0.6 else 2 * _spread(rng, 1, c["d"] // 2),
                         layout=rng.choice(["half", "half", "pairs"]), inverse=rng.random() < 0.3, parts=rng.random() < 0.3,
                         batch=_spread(rng, 1, 64), rows=rng.choice([1, _spread(rng, 2, 32768)]))
                c["len"] = c["rows"] + rng.choice([0, _spread(rng, 1, 100000)])
            else:
                c.update(grad=kind == "grad", batch=_spread(rng, 1, 12), rows=_spread(rng, 1, 8192), causal=rng.random() < 0.8, window=0)
                if c["causal"] and rng.random() < 0.25:
                    c["window"] = _spread(rng, 1, 4096)
        w = work(c)
        # (the plain form holds all the scores of a batch, as long as its longest sequence, at once)
        scores = c["batch"] * c["heads"] * c["rows"] ** 2 if c["kind"] == "attn" else 0
        if c.get("heads", 0) <= 64 and w["bytes"] <= most_bytes and w["flops"] <= most_flops and scores <= 2.2e9:
            return c


# ---------------------------------------------------------------------------------------------------------------------
# sizes
# ---------------------------------------------------------------------------------------------------------------------
def _rows(c):
    """(rows, lengths) of the sequences: their rows in the call, and their tokens up to the last of them.  Fixed by the case."""
    before = c.get("len", c["rows"]) - c["rows"]
    rng = random.Random(1000003 * before + 1009 * c["rows"] + c["batch"])
    rows, lens = [], []
    for b in range(c["batch"]):
        n, p = c["rows"], before
        if b > 0 and c["ragged"]:
            n = _spread(rng, max(1, n // 32), n)
            p = _spread(rng, max(1, p // 64), p) if p else 0
        rows.append(n)
        lens.append(n + p)
    return rows, lens


def _shapes(c):
    """Shapes of the tensors that the optimizer updates: of decoupled layers, or a mixed bag."""
    d, f, e, r = c["d"], c["ffn"], c["experts"], c["rank"]
    out = []
    for _ in range(c["layers"]):
        out += [(d,)] + [(d, d)] * 4 + [(d,)] + [(f, d)] * 2 + [(d, f)] + [(e, r, d)] * 2 + [(e, d, r), (e, d), (2,)]
    rng = random.Random(7919 * c["count"] + c["largest"])
    for i in range(c["count"]):
        out.append((c["largest"],) if i == 0 else (_spread(rng, 1, c["largest"]),))
    return out


def work(c):
    if c["kind"] == "adamw":
        n = sum(math.prod(s) for s in _shapes(c))
        blocks = sum(-(-math.prod(s) // BLOCK) for s in _shapes(c))
        # the gradient is read, the weight read and written; a 16-bit weight with a master is only written
        each = {"f32": 8, "bf16": 4, "bf16+f32": 10}[c["param"]] + (4 if c["grad"] == "f32" else 2)
        # (8 bits: their values are written as well)
        return dict(bytes=n * each + (16 * n if c["state"] == "f32" else 12 * n + 16 * blocks), flops=16 * n)
    rows, _ = _rows(c)
    T, H, Hk, d = sum(rows), c["heads"], c["kv_heads"], c["d"]
    if c["kind"] == "rope":
        n = T * (H + Hk) * d
        return dict(bytes=2 * n * (2 if c["io"] == "bf16" else 4), flops=3 * T * (H + Hk) * c["rot"])
    window = c["window"] or 1 << 40
    pairs = sum(sum(min(p + 1, window) for p in range(n)) if c["causal"] else n * n for n in rows)
    q, kv = T * H * d * 2, T * Hk * d * 2
    if c["grad"]:                  # q, k, v, o, its gradient and lse in; three gradients out.  S, dP, dQ, dK, dV
        return dict(bytes=4 * q + 4 * kv + 4 * T * H, flops=10 * d * H * pairs)
    return dict(bytes=2 * q + 2 * kv + 4 * T * H, flops=4 * d * H * pairs)


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _activations(g, shape, dtype):
    """N(0, 1) with one channel of a head in sixty-four four times larger."""
    x = torch.randn(shape, generator=g, device="cuda")
    x[..., 5::64] *= 4.0
    return x.to(dtype)


def _parts(c, T, g, dtype, values):
    """Queries, keys and (with `values`) values: parts of the rows of a fused projection where those are aligned, tensors of their own otherwise."""
    H, Hk, d, item = c["heads"], c["kv_heads"], c["d"], 2 if dtype == torch.bfloat16 else 4
    make = (lambda shape: _activations(g, shape, dtype)) if g is not None else (lambda shape: torch.empty(shape, dtype=dtype, device="cuda"))
    heads = [H, Hk, Hk] if values else [H, Hk]
    if H * d * item % 16 == 0 and Hk * d * item % 16 == 0:
        return list(make((T, sum(heads), d)).split(heads, dim=1))
    return [make((T, h, d)) for h in heads]


def _frequencies(c):
    """Turns per position of every pair, in 64 bits.  `parts`: eight times the context of 4096; pairs that turn 32 times and more within it are left as
    they are, those that turn less than once are slowed down eight times, a ramp between."""
    i = torch.arange(c["rot"] // 2, dtype=torch.float64)
    f = 10000.0 ** (-2.0 * i / c["rot"]) / (2.0 * math.pi)
    if c["parts"]:
        keep = ((4096.0 * f - 1.0) / 31.0).clamp(0.0, 1.0)
        f = f * (keep + (1.0 - keep) / 8.0)
    return f.cuda()


def _encode(x, top_code):
    """8-bit codes of the square law, |x| = code^2 step, and the step of each block, in 32 bits (the root in 64: the nearest code)."""
    step = (x.abs().amax(-1, keepdim=True) * (1.0 / top_code ** 2)).clamp_min(2.0 ** -126)
    code = (x.abs() * (1.0 / step)).double().sqrt().round().clamp_max(top_code)
    return code.float(), step


def _encode_m(m):
    code, step = _encode(m, 127)
    return torch.where(m < 0, -code, code), step


def _encode_root(r):
    """(a root that is not zero does not become zero: it is divided by)"""
    code, step = _encode(r, 255)
    return torch.where(r > 0, code.clamp_min(1), code), step


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    if c["kind"] == "adamw":
        return _prepare_adamw(c, g)
    rows, lens = _rows(c)
    T, B, H, Hk, d = sum(rows), c["batch"], c["heads"], c["kv_heads"], c["d"]
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    s = dict(case=c, T=T, row_start=i32([sum(rows[:b]) for b in range(B + 1)]), lens=i32(lens))
    if c["kind"] == "rope":
        io = torch.bfloat16 if c["io"] == "bf16" else torch.float32
        s["Q"], s["K"] = _parts(c, T, g, io, False)
        s["out"] = _parts(c, T, None, io, False)
        s["freqs"] = _frequencies(c)
        s["scale"] = 0.1 * math.log(8.0) + 1.0 if c["parts"] else 1.0
        return s
    s["Q"], s["K"], s["V"] = _parts(c, T, g, torch.bfloat16, True)
    s["O"] = torch.empty((T, H, d), dtype=torch.bfloat16, device="cuda")
    s["lse"] = torch.empty((T, H), dtype=torch.float32, device="cuda")
    if c["grad"]:                  # what the forward pass has left, and the gradient of its output
        o, lse = _plain_attention(s)
        s["O"].copy_(o)
        s["lse"].copy_(lse)
        s["dO"] = _activations(g, (T, H, d), torch.bfloat16)
        s["out"] = _parts(c, T, None, torch.bfloat16, True)
    return s


def _prepare_adamw(c, g):
    """Each kind of tensor in one buffer, as training programs keep them: a tensor begins at a multiple of BLOCK elements, zeros up to the next."""
    sizes = [math.prod(shape) for shape in _shapes(c)]
    starts, N = [], 0
    for n in sizes:
        starts.append(N)
        N += -(-n // BLOCK) * BLOCK
    edges = torch.zeros(N + 1, dtype=torch.int8, device="cuda")
    edges[torch.tensor(starts, device="cuda")] += 1
    edges[torch.tensor([a + n for a, n in zip(starts, sizes)], device="cuda")] -= 1
    used = edges[:N].cumsum(0, dtype=torch.int8)
    rand = lambda: torch.randn(N, generator=g, device="cuda") * used
    p = rand() * 0.02
    # gradients whose sizes differ by some powers of ten from element to element
    grad = (rand() * torch.exp(1.5 * rand()) * 1e-3).to(torch.float32 if c["grad"] == "f32" else torch.bfloat16)
    m, v = rand() * 3e-4, (rand() * torch.exp(rand()) * 1e-3) ** 2
    s = dict(case=c, starts=starts, sizes=sizes, grads=grad, masters=None, steps=None, values=None,
             hyper=dict(lr=1e-3, weight_decay=0.1, grad_scale=0.5, step=137, beta1=0.9, beta2=0.95, eps=1e-8))
    if c["param"] == "bf16+f32":
        s["masters"] = p
    s["params"] = p if c["param"] == "f32" else p.to(torch.bfloat16)
    if c["state"] == "f32":
        s["m"], s["v"] = m, v
    else:
        (qm, sm), (qr, sr) = _encode_m(m.view(-1, BLOCK)), _encode_root(v.sqrt().view(-1, BLOCK))
        s["m"], s["v"], s["steps"] = qm.to(torch.int8).view(-1), qr.to(torch.uint8).view(-1), torch.cat([sm, sr], 1).contiguous()
        s["values"] = torch.zeros_like(p), torch.zeros_like(p)
    return s


# ---------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------
def _own(s):
    from paper_2602_22592_amd import binding as pq
    c = s["case"]
    if c["kind"] == "rope":
        if "plan" not in s:
            s["plan"] = pq.make_rope_desc(c["heads"], c["kv_heads"], c["d"], c["batch"], rot_dim=c["rot"],
                                          layout=pq.PQ_ROPE_HALF if c["layout"] == "half" else pq.PQ_ROPE_PAIRS, inverse=c["inverse"],
                                          scale=s["scale"])
        pq.rope(s["plan"], s["Q"], s["K"], s["freqs"], s["out"][0], s["out"][1], row_start=s["row_start"], lens=s["lens"])
        return s["out"]
    if c["kind"] == "attn":
        if "plan" not in s:
            desc = pq.make_self_attn_desc(c["heads"], c["kv_heads"], c["d"], c["batch"], causal=c["causal"], window=c["window"])
            s["plan"] = desc, pq.self_attn_bwd_workspace(desc, s["T"]) if c["grad"] else None
        desc, ws = s["plan"]
        if not c["grad"]:
            pq.self_attn_fwd(desc, s["Q"], s["K"], s["V"], s["row_start"], s["O"], s["lse"])
            return s["O"], s["lse"]
        dQ, dK, dV = s["out"]
        pq.self_attn_bwd(desc, s["dO"], s["Q"], s["K"], s["V"], s["O"], s["lse"], s["row_start"], dQ, dK, dV, ws)
        return s["out"]
    if "plan" not in s:
        h = s["hyper"]
        tensors = lambda x, of=1: None if x is None else [x[a // of:a // of + -(-n // of)] for a, n in zip(s["starts"], s["sizes"])]
        m_values, v_values = s["values"] or (None, None)
        s["plan"] = pq.AdamWTensors(tensors(s["params"]), tensors(s["grads"]), tensors(s["m"]), tensors(s["v"]), steps=tensors(s["steps"], BLOCK),
                                    masters=tensors(s["masters"]), m_values=tensors(m_values), v_values=tensors(v_values), beta1=h["beta1"],
                                    beta2=h["beta2"], eps=h["eps"])
        s["scalars"] = pq.adamw_scalars(s["plan"], h["step"], h["lr"], h["weight_decay"], h["grad_scale"])
    pq.adamw_step(s["plan"], s["scalars"])
    if s["values"]:                # 8-bit states are read back as the values they stand for, as a checkpoint takes them
        pq.adamw_read(s["plan"])
    return _updated(s)


def _updated(s):
    """Weights, masters and states."""
    return [s["params"]] + ([] if s["masters"] is None else [s["masters"]]) + list(s["values"] or (s["m"], s["v"]))


def _places(s):
    """Of every row: its sequence, its number in it, and its position."""
    t = torch.arange(s["T"], device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(s["row_start"][1:].contiguous(), t, right=True)
    number = t.long() - s["row_start"][seq].long()
    n = (s["row_start"][1:] - s["row_start"][:-1]).long()
    return seq, number, s["lens"].long()[seq] - n[seq] + number


def _plain_rope(s):
    c = s["case"]
    rot, half = c["rot"], c["rot"] // 2
    turns = _places(s)[2].double().unsqueeze(-1) * s["freqs"]                           # (positions reach far: angles in 64 bits)
    angle = (turns - turns.round()) * (2.0 * math.pi * (-1.0 if c["inverse"] else 1.0))
    cos, sin = (torch.cos(angle) * s["scale"]).float().unsqueeze(1), (torch.sin(angle) * s["scale"]).float().unsqueeze(1)
    out = []
    for x, y in zip((s["Q"], s["K"]), s["out"]):
        x = x.float()
        a, b = (x[..., :half], x[..., half:rot]) if c["layout"] == "half" else (x[..., 0:rot:2], x[..., 1:rot:2])
        u, w = a * cos - b * sin, b * cos + a * sin
        u = torch.cat([u, w], -1) if c["layout"] == "half" else torch.stack([u, w], -1).flatten(-2)
        out.append(torch.cat([u, x[..., rot:]], -1).to(y.dtype))
    return out


def _batched(s, x, seq, number):
    """Rows [T][h][d] as [B][h][n][d] in 32 bits, zeros behind a sequence's last row."""
    c = s["case"]
    y = torch.zeros((c["batch"], c["rows"], x.shape[1], c["d"]), device="cuda")
    y[seq, number] = x.float()
    return y.permute(0, 2, 1, 3).contiguous()


def _softmax(s, q, k):
    """Probabilities [B][Hk][G n][n] and the logarithm of their sum before the quotient."""
    c = s["case"]
    B, Hk, G, n = c["batch"], c["kv_heads"], c["heads"] // c["kv_heads"], c["rows"]
    scores = torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(1.0 / math.sqrt(c["d"])).view(B, Hk, G, n, n)
    t = torch.arange(n, device="cuda")
    count = (s["row_start"][1:] - s["row_start"][:-1]).view(B, 1, 1)
    hidden = (t >= count).expand(B, n, n)
    if c["causal"]:
        hidden = hidden | (t > t.unsqueeze(-1))
        if c["window"]:
            hidden = hidden | (t <= t.unsqueeze(-1) - c["window"])
    scores.masked_fill_(hidden.view(B, 1, 1, n, n), -math.inf)
    top = scores.amax(-1, keepdim=True).clamp_min(-3e38)
    scores.sub_(top).exp_()
    total = scores.sum(-1, keepdim=True).clamp_min(1e-38)                               # (rows behind the last: nothing seen)
    scores.div_(total)
    return scores.view(B, Hk, G * n, n), (top + total.log()).squeeze(-1)


def _plain_attention(s):
    c = s["case"]
    B, Hk, G, n, d = c["batch"], c["kv_heads"], c["heads"] // c["kv_heads"], c["rows"], c["d"]
    seq, number, _ = _places(s)
    q, k, v = (_batched(s, s[x], seq, number) for x in "QKV")
    p, lse = _softmax(s, q.view(B, Hk, G * n, d), k)
    o = torch.matmul(p, v).view(B, Hk * G, n, d).transpose(1, 2)
    return o[seq, number].to(torch.bfloat16), lse.reshape(B, Hk * G, n).transpose(1, 2)[seq, number]


def _plain_gradient(s):
    c = s["case"]
    B, Hk, G, n, d = c["batch"], c["kv_heads"], c["heads"] // c["kv_heads"], c["rows"], c["d"]
    seq, number, _ = _places(s)
    q, k, v, do = (_batched(s, s[x], seq, number) for x in ("Q", "K", "V", "dO"))
    q, do = q.view(B, Hk, G * n, d), do.view(B, Hk, G * n, d)
    p, _ = _softmax(s, q, k)
    dv = torch.matmul(p.transpose(-1, -2), do)
    dp = torch.matmul(do, v.transpose(-1, -2).contiguous())
    dp.sub_((dp * p).sum(-1, keepdim=True)).mul_(p).mul_(1.0 / math.sqrt(d))
    del p
    dk = torch.matmul(dp.transpose(-1, -2), q)
    dq = torch.matmul(dp, k).view(B, Hk * G, n, d)
    return [x.transpose(1, 2)[seq, number].to(torch.bfloat16) for x in (dq, dk, dv)]


def _decode(qm, qr, steps):
    qm, qr = qm.view(-1, BLOCK).float(), qr.view(-1, BLOCK).float()
    return qm * qm.abs() * steps[:, :1], qr * qr * steps[:, 1:]


def _plain_adamw(s):
    h, eight = s["hyper"], s["steps"] is not None
    f32 = lambda x: torch.tensor(x, dtype=torch.float32).item()                         # a factor in 32 bits
    g = s["grads"].float() * h["grad_scale"]
    if eight:
        g = g.view(-1, BLOCK)
        m, r = _decode(s["m"], s["v"], s["steps"])
        v = r * r
    else:
        m, v = s["m"], s["v"]
    m = m * f32(h["beta1"]) + g * f32(1.0 - h["beta1"])
    v = v * f32(h["beta2"]) + g * f32(1.0 - h["beta2"]) * g
    r = v.double().sqrt().float()
    if eight:
        (qm, sm), (qr, sr) = _encode_m(m), _encode_root(r)
        s["m"].copy_(qm.view(-1))
        s["v"].copy_(qr.view(-1))
        s["steps"].copy_(torch.cat([sm, sr], 1))
        back_m, back_r = _decode(s["m"], s["v"], s["steps"])
        s["values"][0].copy_(back_m.view(-1))
        s["values"][1].copy_((back_r * back_r).view(-1))
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    size, root = h["lr"] / (1.0 - h["beta1"] ** h["step"]), 1.0 / math.sqrt(1.0 - h["beta2"] ** h["step"])
    w = s["params"] if s["masters"] is None else s["masters"]
    w.copy_(w.float() * (1.0 - h["lr"] * h["weight_decay"]) - (m * size / (r * root + h["eps"])).view(-1))
    if s["masters"] is not None:
        s["params"].copy_(w)
    return _updated(s)


def run(state):
    if own:
        return _own(state)
    c = state["case"]
    if c["kind"] == "rope":
        return _plain_rope(state)
    if c["kind"] == "adamw":
        return _plain_adamw(state)
    return _plain_gradient(state) if c["grad"] else _plain_attention(state)


# ---------------------------------------------------------------------------------------------------------------------
# the same in 64 bits, sequence by sequence, head by head, tensor by tensor
# ---------------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rope":
        return _exact_rope(s)
    if case["kind"] == "adamw":
        return _exact_adamw(s)
    return _exact_attention(s)


def _exact_rope(s):
    c, (rows, lens) = s["case"], _rows(s["case"])
    pos = torch.cat([torch.arange(length - n, length, dtype=torch.float64) for n, length in zip(rows, lens)]).cuda()
    outs = [x.double() for x in (s["Q"], s["K"])]
    for i in range(c["rot"] // 2):
        a = torch.remainder(pos * s["freqs"][i], 1.0) * (2.0 * math.pi)
        z = torch.polar(torch.full_like(a, s["scale"]), -a if c["inverse"] else a).view(-1, 1)
        at = (i, i + c["rot"] // 2) if c["layout"] == "half" else (2 * i, 2 * i + 1)
        for x in outs:
            y = torch.complex(x[..., at[0]], x[..., at[1]]) * z
            x[..., at[0]], x[..., at[1]] = y.real, y.imag
    return outs


def _exact_attention(s):
    c, (rows, _) = s["case"], _rows(s["case"])
    H, Hk, d = c["heads"], c["kv_heads"], c["d"]
    f64 = lambda *shape: torch.zeros(shape, dtype=torch.float64, device="cuda")
    o, lse, dq, dk, dv = f64(s["T"], H, d), f64(s["T"], H), f64(s["T"], H, d), f64(s["T"], Hk, d), f64(s["T"], Hk, d)
    at = 0
    for n in rows:
        here = slice(at, at + n)
        at += n
        seen = torch.ones((n, n), dtype=torch.bool, device="cuda")
        if c["causal"]:
            seen = seen.tril()
            if c["window"]:
                seen = seen.triu(1 - c["window"])
        for h in range(H):
            j = h * Hk // H
            q, k, v = s["Q"][here, h].double(), s["K"][here, j].double(), s["V"][here, j].double()
            a = torch.where(seen, q @ k.t().contiguous() / math.sqrt(d), -math.inf)
            lse[here, h] = torch.logsumexp(a, -1)
            p = torch.exp(a - lse[here, h, None])
            o[here, h] = p @ v
            if c["grad"]:
                do = s["dO"][here, h].double()
                dp = do @ v.t().contiguous()
                ds = p * (dp - (p * dp).sum(-1, keepdim=True)) / math.sqrt(d)
                dq[here, h] = ds @ k
                dk[here, j] += ds.t() @ q
                dv[here, j] += p.t() @ do
    return [dq, dk, dv] if c["grad"] else (o, lse)


def _exact_codes(x, top):
    """Nearest codes of the square law among x / step, found among the borders (k + 1/2)^2 between them; the step and the quotient are defined in 32 bits."""
    step = torch.clamp(x.abs().max(-1, keepdim=True).values * (1.0 / top ** 2), min=2.0 ** -126)
    y = (x.abs() * (1.0 / step)).double()
    borders = (torch.arange(top, dtype=torch.float64, device="cuda") + 0.5) ** 2
    code = torch.bucketize(y, borders)
    tie = (code < top) & (y == borders[code.clamp(max=top - 1)]) & (code % 2 == 1)     # halfway: the even one
    return (code + tie.long()).double(), step.double()


def _exact_adamw(s):
    h = s["hyper"]
    b1, b2, t = h["beta1"], h["beta2"], h["step"]
    g = s["grads"].double() * h["grad_scale"]
    if s["steps"] is None:
        m0, v0 = s["m"].double(), s["v"].double()
    else:
        step = s["steps"].repeat_interleave(BLOCK, 0)
        q, u = s["m"].float(), s["v"].float()
        m0 = torch.copysign(q.double().square(), q.double()) * step[:, 0].double()
        v0 = (u.double().square() * step[:, 1].double()).square()
    m, v = b1 * m0 + (1.0 - b1) * g, b2 * v0 + (1.0 - b2) * g * g
    w = (s["params"] if s["masters"] is None else s["masters"]).double()
    w = w - h["lr"] * (h["weight_decay"] * w + (m / (1.0 - b1 ** t)) / ((v / (1.0 - b2 ** t)).sqrt() + h["eps"]))
    out = [w] if s["masters"] is None else [w, w]
    if s["steps"] is None:
        return out + [m, v]
    # the codes are defined by the new moments in 32 bits, each product and sum rounded
    k = torch.tensor([b1, 1.0 - b1, b2, 1.0 - b2], dtype=torch.float64).float().cuda()
    g = g.float()                                                                       # (the scale is a power of two)
    m32 = (q * q.abs() * step[:, 0]) * k[0] + g * k[1]
    root = u.square() * step[:, 1]
    r32 = (root.square() * k[2] + g * k[3] * g).double().sqrt().float()
    (qm, sm), (qr, sr) = _exact_codes(m32.view(-1, BLOCK), 127), _exact_codes(r32.view(-1, BLOCK), 255)
    qr = torch.where(r32.view(-1, BLOCK) > 0, qr.clamp(min=1), qr)
    return out + [(qm.square() * sm * m32.view(-1, BLOCK).sign()).view(-1), (qr.square() * sr).square().view(-1)]
