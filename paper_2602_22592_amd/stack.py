"""Drivers that chain the library's calls into layers.

Stack: a stack of transformer-shaped layers made of pQuant linears only (no attention core, no norms):

    per layer:  q,k,v = L_q(h), L_k(h), L_v(h)      pure 1-bit linears (Sec. 3.1: the MHA projections)
                m = (q + k + v) / 3                 stand-in for the attention core (glue)
                h1 = h + L_o(m)                     residual (glue)
                h2 = h1 + FFN(h1)                   decoupled FFN with routed experts (Sec. 3.2, 3.3)

It exists to time the linears of a 24-layer 1.3B-shaped model end to end.  With an AttentionCore m is attention(rotary(q), rotary(k), v) in its place, and
Stack.optimizer lays out the AdamW step of all layers' weights: forward, backward and that step train these.  An FFN's alpha and beta are host numbers
(`layers[l]["ffn_desc"].alpha` and `.beta`, read by every call, fixed in a captured one); their gradients are in backward's "dab", and nothing here applies them.

CachedAttention: the attention half of a layer at inference, on packed weights and a paged key-value cache:

    q, k, v = L_q(x), L_k(x), L_v(x)                pure 1-bit linears (Sec. 3.1)
    out = x + L_o(attention(q, cache + k, v))       prompts row by row, then one token of every sequence at a time;
                                                    with freqs, q and k turned by their tokens' positions first

This module only sequences C-ABI calls (pq_linear_*, pq_ffn_*, pq_decode_gemv, pq_kv_*, pq_attn_*, pq_rope, pq_self_attn_*, pq_adamw_*, pq_glue_*);
PyTorch provides the device buffers.
"""
from __future__ import annotations

import torch

from . import binding as pq


class AttentionCore:
    """What stands between the q, k, v projections and the o projection in training: rotary positions and attention over packed sequences.

    row_start [n_seqs + 1] int32 on the GPU: the sequences' rows among the `tokens` of a call; it may change from step to step.  Rows of no sequence come
    out as zeros and have no gradient: the kernels leave them alone, so every call clears what it is about to write (the products that read it take all
    rows).  freqs [rot_dim / 2] (rope_freqs), or None for attention without positions.  The workspace is the core's: calls that may overlap need one each."""

    def __init__(self, tokens, n_heads, n_kv_heads, d_head, n_seqs, freqs=None, rot_dim=0, layout=pq.PQ_ROPE_HALF, rope_scale=1.0, window=0, causal=True,
                 device="cuda"):
        self.T, self.H, self.Hk, self.dh = tokens, n_heads, n_kv_heads, d_head
        self.attn = pq.make_self_attn_desc(n_heads, n_kv_heads, d_head, n_seqs, causal=causal, window=window)
        self.freqs = freqs
        if freqs is not None:
            self.turn, self.turn_back = (pq.make_rope_desc(n_heads, n_kv_heads, d_head, n_seqs, rot_dim=rot_dim, layout=layout, inverse=i, scale=rope_scale)
                                         for i in (False, True))
        self.ws = pq.self_attn_bwd_workspace(self.attn, tokens, device)

    def saved(self, device="cuda"):
        """The buffers of one layer that its backward pass reads: turned q and k, v, the output and lse."""
        z = lambda heads: torch.zeros((self.T, heads, self.dh), dtype=torch.bfloat16, device=device)
        return dict(q=z(self.H), k=z(self.Hk), v=z(self.Hk), o=z(self.H), lse=torch.zeros((self.T, self.H), dtype=torch.float32, device=device))

    def check(self, row_start):
        """For whoever launches something in front of the core's calls: a refusal between them would leave buffers that nobody has filled."""
        if row_start is None:
            raise pq.PQError("row_start: a stack with an AttentionCore is given its sequences' rows")
        pq._index_check(self.ws.get_device(), "row_start", row_start, self.attn.n_seqs + 1)

    def forward(self, s, row_start):
        """s: a layer's buffers with the projections in q, k and v.  Turns q and k in place and returns the output [T, n_heads * d_head]."""
        if self.freqs is not None:
            pq.rope(self.turn, s["q"], s["k"], self.freqs, s["q"], s["k"], row_start=row_start)
        s["o"].zero_()
        pq.self_attn_fwd(self.attn, s["q"], s["k"], s["v"], row_start, s["o"], s["lse"])
        return s["o"].view(self.T, -1)

    def backward(self, dm, s, row_start, dq, dk, dv):
        """The gradients of the projections, [T, heads * d_head] each, from that of the output."""
        three = [x.zero_().view(self.T, -1, self.dh) for x in (dq, dk, dv)]
        pq.self_attn_bwd(self.attn, dm, s["q"], s["k"], s["v"], s["o"], s["lse"], row_start, *three, self.ws)
        if self.freqs is not None:
            pq.rope(self.turn_back, three[0], three[1], self.freqs, three[0], three[1], row_start=row_start)


class Stack:
    """core: an AttentionCore of `tokens` rows in place of the stand-in.  Wk and Wv then have n_kv_heads * d_head rows, and forward and backward are given
    row_start."""

    def __init__(self, n_layers, tokens, d_model, d_ffn, n_experts, hp_rank, top_k, alphas, betas, device="cuda", core=None):
        self.L, self.T, self.D, self.F = n_layers, tokens, d_model, d_ffn
        self.E, self.r, self.k = n_experts, hp_rank, top_k
        bf = torch.bfloat16
        self.lin_desc = pq.make_desc(tokens, d_model, d_model, hp_rank=0, io_dtype=pq.PQ_BF16, alpha=0.0, beta=1.0)
        self.core = core
        if core is not None:
            if core.T != tokens or core.H * core.dh != d_model:
                raise pq.PQError(f"the core has {core.T} rows of {core.H} heads of {core.dh}: {tokens} rows of d_model={d_model} are wanted")
            self._build_core(n_layers, tokens, d_model, d_ffn, n_experts, hp_rank, top_k, alphas, betas, device)
            return
        self.layers = []
        lin_ws = ffn_ws = None                       # one scratch buffer per kind, shared by all layers
        for l in range(n_layers):
            ffn_desc = pq.FFNDesc(tokens, d_model, d_ffn, hp_rank, n_experts, top_k, pq.PQ_BF16, alphas[l], betas[l])
            buf = {}
            for n in ("q", "k", "v", "o"):
                buf[n] = pq.LinearBuffers(self.lin_desc, device, ws=lin_ws)
                lin_ws = buf[n].ws
            fb = pq.FFNBuffers(ffn_desc, device, ws=ffn_ws)
            ffn_ws = fb.ws
            st = {n: torch.empty((tokens, d_model), dtype=bf, device=device) for n in ("h", "m", "h1")}
            self.layers.append(dict(ffn_desc=ffn_desc, ffn_buf=fb, lin_buf=buf, **st))
        e = lambda: torch.empty((tokens, d_model), dtype=bf, device=device)
        self.t = [e() for _ in range(5)]              # scratch activations
        self.out = e()
        self.dh = [e(), e()]
        self.dab = torch.empty((2,), dtype=torch.float32, device=device)

    def _build_core(self, n_layers, tokens, d_model, d_ffn, n_experts, hp_rank, top_k, alphas, betas, device):
        core, bf = self.core, torch.bfloat16
        self.kv_desc = pq.make_desc(tokens, d_model, core.Hk * core.dh, hp_rank=0, io_dtype=pq.PQ_BF16, alpha=0.0, beta=1.0)
        self.layers, ws = [], {}
        for l in range(n_layers):
            ffn_desc = pq.FFNDesc(tokens, d_model, d_ffn, hp_rank, n_experts, top_k, pq.PQ_BF16, alphas[l], betas[l])
            buf = {}
            for n in "qkvo":
                wide = n in "qo"
                buf[n] = pq.LinearBuffers(self.lin_desc if wide else self.kv_desc, device, ws=ws.get(wide))
                ws[wide] = buf[n].ws
            fb = pq.FFNBuffers(ffn_desc, device, ws=ws.get("ffn"))
            ws["ffn"] = fb.ws
            st = {n: torch.empty((tokens, d_model), dtype=bf, device=device) for n in ("h", "h1")}
            self.layers.append(dict(ffn_desc=ffn_desc, ffn_buf=fb, lin_buf=buf, core=core.saved(device), **st))
        e = lambda d=d_model: torch.empty((tokens, d), dtype=bf, device=device)
        self.t = [e() for _ in range(5)]
        self.dkv = [torch.zeros((tokens, core.Hk * core.dh), dtype=bf, device=device) for _ in range(2)]
        self.dq = torch.zeros((tokens, d_model), dtype=bf, device=device)
        self.out = e()
        self.dh = [e(), e()]
        self.dab = torch.empty((2,), dtype=torch.float32, device=device)

    def _desc(self, n):
        return self.kv_desc if self.core is not None and n in "kv" else self.lin_desc

    def _forward_core(self, h0, weights, row_start):
        h, core = h0, self.core
        core.check(row_start)
        o, f = self.t[:2]
        for ly, w in zip(self.layers, weights):
            ly["h"].copy_(h)
            s = ly["core"]
            for n in "qkv":
                pq.linear_fwd(self._desc(n), ly["h"], w["W" + n], s[n].view(self.T, -1), ly["lin_buf"][n])
            m = core.forward(s, row_start)
            pq.linear_fwd(self.lin_desc, m, w["Wo"], o, ly["lin_buf"]["o"])
            pq.glue_lincomb(ly["h1"], [ly["h"], o], [1.0, 1.0])
            pq.ffn_fwd(ly["ffn_desc"], ly["h1"], w["W_up"], w["W_gate"], w["W_down"], w["Up"], w["Gate"], w["Down"], w["Wr"],
                       f, ly["ffn_buf"])
            pq.glue_lincomb(self.out, [ly["h1"], f], [1.0, 1.0])
            h = self.out
        return self.out

    def _attention_backward(self, d_out, ly, w, g, row_start):
        """d_out: the gradient of the o projection's output.  Returns those of the layer's input through q, k and v."""
        s, (dm, dxq, dxk, dxv) = ly["core"], self.t[1:]
        pq.linear_bwd(self.lin_desc, d_out, s["o"].view(self.T, -1), w["Wo"], ly["lin_buf"]["o"], dm, g["Wo"], self.dab)
        self.core.backward(dm.view(self.T, self.core.H, self.core.dh), s, row_start, self.dq, *self.dkv)
        for n, dy, dx in (("q", self.dq, dxq), ("k", self.dkv[0], dxk), ("v", self.dkv[1], dxv)):
            pq.linear_bwd(self._desc(n), dy, ly["h"], w["W" + n], ly["lin_buf"][n], dx, g["W" + n], self.dab)
        return [dxq, dxk, dxv]

    def optimizer(self, weights, grads, names=None, **kw):
        """The AdamW step over all layers' weights with backward's gradients (`names`: all of a layer's tensors unless given; alpha and beta are none of
        them).  kw: as AdamWTensors takes them; masters=True makes fp32 masters of the weights as they are."""
        pairs = [(w[n], g[n]) for w, g in zip(weights, grads) for n in (names or [n for n in w if n in g])]
        if kw.get("masters") is True:
            kw["masters"] = [p.float() for p, _ in pairs]
        return pq.AdamWTensors([p for p, _ in pairs], [g for _, g in pairs], **kw)

    def forward(self, h0, weights, row_start=None):
        if self.core is not None:
            return self._forward_core(h0, weights, row_start)
        h = h0
        q, k, v, o, f = self.t
        for l, (ly, w) in enumerate(zip(self.layers, weights)):
            ly["h"].copy_(h)
            for n, y in (("q", q), ("k", k), ("v", v)):
                pq.linear_fwd(self.lin_desc, ly["h"], w["W" + n], y, ly["lin_buf"][n])
            pq.glue_lincomb(ly["m"], [q, k, v], [1 / 3, 1 / 3, 1 / 3])
            pq.linear_fwd(self.lin_desc, ly["m"], w["Wo"], o, ly["lin_buf"]["o"])
            pq.glue_lincomb(ly["h1"], [ly["h"], o], [1.0, 1.0])
            pq.ffn_fwd(ly["ffn_desc"], ly["h1"], w["W_up"], w["W_gate"], w["W_down"], w["Up"], w["Gate"], w["Down"], w["Wr"],
                       f, ly["ffn_buf"])
            pq.glue_lincomb(self.out, [ly["h1"], f], [1.0, 1.0])
            h = self.out
        return self.out

    def backward(self, dY, weights, grads, row_start=None):
        """grads: per-layer dict of fp32 tensors shaped like the weights (plus 'dab' [2])."""
        if self.core is not None:
            self.core.check(row_start)
        d_cur, d_tmp = self.dh
        d_cur.copy_(dY)
        dq, dk, dv, dm, dx = self.t
        for l in reversed(range(self.L)):
            ly, w, g = self.layers[l], weights[l], grads[l]
            # h2 = h1 + FFN(h1)
            pq.ffn_bwd(ly["ffn_desc"], d_cur, ly["h1"], w["Up"], w["Gate"], w["Down"], w["Wr"], ly["ffn_buf"], dx, g["W_up"],
                       g["W_gate"], g["W_down"], g["Up"], g["Gate"], g["Down"], g["Wr"], g["dab"])
            pq.glue_lincomb(d_tmp, [d_cur, dx], [1.0, 1.0])            # d h1
            # h1 = h + L_o(m)
            if self.core is not None:
                pq.glue_lincomb(d_cur, [d_tmp] + self._attention_backward(d_tmp, ly, w, g, row_start), [1.0, 1.0, 1.0, 1.0])
                continue
            pq.linear_bwd(self.lin_desc, d_tmp, ly["m"], w["Wo"], ly["lin_buf"]["o"], dm, g["Wo"], self.dab)
            pq.glue_lincomb(dm, [dm], [1 / 3])                         # d q = d k = d v = d m / 3
            for n, dxn in (("q", dq), ("k", dk), ("v", dv)):
                pq.linear_bwd(self.lin_desc, dm, ly["h"], w["W" + n], ly["lin_buf"][n], dxn, g["W" + n], self.dab)
            pq.glue_lincomb(d_cur, [d_tmp, dq, dk, dv], [1.0, 1.0, 1.0, 1.0])
        return d_cur


class CachedAttention:
    """One layer's attention over a cache of `n_pages` pages for `n_seqs` sequences (decoding: at most 16, the packed product's limit).

    Weights: latent Wq [d][d], Wk, Wv [n_kv_heads * d_head][d], Wo [d][d] (bf16, d = d_model), packed here once.  The caller keeps the pages:
    page_table [n_seqs, max_pages] int32 and lens [n_seqs] int32, which count the tokens of a call before it is made.  A prompt's
    buffers are made by the call; those of a decoding step are the object's, so that a step can be captured into a graph.  freqs [rot_dim / 2]
    (rope_freqs): rotary positions of queries and keys, turned before the keys are written."""

    freqs = None

    def __init__(self, weights, n_heads, n_kv_heads, n_pages, n_seqs, max_pages, page_tokens=64, kv_kind=pq.PQ_KV_INT8, max_len=0,
                 device="cuda", freqs=None, rot_dim=0, rope_layout=pq.PQ_ROPE_HALF, rope_scale=1.0):
        d = weights["Wq"].shape[1]
        if n_heads < 1 or n_kv_heads < 1 or d % n_heads or n_heads % n_kv_heads:
            raise pq.PQError(f"d_model={d} is a multiple of n_heads={n_heads}, and that of n_kv_heads={n_kv_heads}")
        for n in ("q", "k", "v", "o"):
            W, rows = weights["W" + n], d if n in "qo" else n_kv_heads * (d // n_heads)
            if W.shape != (rows, d) or not W.is_contiguous():
                raise pq.PQError(f"W{n} of shape {tuple(W.shape)}: a contiguous [{rows}, {d}] is wanted")
        dev, want = weights["Wq"].device, torch.device(device)
        if dev.type != "cuda" or want.type != "cuda" or want.index not in (None, dev.index) or any(weights["W" + n].device != dev for n in "kvo"):
            raise pq.PQError(f"the weights are on one GPU, that of device={device}")
        self.d, self.H, self.Hk, self.dh, self.B = d, n_heads, n_kv_heads, d // n_heads, n_seqs
        if freqs is not None:
            self.freqs = freqs
            self.turn = pq.make_rope_desc(n_heads, n_kv_heads, self.dh, n_seqs, rot_dim=rot_dim, layout=rope_layout, scale=rope_scale)
        with torch.cuda.device(dev):                                     # (whichever is current)
            self._build(weights, n_pages, n_seqs, max_pages, page_tokens, kv_kind, max_len, dev)

    def _build(self, weights, n_pages, n_seqs, max_pages, page_tokens, kv_kind, max_len, device):
        d, n_heads, n_kv_heads = self.d, self.H, self.Hk
        self.packed = {}
        for n in ("q", "k", "v", "o"):
            P, _, ml = pq.pack_sign(weights["W" + n])
            scale = ml[1:2].to(torch.float16).view(torch.int16)          # the one stored scale of a packed layer
            self.packed[n] = (weights["W" + n].shape[0], P, ml, pq.pack_retile64(P, d), scale)
        self.kv = pq.make_kv_desc(kv_kind, n_kv_heads, self.dh, page_tokens, n_pages, n_seqs, max_pages)
        self.attn = pq.make_attn_desc(self.kv, n_heads, max_len=max_len)
        self.cache = pq.kv_cache(self.kv, device)
        e = lambda n: torch.empty((n_seqs, n), dtype=torch.bfloat16, device=device)
        self.step = {n: e(p[0]) for n, p in self.packed.items()}
        self.step["a"] = e(d)
        self.decode = {n: pq.DecodeDesc(n_seqs, d, p[0], 0, 1, 1, 1, pq.PQ_PACKED_TILED64, 0.0) for n, p in self.packed.items()}
        self.decode_ws = {n: pq.decode_workspace(dd, device) for n, dd in self.decode.items()}
        self.attn_ws = pq.attn_decode_workspace(self.attn, device)

    def _check(self, x, T):
        if x.shape != (T, self.d) or x.dtype is not torch.bfloat16 or not x.is_contiguous() or x.get_device() != self.cache.get_device():
            raise pq.PQError(f"a tensor of shape {tuple(x.shape)}: a contiguous bf16 [{T}, {self.d}] on the cache's device is wanted")

    def _heads(self, x, heads):
        return x.view(x.shape[0], heads, self.dh)

    def _turn(self, q, k, lens, row_start):
        if self.freqs is not None:
            q, k = self._heads(q, self.H), self._heads(k, self.Hk)
            pq.rope(self.turn, q, k, self.freqs, q, k, row_start=row_start, lens=lens)

    def prompt(self, x, lens, page_table, row_start):
        """x [T, d] bf16: the last row_start[b + 1] - row_start[b] tokens of every sequence.  Returns [T, d]; rows of no sequence are undefined."""
        T = x.shape[0] if x.dim() else 0
        self._check(x, T)
        if T == 0:
            return torch.empty_like(x)
        if pq._current_device() != self.cache.get_device():
            with torch.cuda.device(self.cache.device):
                return self.prompt(x, lens, page_table, row_start)

        def linear(n, x):
            N, P, ml, _, _ = self.packed[n]
            desc = pq.make_desc(T, self.d, N, w_kind=pq.PQ_W_PACKED, alpha=0.0, beta=1.0)
            y = torch.empty((T, N), dtype=torch.bfloat16, device=x.device)
            return pq.linear_fwd(desc, x, P, y, pq.LinearBuffers(desc, x.device), mu_lambda=ml, save=False)
        q, k, v = linear("q", x), linear("k", x), linear("v", x)
        self._turn(q, k, lens, row_start)
        pq.kv_write(self.kv, self._heads(k, self.Hk), self._heads(v, self.Hk), self.cache, lens, page_table, row_start=row_start)
        a = torch.empty_like(q)
        pq.attn_prefill(self.attn, self._heads(q, self.H), self.cache, lens, page_table, row_start, self._heads(a, self.H))
        return pq.glue_lincomb(torch.empty_like(x), [x, linear("o", a)], [1.0, 1.0])

    def token(self, x, lens, page_table, out):
        """x [n_seqs, d] bf16: the newest token of every sequence, counted in lens already.  Writes out [n_seqs, d]."""
        s = self.step
        self._check(x, self.B)
        self._check(out, self.B)
        if pq._current_device() != self.cache.get_device():
            with torch.cuda.device(self.cache.device):
                return self.token(x, lens, page_table, out)

        def linear(n, x):
            _, _, _, tiled, scale = self.packed[n]
            return pq.decode_gemv(self.decode[n], x, tiled, scale, s[n], self.decode_ws[n])
        for n in ("q", "k", "v"):
            linear(n, x)
        self._turn(s["q"], s["k"], lens, None)
        pq.kv_write(self.kv, self._heads(s["k"], self.Hk), self._heads(s["v"], self.Hk), self.cache, lens, page_table)
        pq.attn_decode(self.attn, self._heads(s["q"], self.H), self.cache, lens, page_table, self._heads(s["a"], self.H), self.attn_ws)
        return pq.glue_lincomb(out, [x, linear("o", s["a"])], [1.0, 1.0])
