"""Drivers that chain the library's calls into layers.

Stack: a stack of transformer-shaped layers made of pQuant linears only (no attention core, no norms):

    per layer:  q,k,v = L_q(h), L_k(h), L_v(h)      pure 1-bit linears (Sec. 3.1: the MHA projections)
                m = (q + k + v) / 3                 stand-in for the attention core (glue)
                h1 = h + L_o(m)                     residual (glue)
                h2 = h1 + FFN(h1)                   decoupled FFN with routed experts (Sec. 3.2, 3.3)

It exists to time the linears of a 24-layer 1.3B-shaped model end to end.

CachedAttention: the attention half of a layer at inference, on packed weights and a paged key-value cache:

    q, k, v = L_q(x), L_k(x), L_v(x)                pure 1-bit linears (Sec. 3.1)
    out = x + L_o(attention(q, cache + k, v))       prompts row by row, then one token of every sequence at a time

This module only sequences C-ABI calls (pq_linear_*, pq_ffn_*, pq_decode_gemv, pq_kv_*, pq_attn_*, pq_glue_*); PyTorch provides the
device buffers.
"""
from __future__ import annotations

import torch

from . import binding as pq


class Stack:
    def __init__(self, n_layers, tokens, d_model, d_ffn, n_experts, hp_rank, top_k, alphas, betas, device="cuda"):
        self.L, self.T, self.D, self.F = n_layers, tokens, d_model, d_ffn
        self.E, self.r, self.k = n_experts, hp_rank, top_k
        bf = torch.bfloat16
        self.lin_desc = pq.make_desc(tokens, d_model, d_model, hp_rank=0, io_dtype=pq.PQ_BF16, alpha=0.0, beta=1.0)
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

    def forward(self, h0, weights):
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

    def backward(self, dY, weights, grads):
        """grads: per-layer dict of fp32 tensors shaped like the weights (plus 'dab' [2])."""
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
    buffers are made by the call; those of a decoding step are the object's, so that a step can be captured into a graph."""

    def __init__(self, weights, n_heads, n_kv_heads, n_pages, n_seqs, max_pages, page_tokens=64, kv_kind=pq.PQ_KV_INT8, max_len=0,
                 device="cuda"):
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
        pq.kv_write(self.kv, self._heads(s["k"], self.Hk), self._heads(s["v"], self.Hk), self.cache, lens, page_table)
        pq.attn_decode(self.attn, self._heads(s["q"], self.H), self.cache, lens, page_table, self._heads(s["a"], self.H), self.attn_ws)
        return pq.glue_lincomb(out, [x, linear("o", s["a"])], [1.0, 1.0])
