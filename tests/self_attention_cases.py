"""Packed sequences for the attention over the rows of a call: inputs on the GPU, the definition in fp64, and how far each output may be from it.

Tolerances count roundings.  u = 2^-8 is half a step of bf16, f = 2^-24 of fp32.  A score is a sum of d products in fp32, off by at most
(d + 2) f scale sum |q k|, and its exponential by that much relatively, with 2^-20 for exp2, its argument and lse (|s| log2 e < 64: 2^-24 of it is 2^-18 / 64).
p is rounded to bf16 (u), every sum of n terms in fp32 adds n f of the terms' absolute sum, an output is rounded once (u of itself)."""
import numpy as np
import torch

from oracle import attention_oracle as ao
from oracle import training_oracle as to
from paper_2602_22592_amd import binding as pq

U, F = 2.0 ** -8, 2.0 ** -24


class Packed:
    def __init__(self, rows, H, Hk, d, causal=True, window=0, scale=None, gap=0, before=0, behind=0, seed=0, size=1.0):
        self.rows, self.H, self.Hk, self.d, self.causal, self.window = list(rows), H, Hk, d, causal, window
        self.scale = d ** -0.5 if scale is None else scale
        self.before, self.T, self.gap = before, before + sum(rows) + behind, gap
        self.starts = before + np.concatenate([[0], np.cumsum(rows)]).astype(int)
        r = np.random.default_rng(seed)
        draw = lambda h: ao.bf16(r.standard_normal((self.T, h, d)) * size)
        self.q, self.k, self.v, self.do = draw(H), draw(Hk), draw(Hk), ao.bf16(r.standard_normal((self.T, H, d)))

    def gpu(self, x, gap=None):
        """bf16 on the GPU, rows `gap` elements apart from each other, NaN between them."""
        gap, (T, h, d) = self.gap if gap is None else gap, x.shape
        buf = torch.full((T, h * d + gap), float("nan"), dtype=torch.bfloat16, device="cuda")
        buf[:, :h * d] = torch.from_numpy(np.ascontiguousarray(x).reshape(T, h * d)).cuda().bfloat16()
        return buf[:, :h * d].unflatten(1, (h, d)) if gap else buf.view(T, h, d)

    def desc(self):
        return pq.make_self_attn_desc(self.H, self.Hk, self.d, len(self.rows), scale=self.scale, causal=self.causal, window=self.window)

    def row_start(self):
        return torch.tensor(self.starts, dtype=torch.int32).cuda()

    def inputs(self):
        return self.gpu(self.q), self.gpu(self.k), self.gpu(self.v)

    def outputs(self):
        """O and lse, filled with 7."""
        return (torch.full((self.T, self.H, self.d), 7.0, dtype=torch.bfloat16, device="cuda"),
                torch.full((self.T, self.H), 7.0, device="cuda"))

    def gradients(self):
        return [self.gpu(np.full((self.T, h, self.d), 7.0)) for h in (self.H, self.Hk, self.Hk)]

    def forward(self, dev=None):
        Q, K, V = dev or self.inputs()
        O, lse = self.outputs()
        pq.self_attn_fwd(self.desc(), Q, K, V, self.row_start(), O, lse)
        torch.cuda.synchronize()
        return O, lse

    def backward(self, O, lse, dev=None, pieces=None):
        Q, K, V = dev or self.inputs()
        out, desc = self.gradients(), self.desc()
        ws = pq.self_attn_bwd_workspace(desc, self.T)
        if pieces is not None:                               # a workspace with room for so many pieces of dK and dV, less than the call would take
            few = (self.T * self.H * 8 + 255) // 256 * 256 + 256 + pieces * self.T * self.Hk * 2 * self.d * 4
            assert few < ws.numel()
            ws = ws[:few]
        ws.fill_(255)
        pq.self_attn_bwd(desc, self.gpu(self.do, 0), Q, K, V, O, lse, self.row_start(), *out, ws)
        torch.cuda.synchronize()
        return out

    def each(self):
        """(sequence's rows, head, its key-value head, what is seen)"""
        for b, n in enumerate(self.rows):
            if n:
                seen = to.seen_by(n, self.causal, self.window)
                for h in range(self.H):
                    yield slice(self.starts[b], self.starts[b] + n), h, h * self.Hk // self.H, seen

    def others(self):
        """Rows of no sequence."""
        x = np.ones(self.T, bool)
        x[self.starts[0]:self.starts[-1]] = False
        return x

    def score_error(self, q, k, seen):
        """Relative error of exp(s - lse), row by row."""
        return (self.d + 2) * F * abs(self.scale) * np.where(seen, np.abs(q) @ np.abs(k).T, 0).max(1, keepdims=True) + 2.0 ** -18

    def check_forward(self, O, lse):
        O, lse = O.float().cpu().numpy(), lse.cpu().numpy()
        assert (O[self.others()] == 7).all() and (lse[self.others()] == 7).all()
        for here, h, hk, seen in self.each():
            q, k, v = (x[here, j].astype(np.float64) for x, j in ((self.q, h), (self.k, hk), (self.v, hk)))
            o, l, p = to.self_attention(q, k, v, seen, self.scale)
            e, a = self.score_error(q, k, seen), p @ np.abs(v)
            tol = U * np.abs(o) + (U + 2 * e + 2 * len(q) * F) * a * (1 + U)
            bad = ~(np.abs(O[here, h] - o) <= tol)
            assert not bad.any(), (here, h, np.argwhere(bad)[:4], np.abs(O[here, h] - o).max())
            assert (np.abs(lse[here, h] - l) <= e[:, 0] + len(q) * F + 2 * F * np.abs(l)).all(), (here, h)

    def check_backward(self, O, lse, out, operand=U):
        """Against the formula in 64 bits on the lse that the call was given (O is where delta begins, not what it is).  `operand`: what p and dS are off
        by, relative, as operands of the second products (U; U U where they are sums of two bf16 numbers, but for p in m)."""
        dQ, dK, dV = (x.float().cpu().numpy() for x in out)
        for x in (dQ, dK, dV):
            assert (x[self.others()] == 7).all()
        O, lse = O.float().cpu().numpy(), lse.cpu().numpy()
        want = {n: (np.zeros(x.shape), np.zeros(x.shape)) for n, x in (("dQ", self.q), ("dK", self.k), ("dV", self.v))}

        def add(name, here, head, value, error):
            want[name][0][here, head] += value
            want[name][1][here, head] += error
        for here, h, hk, seen in self.each():
            q, k, v, do, o = (x[here, j].astype(np.float64) for x, j in ((self.q, h), (self.k, hk), (self.v, hk), (self.do, h), (O, h)))
            dq, dk, dv, p, ds = to.self_attention_gradients(do, q, k, v, lse[here, h], seen, self.scale)
            e = self.score_error(q, k, seen)
            # dP - delta: a sum of d products in fp32, and delta, a sum of as many products as the row sees, each with its p off by e and n f
            slopes = np.abs(do) @ np.abs(v).T
            diff = (self.d + 2) * F * slopes + ((self.d + 2 + len(q)) * F + 2 * e) * (p * slopes).sum(1, keepdims=True)
            diff = np.where(seen & (seen.sum(1) > 1)[:, None], diff, 0)
            # dQ = sum_j D_j k_j - (sum_j D_j) m, with D the rounded dS that are formed with dO . O (off by p `rest`, from O's rounding) and m = sum p~ k,
            # p~ the rounded p.  D_j = x_j + r_j, |r_j| <= U |x_j|, |x_j| <= |dS_j| + p_j rest.  The x_j alone give dQ exactly (sum x_j (k_j - m) with
            # m exact), so the error is sum r_j (k_j - m), at most U sum |x_j| (|k_j| + |m|), and (sum D_j) (m~ - m), at most (rest + U sum |x_j|) U sum p |k|.
            many = seen.sum(1, keepdims=True) > 1
            rest = np.abs((do * o).sum(1, keepdims=True) - (p * (do @ v.T)).sum(1, keepdims=True)) * many
            dse = (np.abs(ds) * (operand + e) + p * diff * (1 + e)) * (1 + U)
            dsq = dse + p * rest * (operand + 2 * e)
            x = (np.abs(ds) + p * rest) * many
            mean = operand * x.sum(1, keepdims=True) * np.abs(p @ k) + (rest + operand * x.sum(1, keepdims=True)) * U * (p @ np.abs(k))
            n = len(q) * self.H // self.Hk + 4
            add("dQ", here, h, dq, abs(self.scale) * (dsq @ np.abs(k) + mean + n * F * np.abs(ds) @ np.abs(k)))
            add("dK", here, hk, dk, abs(self.scale) * (dse.T @ np.abs(q) + n * F * np.abs(ds).T @ np.abs(q)))
            add("dV", here, hk, dv, (p * (operand + e + n * F)).T @ np.abs(do))
        mine = ~self.others()
        for name, x in (("dQ", dQ), ("dK", dK), ("dV", dV)):
            value, error = want[name]
            bad = ~(np.abs(x - value) <= error * (1 + U) + U * np.abs(value) + 1e-37)
            bad[~mine] = False
            assert not bad.any(), (name, np.argwhere(bad)[:4], x[bad][:4], value[bad][:4], error[bad][:4])
