"""Ragged batches over a paged key-value cache for the tests: sequences, their pages, keys and values, and what the oracle makes of them."""
import numpy as np
import torch

from oracle import attention_oracle as ao
from paper_2602_22592_amd import binding as pq


def padded(d):
    return -(-d // 32) * 32


class Paged:
    """Sequences of `lens` tokens, all of whose keys and values are written; pages scattered over the pool, the pool full of NaN before."""

    def __init__(self, kind, lens, Hk, d, page, seed=0, spare=2, key_scale=1.0, poison=255, n_pages=None):
        rng = self.rng = np.random.default_rng(seed)
        self.kind, self.lens, self.Hk, self.d, self.page, self.B = kind, list(lens), Hk, d, page, len(lens)
        need = [-(-n // page) for n in lens]
        self.n_pages = n_pages or sum(need) + spare
        self.max_pages = max(need + [1]) + 1
        order = rng.permutation(self.n_pages)
        self.table = np.full((self.B, self.max_pages), -1, np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.K = [ao.bf16(rng.standard_normal((n, Hk, d)) * key_scale) for n in lens]
        self.V = [ao.bf16(rng.standard_normal((n, Hk, d))) for n in lens]
        self.poison = poison

    @property
    def int8(self):
        return self.kind == pq.PQ_KV_INT8

    def desc(self):
        return pq.make_kv_desc(self.kind, self.Hk, self.d, self.page, self.n_pages, self.B, self.max_pages)

    def device(self):
        """The cache, written through pq_kv_write, with lens and page table, on the GPU."""
        desc = self.desc()
        cache = pq.kv_cache(desc)
        cache.fill_(self.poison)
        lens, table = torch.tensor(self.lens, dtype=torch.int32).cuda(), torch.from_numpy(self.table).cuda()
        starts = torch.from_numpy(np.concatenate([[0], np.cumsum(self.lens)]).astype(np.int32)).cuda()
        K, V = (torch.from_numpy(np.concatenate(x + [np.zeros((0, self.Hk, self.d), np.float32)])).float().cuda() for x in (self.K, self.V))
        pq.kv_write(desc, K, V, cache, lens, table, row_start=starts)
        return cache, lens, table

    def stored(self, b):
        return ao.stored(self.K[b], self.int8), ao.stored(self.V[b], self.int8)


def expected(case, q, rows, scale, causal=True, window=0, present=None, p_bits=0, fixed_point=False):
    """Oracle outputs of the last rows[b] tokens of every sequence and elementwise bounds: (o, lse, tol_o, tol_lse).

    q [T][H][d].  present: per sequence, which tokens have a page.  p_bits > 0: a probability is rounded to that many significant bits
    (relative error 2^-p_bits each).  The bounds count: the rounding of o to bf16 (2^-8), fp32 sums of n terms (n 2^-24 each of a score,
    of the sum of the probabilities and of the weighted values), exponentials (2^-21), and, for `fixed_point`, queries and weighted
    probabilities held as 24-bit numbers relative to their largest (2^-22 of it per element, 127 codes at most)."""
    H = q.shape[1]
    G, d = H // case.Hk, case.d
    out, t = [], 0
    for b, n in enumerate(rows):
        K, V = case.stored(b)
        L = len(K)
        for i in range(n):
            pos = L - n + i
            seen = ao.visible(L, pos, causal, window)
            if present is not None:
                seen &= present[b]
            for h in range(H):
                k, v = K[:, h // G], V[:, h // G]
                o, lse, a = ao.attention_row(q[t, h], k, v, seen, scale)
                ns = int(seen.sum())
                if ns:
                    dots = np.abs(k[seen].astype(np.float64)) @ np.abs(q[t, h]).astype(np.float64)
                    ds = abs(scale) * dots.max() * (d + 4) * 2.0 ** -24
                    if fixed_point:
                        ds += abs(scale) * 2.0 ** -22 * np.abs(q[t, h]).max() * np.abs(k[seen].astype(np.float64)).sum(-1).max()
                    rel = 2 * ds + 2.0 ** -20 + (ns + 64) * 2.0 ** -23 + (2.0 ** -p_bits if p_bits else 0.0)
                    tol = 2.0 ** -8 * np.abs(o) + rel * a * 1.01
                    if fixed_point:
                        tol = tol + ns * 2.0 ** -22 * a.max()
                    tl = ds + 2.0 ** -20 + (ns + 64) * 2.0 ** -24 + 2.0 ** -22 * abs(lse)
                else:
                    tol, tl = np.zeros(d), 0.0
                out.append((o, lse, tol, tl))
            t += 1
    o, lse, tol, tl = (np.array([x[j] for x in out]) for j in range(4))
    T = sum(rows)
    return o.reshape(T, H, d), lse.reshape(T, H), tol.reshape(T, H, d), tl.reshape(T, H)


def check(O, lse, ref, name=""):
    o, l, tol, tl = ref
    got, gl = O.float().cpu().numpy().reshape(o.shape), lse.cpu().numpy().reshape(l.shape)
    empty = np.isneginf(l)
    assert np.array_equal(np.isneginf(gl), empty), name
    assert np.isfinite(got).all(), name
    assert (got[empty] == 0).all(), name
    err = np.abs(got - o)
    worst = float((err / np.maximum(tol, 1e-30))[~empty].max()) if (~empty).any() else 0.0
    lerr = float((np.abs(gl[~empty] - l[~empty]) / tl[~empty]).max()) if (~empty).any() else 0.0
    print(f"{name}: error over bound: o {worst:.2f}, lse {lerr:.2f}", flush=True)
    assert worst <= 1.0 and lerr <= 1.0, (name, worst, lerr)
