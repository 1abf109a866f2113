"""The cache, its attention and the packed projections around it run together: a prompt, then tokens one at a time, against the oracle's
projections and the attention's definition, and a captured step against the eager one."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as ao
from oracle import pquant_oracle as po
from paper_2602_22592_amd import binding as pq
from paper_2602_22592_amd import workloads as wl
from paper_2602_22592_amd.stack import CachedAttention

pytestmark = pytest.mark.gpu
t32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32).cuda()


def _linear(x, W):
    return ao.bf16(po.linear_fwd(x, W, 0.0, 1.0)["Y"])


def _oracle(x, W, H, Hk, int8):
    """The layer on whole sequences: every projection rounded to bf16, as it is stored."""
    d = x.shape[1]
    dh, G = d // H, H // Hk
    q, k, v = (_linear(x, W["W" + n]) for n in "qkv")
    k, v = (ao.stored(y.reshape(len(x), Hk, dh), int8) for y in (k, v))
    q = q.reshape(len(x), H, dh)
    a = np.zeros_like(q)
    for i in range(len(x)):
        for h in range(H):
            a[i, h] = ao.attention_row(q[i, h], k[:, h // G], v[:, h // G], ao.visible(len(x), i), dh ** -0.5)[0]
    return ao.bf16(x + _linear(ao.bf16(a.reshape(len(x), d)), W["Wo"]))


@pytest.mark.parametrize("kind,H,Hk", [(pq.PQ_KV_INT8, 8, 8), (pq.PQ_KV_INT8, 8, 2), (pq.PQ_KV_BF16, 4, 1)])
def test_prompt_then_tokens(kind, H, Hk):
    d, page, steps = 512, 16, 4
    dh = d // H
    prompt = [37, 5]
    full = [n + steps for n in prompt]
    rng = np.random.default_rng(11)
    W = {"W" + n: wl.normal(rng, (d if n in "qo" else Hk * dh, d), 0.06, True) for n in "qkvo"}
    xs = [wl.activations(rng, n, d, outlier_frac=0.01, outlier_scale=5.0, bf16=True) for n in full]
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda().bfloat16()
    layer = CachedAttention({n: dev(w) for n, w in W.items()}, H, Hk, n_pages=12, n_seqs=2, max_pages=4, page_tokens=page, kv_kind=kind, max_len=64)
    layer.cache.fill_(255)
    table, lens = t32([[7, 1, 9, -1], [3, -1, -1, -1]]), t32(prompt)
    out = layer.prompt(dev(np.concatenate([x[:n] for x, n in zip(xs, prompt)])), lens, table, t32([0, 37, 42]))
    got = [[out[:37].float().cpu().numpy()], [out[37:].float().cpu().numpy()]]
    x1, y1 = torch.empty((2, d), dtype=torch.bfloat16, device="cuda"), torch.empty((2, d), dtype=torch.bfloat16, device="cuda")
    graph = None
    for i in range(steps):
        x1.copy_(dev(np.stack([x[n + i] for x, n in zip(xs, prompt)])))
        lens.add_(1)
        if i == 0:
            layer.token(x1, lens, table, y1)
        elif i == 1:
            eager = layer.token(x1, lens, table, y1).clone()
            graph = torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph):
                layer.token(x1, lens, table, y1)
            y1.zero_()
            graph.replay()
            assert torch.equal(y1, eager)                      # the same token again, replayed: bit for bit
        else:
            graph.replay()
        torch.cuda.synchronize()
        for b in range(2):
            got[b].append(y1[b:b + 1].float().cpu().numpy())
    for b in range(2):
        want = _oracle(xs[b], W, H, Hk, kind == pq.PQ_KV_INT8)
        err = (np.abs(np.concatenate(got[b]) - want).max(1) / np.abs(want).max(1)).max()
        print(f"sequence {b}: {err:.2e}", flush=True)
        assert err <= 2e-2                                     # the bar of every bf16 output in this library, here row by row
