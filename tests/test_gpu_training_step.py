"""Rotary positions, attention with its gradient and the optimizer run together, as the layer stack and the cached layer call them."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as ao
from oracle import pquant_oracle as po
from oracle import training_oracle as to
from paper_2602_22592_amd import binding as pq
from paper_2602_22592_amd import workloads as wl
from paper_2602_22592_amd.stack import AttentionCore, CachedAttention, Stack
from parity_metrics import relerr

pytestmark = pytest.mark.gpu
t32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32).cuda()
dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda().to(torch.bfloat16)
host = lambda x: x.float().cpu().numpy()
NAMES = ("Wq", "Wk", "Wv", "Wo", "W_up", "W_gate", "W_down", "Up", "Gate", "Down", "Wr")


def _linear(x, W):
    return po.linear_fwd(x, W, 0.0, 1.0)


def _core_oracle(q, k, v, rows, H, Hk, freqs):
    """Per sequence: turned q and k as they are stored, output and lse."""
    dh = q.shape[1] // H
    out = []
    for b in range(len(rows) - 1):
        here = slice(rows[b], rows[b + 1])
        n = rows[b + 1] - rows[b]
        qt, kt = (ao.bf16(to.rope(x[here].reshape(n, h, dh), freqs, np.arange(n), "half")) for x, h in ((q, H), (k, Hk)))
        out.append((here, qt, kt, v[here].reshape(n, Hk, dh)))
    return out


def test_a_layer_with_attention_against_the_oracle():
    """One layer's forward pass and gradients.  2e-2 in the max-norm, the bar of bf16 outputs behind chained projections."""
    T, D, F, E, r, H, Hk = 128, 128, 96, 2, 8, 4, 2
    rows = [0, 50, 120]                                              # (the last 8 rows are no sequence's)
    c = wl.stack_case(5, 1, T, D, F, E, r, vocab=100)
    w = dict(c["layers"][0])
    w["Wk"], w["Wv"] = w["Wk"][:Hk * D // H], w["Wv"][:Hk * D // H]
    weights = [{n: dev(w[n]) for n in NAMES}]
    grads = [dict({n: torch.empty(w[n].shape, dtype=torch.float32, device="cuda") for n in NAMES}, dab=torch.empty(2, device="cuda"))]
    freqs = pq.rope_freqs(D // H)
    core = AttentionCore(T, H, Hk, D // H, 2, freqs=freqs)
    st = Stack(1, T, D, F, E, r, 1, [w["alpha"]], [w["beta"]], core=core)
    x = c["table"][c["ids"]]
    out = host(st.forward(dev(x), weights, t32(rows)))
    dx = host(st.backward(dev(c["dY"]), weights, grads, t32(rows)))

    fq, fk, fv = (_linear(x, w["W" + n]) for n in "qkv")
    q, k, v = (ao.bf16(f["Y"]) for f in (fq, fk, fv))
    a = np.zeros((T, D))
    parts = _core_oracle(q, k, v, rows, H, Hk, freqs.cpu().numpy())
    dh, G = D // H, H // Hk
    lse = {}
    for here, qt, kt, vv in parts:
        seen = to.seen_by(len(qt))
        for h in range(H):
            o, lse[here.start, h], _ = to.self_attention(qt[:, h], kt[:, h // G], vv[:, h // G], seen, dh ** -0.5)
            a[here, h * dh:(h + 1) * dh] = o
    a = ao.bf16(a)
    assert relerr(host(st.layers[0]["core"]["o"]).reshape(T, D), a) <= 2e-2
    fo = _linear(a, w["Wo"])
    h1 = ao.bf16(x + ao.bf16(fo["Y"]))
    assert relerr(host(st.layers[0]["h1"]), h1) <= 2e-2
    # the attention half's gradients, from the gradient that reached it
    d_tmp = host(st.dh[1])
    go = po.linear_bwd(d_tmp, a, w["Wo"], 0.0, 1.0, fo)
    dm = ao.bf16(go["dX"])
    dq, dk, dv = np.zeros((T, D)), np.zeros((T, Hk * dh)), np.zeros((T, Hk * dh))
    for here, qt, kt, vv in parts:
        n = len(qt)
        g = [np.zeros((n, h, dh)) for h in (H, Hk, Hk)]
        for h in range(H):
            one = to.self_attention_gradients(dm[here, h * dh:(h + 1) * dh], qt[:, h], kt[:, h // G], vv[:, h // G], lse[here.start, h], to.seen_by(n), dh ** -0.5)
            g[0][:, h] = one[0]
            g[1][:, h // G] += one[1]
            g[2][:, h // G] += one[2]
        back = lambda x: to.rope(x, freqs.cpu().numpy(), np.arange(n), "half", inverse=True)
        dq[here], dk[here], dv[here] = back(g[0]).reshape(n, -1), back(g[1]).reshape(n, -1), g[2].reshape(n, -1)
    errs = {"dq": relerr(host(st.dq), dq), "dk": relerr(host(st.dkv[0]), dk), "dv": relerr(host(st.dkv[1]), dv)}
    total = d_tmp.astype(np.float64)
    for n, dy, f in (("q", dq, fq), ("k", dk, fk), ("v", dv, fv)):
        b = po.linear_bwd(ao.bf16(dy), x, w["W" + n], 0.0, 1.0, f)
        errs["W" + n] = relerr(grads[0]["W" + n].cpu().numpy(), b["dW"])
        total = total + b["dX"]
    errs["dx"] = relerr(dx, total)
    assert np.isfinite(out).all() and max(errs.values()) <= 2e-2, errs


def test_training_steps_with_the_optimizer():
    """Two layers: forward, backward, the step; the weights move as the formula on the gradients says, and the next forward uses them."""
    T, D, F, E, r, H, Hk = 96, 64, 96, 2, 8, 2, 1
    c = wl.stack_case(9, 2, T, D, F, E, r, vocab=100)
    layers = [dict(w, Wk=w["Wk"][:32], Wv=w["Wv"][:32]) for w in c["layers"]]
    weights = [{n: dev(w[n]) for n in NAMES} for w in layers]
    grads = [dict({n: torch.empty(w[n].shape, dtype=torch.float32, device="cuda") for n in NAMES}, dab=torch.empty(2, device="cuda")) for w in layers]
    core = AttentionCore(T, H, Hk, 32, 3, freqs=pq.rope_freqs(16), rot_dim=16, layout=pq.PQ_ROPE_PAIRS, window=20)
    st = Stack(2, T, D, F, E, r, 1, [w["alpha"] for w in layers], [w["beta"] for w in layers], core=core)
    opt = st.optimizer(weights, grads, masters=True, state=pq.PQ_STATE_8BIT, beta1=0.9, beta2=0.95)
    rows, x, dY = t32([0, 40, 41, 96]), dev(c["table"][c["ids"]]), dev(c["dY"])
    before = st.forward(x, weights, rows).clone()
    for step in (1, 2):
        st.forward(x, weights, rows)
        st.backward(dY, weights, grads, rows)
        old = [m.clone() for m in opt.masters]
        m0 = [pq_state(opt, i) for i in range(len(old))]
        pq.adamw_step(opt, pq.adamw_scalars(opt, step, 1e-3, 0.1))
        for i, (m, r0) in enumerate(m0):
            g = opt.grads[i].double().view(-1)
            m1, v1 = 0.9 * m + 0.1 * g, 0.95 * r0 * r0 + 0.05 * g * g
            want = old[i].double().view(-1) * (1 - 1e-4) - 1e-3 / (1 - 0.9 ** step) * m1 / ((v1 / (1 - 0.95 ** step)).sqrt() + 1e-8)
            moved = (want - old[i].double().view(-1)).abs().max()
            assert torch.isfinite(want).all() and (opt.masters[i].double().view(-1) - want).abs().max() <= 1e-5 * moved + 1e-7
            assert torch.equal(opt.params[i], opt.masters[i].bfloat16())
    assert opt.params[0].data_ptr() == weights[0]["Wq"].data_ptr()
    after = st.forward(x, weights, rows)
    assert torch.isfinite(after).all() and not torch.equal(after, before)


def pq_state(opt, i):
    """(m, r) of one tensor's 8-bit states, in 64 bits."""
    n, steps = opt.m[i].numel(), opt.steps[i].double().repeat_interleave(256, 0)
    q, u = opt.m[i].double().view(-1), opt.v[i].double().view(-1)
    return q * q.abs() * steps[:n, 0], u * u * steps[:n, 1]


@pytest.mark.parametrize("kind", [pq.PQ_KV_INT8, pq.PQ_KV_BF16])
def test_cached_layer_with_positions(kind):
    """A prompt, then tokens one at a time (captured), against whole sequences: positions go on where the prompt ended."""
    d, H, Hk, page, steps = 256, 4, 2, 16, 3
    dh = d // H
    prompt = [21, 4]
    rng = np.random.default_rng(4)
    W = {"W" + n: wl.normal(rng, (d if n in "qo" else Hk * dh, d), 0.06, True) for n in "qkvo"}
    xs = [wl.activations(rng, n + steps, d, bf16=True) for n in prompt]
    freqs = pq.rope_freqs(dh, factor=2.0)
    layer = CachedAttention({n: dev(w) for n, w in W.items()}, H, Hk, n_pages=8, n_seqs=2, max_pages=4, page_tokens=page, kv_kind=kind, max_len=64,
                            freqs=freqs)
    table, lens = t32([[7, 1, -1, -1], [3, -1, -1, -1]]), t32(prompt)
    out = layer.prompt(dev(np.concatenate([x[:n] for x, n in zip(xs, prompt)])), lens, table, t32([0, 21, 25]))
    got = [[host(out[:21])], [host(out[21:])]]
    x1, y1 = (torch.empty((2, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for i in range(steps):
        x1.copy_(dev(np.stack([x[n + i] for x, n in zip(xs, prompt)])))
        lens.add_(1)
        if i == 0:
            layer.token(x1, lens, table, y1)
        elif i == 1:
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                layer.token(x1, lens, table, y1)
            graph.replay()
        else:
            graph.replay()
        torch.cuda.synchronize()
        for b in range(2):
            got[b].append(host(y1[b:b + 1]))
    for b, x in enumerate(xs):
        n = len(x)
        q, k, v = (ao.bf16(_linear(x, W["W" + m])["Y"]) for m in "qkv")
        (_, qt, kt, vv), = _core_oracle(q, k, v, [0, n], H, Hk, freqs.cpu().numpy())
        kt, vv = (ao.stored(y, kind == pq.PQ_KV_INT8) for y in (kt, vv))
        a = np.zeros((n, H, dh))
        for h in range(H):
            a[:, h] = to.self_attention(qt[:, h], kt[:, h * Hk // H], vv[:, h * Hk // H], to.seen_by(n), dh ** -0.5)[0]
        want = ao.bf16(x + ao.bf16(_linear(ao.bf16(a.reshape(n, d)), W["Wo"])["Y"]))
        assert (np.abs(np.concatenate(got[b]) - want).max(1) / np.abs(want).max(1)).max() <= 2e-2
