"""The AdamW step over many tensors: 8-bit codes and steps are equal to the oracle's, moments and weights within the roundings of their formula."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as ao
from oracle import training_oracle as to
from paper_2602_22592_amd import binding as pq

pytestmark = pytest.mark.gpu
F = 2.0 ** -24
H = dict(lr=1e-3, weight_decay=0.1)
B1, B2, EPS = 0.9, 0.95, 1e-8
SIZES = {"one": [1], "three": [3, 4, 5], "blocks": [256, 255, 257, 512, 1000], "mixed": [1, 70001, 33, 4096, 4097, 1024, 1025, 2], "large": [5000001, 7]}
F32 = np.float32


def make(sizes, param, grad, state, masters, seed=0):
    r = np.random.default_rng(seed)
    p = [(r.standard_normal(n) * 0.02).astype(F32) for n in sizes]
    g = [(r.standard_normal(n) * np.exp(1.5 * r.standard_normal(n)) * 1e-3).astype(F32) for n in sizes]
    m = [(r.standard_normal(n) * 3e-4).astype(F32) for n in sizes]
    v = [((r.standard_normal(n) * np.exp(r.standard_normal(n)) * 1e-3) ** 2).astype(F32) for n in sizes]
    s = dict(sizes=sizes, masters=None, steps=None, eight=state == "8bit")
    if masters:
        s["masters"] = [x.copy() for x in p]
    s["p"] = [ao.bf16(x) for x in p] if param is torch.bfloat16 else p
    s["g"] = [ao.bf16(x) for x in g] if grad is torch.bfloat16 else g
    if s["eight"]:
        s["m"], s["v"], s["steps"] = [], [], []
        for x, y in zip(m, v):
            (qm, sm), (qr, sr) = to.nearest_codes(to.blocks(x), 127), to.nearest_codes(np.sqrt(to.blocks(y)), 255)
            qm = np.where(to.blocks(x) < 0, -qm, qm)
            s["m"].append(qm.astype(np.int8).reshape(-1)[:len(x)])
            s["v"].append(qr.astype(np.uint8).reshape(-1)[:len(x)])
            s["steps"].append(np.concatenate([sm, sr], 1))
    else:
        s["m"], s["v"] = m, v
    cuda = lambda xs, dtype: xs and [torch.from_numpy(x).cuda().to(dtype) for x in xs]
    as_is = lambda xs: xs and [torch.from_numpy(x).cuda() for x in xs]
    values = [[torch.zeros(n, device="cuda") for n in sizes] for _ in range(2)] if s["eight"] else [None, None]
    s["t"] = pq.AdamWTensors(cuda(s["p"], param), cuda(s["g"], grad), as_is(s["m"]), as_is(s["v"]), steps=as_is(s["steps"]), masters=as_is(s["masters"]),
                             m_values=values[0], v_values=values[1], beta1=B1, beta2=B2, eps=EPS)
    return s


def oracle_step(s, step, gscale):
    """Advances the oracle's states by one step; the weights with how far they may be off."""
    out = []
    for i in range(len(s["sizes"])):
        n = s["sizes"][i]
        if s["eight"]:
            m0, r0 = to.decode(to.blocks(s["m"][i]), to.blocks(s["v"][i]), s["steps"][i])
            m, v, r = to.moments(to.blocks(s["g"][i]), m0, r0 * r0, B1, B2, gscale)
            (qm, sm), (qr, sr) = to.nearest_codes(m, 127), to.nearest_codes(r, 255)
            qm, qr = np.where(m < 0, -qm, qm), np.where(r > 0, np.maximum(qr, 1), qr)
            s["m"][i], s["v"][i] = qm.astype(np.int8).reshape(-1)[:n], qr.astype(np.uint8).reshape(-1)[:n]
            s["steps"][i] = np.concatenate([sm, sr], 1).astype(F32)
            m, v = m.reshape(-1)[:n], v.reshape(-1)[:n]
        else:
            m, v, _ = to.moments(s["g"][i], s["m"][i], s["v"][i], B1, B2, gscale)
            s["m"][i], s["v"][i] = m, v
        w = (s["masters"] or s["p"])[i]
        new = to.adamw_weight(w, m, v, step, H["lr"], H["weight_decay"], B1, B2, EPS)
        # one product, a quotient of three roundings each above and below (its factors rounded), their difference
        update = np.abs(new - w.astype(np.float64) * (1 - H["lr"] * H["weight_decay"]))
        out.append((new, F * (3 * np.abs(w) + 8 * update + np.abs(new))))
    return out


@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("state", ["f32", "8bit"])
@pytest.mark.parametrize("kind", ["f32", "bf16", "masters", "bf16_grads"])
def test_steps_against_the_definition(sizes, state, kind):
    param = torch.float32 if kind in ("f32", "bf16_grads") else torch.bfloat16
    grad = torch.bfloat16 if kind in ("bf16_grads", "masters") else torch.float32
    s = make(SIZES[sizes], param, grad, state, kind == "masters", seed=len(sizes))
    t = s["t"]
    for step, gscale in ((1, 1.0), (2, 0.37), (1000, 2.0)):
        pq.adamw_step(t, pq.adamw_scalars(t, step, H["lr"], H["weight_decay"], gscale))
        if s["eight"]:
            pq.adamw_read(t)
        for i, (w, tol) in enumerate(oracle_step(s, step, gscale)):
            got = lambda ts: ts[i].float().cpu().numpy()
            assert np.array_equal(t.m[i].cpu().numpy(), s["m"][i]) and np.array_equal(t.v[i].cpu().numpy(), s["v"][i])   # (bit for bit, fp32 ones too)
            if s["eight"]:
                assert np.array_equal(t.steps[i].cpu().numpy(), s["steps"][i])
                m, r = to.decode(to.blocks(s["m"][i]), to.blocks(s["v"][i]), s["steps"][i])
                n = s["sizes"][i]
                assert np.array_equal(got(t.m_values), m.reshape(-1)[:n]) and np.array_equal(got(t.v_values), (r * r).reshape(-1)[:n])
            if s["masters"]:
                assert (np.abs(got(t.masters) - w) <= tol).all()
                assert np.array_equal(got(t.params), ao.bf16(got(t.masters)))
                s["masters"][i] = got(t.masters)                     # (the next step from what is there)
            else:
                assert (np.abs(got(t.params) - w) <= tol + (2.0 ** -8 * np.abs(w) if param is torch.bfloat16 else 0)).all()
            s["p"][i] = got(t.params)


def test_border_codes():
    """Quotients at and next to every border between two codes: a block whose largest value gives the step 1 exactly, beta1 = 0, one gradient."""
    k = np.arange(127)
    border = ((k + 0.5) ** 2).astype(F32)
    x = np.concatenate([[127.0 ** 2], border, np.nextafter(border, F32(0)), np.nextafter(border, F32(1e9)), -border, [0.0, 1.0, 4.0]]).astype(F32)
    x = to.blocks(x).copy()
    x[:, 0] = F32(127.0 ** 2)                                        # (every block has the step fl(127^2 fl(1 / 127^2)))
    x = x.reshape(-1)
    p = [torch.zeros(len(x), device="cuda")]
    t = pq.AdamWTensors(p, [torch.from_numpy(x).cuda()], beta1=0.0, beta2=0.0, state=pq.PQ_STATE_8BIT)
    pq.adamw_step(t, pq.adamw_scalars(t, 1, 1e-3))
    code, step = to.nearest_codes(to.blocks(x), 127)
    assert np.array_equal(t.m[0].cpu().numpy(), np.where(x < 0, -code.reshape(-1), code.reshape(-1)).astype(np.int8))
    root, rstep = to.nearest_codes(to.blocks(np.sqrt((x.astype(np.float64) * x).astype(F32).astype(np.float64)).astype(F32)), 255)
    assert np.array_equal(t.v[0].cpu().numpy(), np.where(x != 0, np.maximum(root.reshape(-1), 1), root.reshape(-1)).astype(np.uint8))
    assert np.array_equal(t.steps[0].cpu().numpy(), np.concatenate([step, rstep], 1))


def test_blocks_with_infinities_and_nan_do_not_reach_others():
    n = 1024
    g = torch.randn(n, generator=torch.Generator().manual_seed(0)) * 1e-3
    g[300], g[600] = float("nan"), float("inf")
    p = torch.ones(n)
    values = [[torch.zeros(n, device="cuda")] for _ in range(2)]
    t = pq.AdamWTensors([p.cuda()], [g.cuda()], state=pq.PQ_STATE_8BIT, m_values=values[0], v_values=values[1])
    pq.adamw_step(t, pq.adamw_scalars(t, 1, 1e-3))
    pq.adamw_read(t)
    m, v, w = t.m_values[0].cpu(), t.v_values[0].cpu(), t.params[0].cpu()
    assert torch.isfinite(m[:256]).all() and torch.isfinite(m[768:]).all() and torch.isfinite(v[:256]).all() and torch.isfinite(v[768:]).all()
    assert m[256:768].isnan().all() and v[256:768].isnan().all()
    assert w.isnan().nonzero().view(-1).tolist() == [300, 600]


def test_all_zero_states_and_gradients():
    t = pq.AdamWTensors([torch.ones(300, device="cuda")], [torch.zeros(300, device="cuda")], state=pq.PQ_STATE_8BIT)
    pq.adamw_step(t, pq.adamw_scalars(t, 1, 1e-3, 0.5))
    assert (t.m[0] == 0).all() and (t.v[0] == 0).all()
    assert (t.params[0] == torch.tensor(1.0 - 1e-3 * 0.5, dtype=torch.float64).float().item()).all()


def test_neighbours_are_left_alone():
    """Tensors that are parts of one buffer, with elements between them that belong to nobody."""
    buf = {n: torch.full((4096,), 7, dtype=d, device="cuda") for n, d in (("p", torch.bfloat16), ("g", torch.float32), ("m", torch.int8), ("v", torch.uint8))}
    at = [(0, 259), (512, 1), (1024, 1030)]
    cut = lambda x: [x[a:a + n] for a, n in at]
    steps = [torch.ones((-(-n // 256), 2), device="cuda") * 1e-6 for _, n in at]
    t = pq.AdamWTensors(cut(buf["p"]), cut(buf["g"]), cut(buf["m"]), cut(buf["v"]), steps=steps)
    pq.adamw_step(t, pq.adamw_scalars(t, 3, 1e-3))
    inside = torch.zeros(4096, dtype=torch.bool)
    for a, n in at:
        inside[a:a + n] = True
    # (a weight of 7 moves by about lr = 1e-3, less than half a step of bf16 there, 2^-6: it stays 7, the states do not)
    for n in "pmv":
        assert (buf[n].cpu()[~inside] == 7).all() and (n == "p" or (buf[n].cpu()[inside] != 7).any()), n


def test_a_captured_step_is_replayed_with_other_scalars_and_gradients():
    s, e = (make([1000, 33], torch.float32, torch.float32, "8bit", False) for _ in range(2))
    t, u = s["t"], e["t"]
    scalars = pq.adamw_scalars(t, 1, 1e-3)
    g = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.graph(g, stream=side):
        pq.adamw_step(t, scalars)
    for step in (1, 2, 3, 4):
        pq.adamw_scalars(t, step, 1e-3 / step, 0.1, out=scalars)
        for x, y in zip(t.grads, u.grads):
            y.mul_(1.5)
            x.copy_(y)
        g.replay()
        pq.adamw_step(u, pq.adamw_scalars(u, step, 1e-3 / step, 0.1))
        torch.cuda.synchronize()
        for a, b in zip(t.params + t.m + t.v + t.steps, u.params + u.m + u.v + u.steps):
            assert torch.equal(a, b)


def test_tensors_that_share_memory_are_refused():
    x = torch.zeros(2048, device="cuda")
    new = lambda n=256: torch.zeros(n, device="cuda")
    with pytest.raises(pq.PQError, match="overlap"):
        pq.AdamWTensors([x[:256], x[:256]], [new(), new()])
    with pytest.raises(pq.PQError, match="overlap"):
        pq.AdamWTensors([x[128:384], new(4)], [x[:256], new(4)])
    with pytest.raises(pq.PQError, match="overlap"):                  # (behind a shorter gradient inside of a longer one)
        pq.AdamWTensors([new(1024), new(16), x[512:768]], [x[:1024], x[16:32], new()])
    with pytest.raises(pq.PQError, match="overlap"):
        pq.AdamWTensors([x[:256]], [new()], m=[x[252:508]], v=[new()])
    t = pq.AdamWTensors([new(), new()], [x[:256], x[:256]])            # one gradient for two tensors
    pq.adamw_step(t, pq.adamw_scalars(t, 1, 1e-3))


def test_empty_tensors_and_another_stream():
    p = [torch.ones(n, device="cuda") for n in (0, 5, 0)]
    g = [torch.ones(n, device="cuda") for n in (0, 5, 0)]
    t = pq.AdamWTensors(p, g, state=pq.PQ_STATE_8BIT)
    s = pq.adamw_scalars(t, 1, 0.5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        pq.adamw_step(t, s)
    side.synchronize()
    assert (p[1] - 0.5).abs().max() < 1e-5                            # (the first step is lr, whatever the gradient's size)
    with pytest.raises(pq.PQError, match="read back"):
        pq.adamw_read(t)
