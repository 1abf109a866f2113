"""Attention over the rows of a call where it can go wrong: what is not finite, far addresses, streams, captured calls, broken row_start."""
import numpy as np
import pytest
import torch

from self_attention_cases import Packed
from paper_2602_22592_amd import binding as pq

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


def spoiled(c, where):
    """c with single rows (or elements) of its inputs replaced, and the same with zeros there."""
    kw = dict(rows=c.rows, H=c.H, Hk=c.Hk, d=c.d, causal=c.causal, window=c.window, seed=11)
    bad, clean = Packed(**kw), Packed(**kw)
    for name, index, value in where:
        getattr(bad, name)[index] = value
        getattr(clean, name)[index] = 0.0
    return bad, clean


@pytest.mark.parametrize("d,window", [(64, 0), (128, 0), (90, 0), (64, 10), (32, 0)])
@pytest.mark.parametrize("value", [NAN, INF, -INF])
def test_hidden_values_have_no_effect(d, window, value):
    """A value that only later rows see: earlier rows (of the same tile of scores) and other sequences are as if it were not there."""
    c = Packed(rows=[70, 40], H=2, Hk=1, d=d, window=window)
    j = 33
    bad, clean = spoiled(c, [("v", (j, 0, 3), value)])
    (O, lse), (Oc, lsec) = bad.forward(), clean.forward()
    sees = np.zeros(110, bool)
    sees[j:min(70, j + window) if window else 70] = True
    hit = O[torch.from_numpy(sees).cuda()][:, :, 3].float()
    assert (~torch.isfinite(hit)).all()
    other = torch.ones_like(O, dtype=torch.bool)
    other[torch.from_numpy(sees).cuda(), :, 3] = False
    assert torch.isfinite(O[other].float()).all()
    O[~other] = Oc[~other]
    clean.check_forward(O, lse)


@pytest.mark.parametrize("d", [64, 128, 90])
@pytest.mark.parametrize("value", [NAN, INF])
def test_hidden_keys_and_queries(d, value):
    c = Packed(rows=[70, 40], H=2, Hk=1, d=d)
    bad, clean = spoiled(c, [("k", (33, 0, 5), value), ("q", (12, 1, 7), value)])
    (O, lse), (Oc, lsec) = bad.forward(), clean.forward()
    hit = torch.zeros((110, 2), dtype=torch.bool, device="cuda")
    hit[12, 1] = True
    if value != value:
        hit[33:70] = True
        assert O[hit].isnan().all()
    else:                                                            # (a score of -infinity weighs nothing, one of +infinity is NaN)
        k_hit = ~torch.isfinite(O.float()).all(2)
        assert k_hit[12, 1] and not k_hit[:12].any() and not k_hit[13:33].any() and not k_hit[70:].any() and not k_hit[12, 0]
        hit[33:70] = True
    O[hit], lse[hit] = Oc[hit], lsec[hit]
    clean.check_forward(O, lse)


@pytest.mark.parametrize("d", [64, 128, 90, 32])
@pytest.mark.parametrize("value", [NAN, INF])
def test_gradients_of_hidden_rows(d, value):
    """The gradient of one row's output is not finite: dQ of other rows, dK and dV of tokens that it does not see, and other sequences are unaffected."""
    c = Packed(rows=[70, 40], H=2, Hk=2, d=d)
    i = 40
    bad, clean = spoiled(c, [("do", (i, 0), value)])
    O, lse = clean.forward()
    out, want = bad.backward(O, lse), clean.backward(O, lse)
    assert (~torch.isfinite(out[0][i, 0].float())).all()
    for x in out[1:]:
        assert (~torch.isfinite(x[:i + 1, 0].float())).any(1).all()
    for x, y, rows in zip(out, want, (slice(i, i + 1), slice(0, i + 1), slice(0, i + 1))):
        x[rows, 0] = y[rows, 0]
        assert torch.isfinite(x.float()).all()
    clean.check_backward(O, lse, out)


@pytest.mark.parametrize("d", [64, 128, 90])
def test_gradients_of_rows_before_a_value_that_is_not_finite(d):
    c = Packed(rows=[70, 40], H=1, Hk=1, d=d)
    bad, clean = spoiled(c, [("v", (33, 0, 3), INF), ("k", (50, 0, 1), NAN)])
    O, lse = bad.forward()
    Oc, lsec = clean.forward()
    dQ, dK, dV = bad.backward(O, lse)
    cQ, cK, cV = clean.backward(Oc, lsec)
    assert (~torch.isfinite(dQ[33:70].float())).any(2).all()
    dQ[33:70] = cQ[33:70]
    dK[:70], dV[:70] = cK[:70], cV[:70]                               # (rows 33 .. 69 see all of these)
    clean.check_backward(Oc, lsec, (dQ, dK, dV))


@pytest.mark.parametrize("d", [64, 128])
def test_scores_far_above_the_first_ones(d):
    """The reference is the first stage's maximum; later scores 2^7 .. 2^10 powers of two above it overflow and are taken with care."""
    c = Packed(rows=[200], H=1, Hk=1, d=d, scale=1.0)
    c.q[:], c.k[:] = 0.0, 0.0
    c.q[:, :, 0] = 8.0
    c.k[:64, :, 0] = 0.0
    c.k[64:, :, 0] = np.linspace(10, 90, 136).astype(np.int32)[:, None]
    O, lse = c.forward()
    c.check_forward(O, lse)
    c.check_backward(O, lse, c.backward(O, lse))


@pytest.mark.parametrize("bad", [[0, 50, 20, 110], [-5, 40, 500, 90], [110, 0, 0, 0], [2 ** 31 - 1, -2 ** 31, 5, 7]])
def test_broken_row_start_stays_inside_the_buffers(bad):
    """What comes out is not defined; nothing behind the rows is written, by any of the calls."""
    c = Packed(rows=[40, 40, 30], H=2, Hk=1, d=64)
    Q, K, V = c.inputs()
    rs = torch.tensor(bad, dtype=torch.int32).cuda()
    O, lse = torch.full((140, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((140, 2), 7.0, device="cuda")
    out = [torch.full((140, h, 64), 7.0, dtype=torch.bfloat16, device="cuda") for h in (2, 1, 1)]
    pq.self_attn_fwd(c.desc(), Q, K, V, rs, O[:110], lse[:110])
    pq.self_attn_bwd(c.desc(), O[:110], Q, K, V, O[:110], lse[:110], rs, *[x[:110] for x in out], pq.self_attn_bwd_workspace(c.desc(), 110))
    rope = pq.make_rope_desc(2, 1, 64, 3)
    turned = [torch.full((140, h, 64), 7.0, dtype=torch.bfloat16, device="cuda") for h in (2, 1)]
    pq.rope(rope, Q, K, pq.rope_freqs(64), turned[0][:110], turned[1][:110], row_start=rs)
    torch.cuda.synchronize()
    for x in [O, lse] + out + turned:
        assert (x[110:] == 7).all()


def test_rows_beyond_32_bits():
    """Rows 2^31 and more elements from the buffers' beginning."""
    stride, T, n = 1 << 16, 33000, 70
    c = Packed(rows=[n], H=2, Hk=1, d=64)
    at = T - n
    big = [torch.empty((T, stride), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    q, k = (b[:, :64 * h].unflatten(1, (h, 64)) for b, h in zip(big, (2, 1)))
    v = big[0][:, 256:320].unflatten(1, (1, 64))
    for x, y in ((q, c.q), (k, c.k), (v, c.v)):
        x[at:] = torch.from_numpy(y).cuda().bfloat16()
    rs = torch.tensor([at, T], dtype=torch.int32).cuda()
    O, lse = torch.empty((T, 2, 64), dtype=torch.bfloat16, device="cuda"), torch.empty((T, 2), device="cuda")
    pq.self_attn_fwd(c.desc(), q, k, v, rs, O, lse)
    c.check_forward(O[at:], lse[at:])
    dO = torch.zeros((T, 2, 64), dtype=torch.bfloat16, device="cuda")
    dO[at:] = torch.from_numpy(c.do).cuda().bfloat16()
    dq, dk, dv = (big[1][:, a:a + 64 * h].unflatten(1, (h, 64)) for a, h in ((1024, 2), (2048, 1), (4096, 1)))
    pq.self_attn_bwd(c.desc(), dO, q, k, v, O, lse, rs, dq, dk, dv, pq.self_attn_bwd_workspace(c.desc(), T))
    c.check_backward(O[at:], lse[at:], [x[at:] for x in (dq, dk, dv)])
    turned = big[1][:, 8192:8192 + 128].unflatten(1, (2, 64))
    fr = pq.rope_freqs(64)
    pq.rope(pq.make_rope_desc(2, 0, 64, 1), q, None, fr, turned, None, row_start=rs)
    small = torch.empty((n, 2, 64), dtype=torch.bfloat16, device="cuda")
    pq.rope(pq.make_rope_desc(2, 0, 64, 1), q[at:].contiguous(), None, fr, small, None, row_start=torch.tensor([0, n], dtype=torch.int32).cuda())
    assert torch.equal(turned[at:], small)


def test_captured_calls_are_replayed_with_other_inputs_and_sequences():
    c = Packed(rows=[60, 70, 20], H=4, Hk=2, d=64)
    Q, K, V = c.inputs()
    dO, rs = c.gpu(c.do), c.row_start()
    desc, fr = c.desc(), pq.rope_freqs(64)
    turn, back = (pq.make_rope_desc(4, 2, 64, 3, inverse=i) for i in (False, True))

    def step(x, out, ws):
        Q, K, V = x
        qt, kt, O, lse, dq, dk, dv = out
        pq.rope(turn, Q, K, fr, qt, kt, row_start=rs)
        pq.self_attn_fwd(desc, qt, kt, V, rs, O, lse)
        pq.self_attn_bwd(desc, dO, qt, kt, V, O, lse, rs, dq, dk, dv, ws)
        pq.rope(back, dq, dk, fr, dq, dk, row_start=rs)
    new = lambda: [torch.zeros_like(Q), torch.zeros_like(K), torch.zeros_like(Q), torch.zeros((150, 4), device="cuda"), torch.zeros_like(Q),
                   torch.zeros_like(K), torch.zeros_like(V)]
    got, want = new(), new()
    ws, ws2 = (pq.self_attn_bwd_workspace(desc, 150) for _ in range(2))
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        step((Q, K, V), got, ws)
    for i, starts in enumerate(([0, 60, 130, 150], [0, 1, 2, 150], [0, 150, 150, 150], [0, 0, 75, 150])):
        for x in (Q, K, V, dO):
            x.mul_(1.0 + 0.125 * i)
        rs.copy_(torch.tensor(starts, dtype=torch.int32))
        g.replay()
        step((Q, K, V), want, ws2)
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), (i, starts)


def test_calls_on_two_streams_at_once():
    cs = [Packed(rows=[200, 90], H=4, Hk=2, d=128, seed=i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    work = []
    for c in cs:
        dev = c.inputs()
        O, lse = c.outputs()
        work.append((c, dev, O, lse, c.gradients(), c.gpu(c.do), pq.self_attn_bwd_workspace(c.desc(), c.T), c.row_start()))
    torch.cuda.synchronize()
    for _ in range(3):
        for s, (c, dev, O, lse, out, dO, ws, rs) in zip(streams, work):
            with torch.cuda.stream(s):
                pq.self_attn_fwd(c.desc(), *dev, rs, O, lse)
                pq.self_attn_bwd(c.desc(), dO, *dev, O, lse, rs, *out, ws)
    torch.cuda.synchronize()
    for c, dev, O, lse, out, *_ in work:
        c.check_forward(O, lse)
        c.check_backward(O, lse, out)


def test_gradients_against_differences():
    """The kernel's gradients against difference quotients of the definition in fp64 (central, 2^-12 wide: off by its third derivatives, below 1e-5)."""
    from oracle import training_oracle as to
    c = Packed(rows=[12], H=2, Hk=1, d=8)
    O, lse = c.forward()
    grads = [x.float().cpu().numpy() for x in c.backward(O, lse)]
    seen = to.seen_by(12)

    def loss(q, k, v):
        return sum((to.self_attention(q[:, h], k[:, 0], v[:, 0], seen, c.scale)[0] * c.do[:, h]).sum() for h in range(2))
    r = np.random.default_rng(2)
    xs = [x.astype(np.float64) for x in (c.q, c.k, c.v)]
    for n, (x, g) in enumerate(zip(xs, grads)):
        for _ in range(12):
            at = tuple(r.integers(0, s) for s in x.shape)
            step, e = np.zeros_like(x), 2.0 ** -12
            step[at] = e
            up, down = (loss(*[y + (sign * step if m == n else 0) for m, y in enumerate(xs)]) for sign in (1, -1))
            # products of bf16-rounded p and dS: 2^-8 of the terms' sizes, which are at most a few units here
            assert abs((up - down) / (2 * e) - g[at]) <= 2.0 ** -8 * (abs(g[at]) + np.abs(g).max()) + 1e-5, (n, at)
