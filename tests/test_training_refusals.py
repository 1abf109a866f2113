"""What rotary positions, attention over packed rows and the optimizer refuse, on the host, before anything is launched (no GPU needed)."""
import ctypes as C
import os

import pytest
import torch

from oracle import training_oracle as to
from paper_2602_22592_amd import binding as pq

fake, big = C.c_void_p(0x1000), C.c_size_t(1 << 50)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(pq.LIB_PATH):
        from paper_2602_22592_amd.build import build
        build(verbose=False)
    return pq.lib()


def rope_call(lib, d, T=4, dtype=1, Q=fake, qs=256, ks=128, freqs=fake, rs=fake, lens=fake, Qr=None, qrs=256, K=fake, Kr=fake, krs=128):
    Qr = C.c_void_p(0x2000) if Qr is None else Qr
    return lib.pq_rope(C.byref(d), Q, qs, K, ks, dtype, T, freqs, rs, lens, Qr, qrs, Kr, krs, None)


@pytest.mark.parametrize("bad,code", [(dict(n_heads=0), -1), (dict(n_kv_heads=-1), -1), (dict(n_heads=70000), -1), (dict(d_head=63), -2), (dict(d_head=0), -2),
                                      (dict(d_head=258), -2), (dict(rot_dim=66), -2), (dict(rot_dim=3), -2), (dict(layout=2), -1), (dict(inverse=2), -1),
                                      (dict(scale=float("inf")), -1), (dict(n_seqs=-1), -1)])
def test_rope_descriptors(lib, bad, code):
    d = pq.make_rope_desc(4, 2, 64, 2)
    for k, v in bad.items():
        setattr(d, k, v)
    assert rope_call(lib, d) == code


def test_rope_arguments(lib):
    d = pq.make_rope_desc(4, 2, 64, 2)
    assert rope_call(lib, d, T=0) == 0 and rope_call(lib, pq.make_rope_desc(4, 2, 64, 0)) == 0
    assert rope_call(lib, d, T=-1) == -1
    assert rope_call(lib, d, dtype=2) == -3
    assert rope_call(lib, d, Q=None) == -1 and rope_call(lib, d, K=None) == -1 and rope_call(lib, d, freqs=None) == -1
    assert rope_call(lib, d, rs=None, lens=None) == -1
    assert rope_call(lib, d, qs=254) == -2 and rope_call(lib, d, qs=257) == -2 and rope_call(lib, d, krs=126) == -2
    assert rope_call(lib, d, Q=C.c_void_p(0x1008)) == -2
    assert rope_call(lib, d, Qr=fake, qrs=512) == -2                  # in place with another stride


def attn(**k):
    return pq.make_self_attn_desc(**dict(dict(n_heads=4, n_kv_heads=2, d_head=64, n_seqs=2), **k))


out = C.c_void_p(0x2000)


def fwd(lib, d, T=4, Q=fake, qs=256, ks=128, vs=128, rs=fake, O=out, lse=fake):
    return lib.pq_self_attn_fwd(C.byref(d), Q, qs, fake, ks, fake, vs, T, rs, O, lse, None)


def bwd(lib, d, T=4, dO=fake, ws=fake, n=big, dqs=256, dQ=out, dK=out):
    return lib.pq_self_attn_bwd(C.byref(d), dO, fake, 256, fake, 128, fake, 128, fake, fake, T, fake, dQ, dqs, dK, 128, out, 128, ws, n, None)


@pytest.mark.parametrize("bad,code", [(dict(n_heads=3), -2), (dict(n_kv_heads=0), -2), (dict(d_head=63), -2), (dict(d_head=130), -2), (dict(d_head=0, scale=1.0), -2),
                                      (dict(n_seqs=-1), -1), (dict(causal=2), -1), (dict(causal=False, window=4), -1), (dict(window=-1), -1),
                                      (dict(scale=float("nan")), -1), (dict(n_heads=1 << 18, n_kv_heads=1), -2)])
def test_attention_descriptors(lib, bad, code):
    d = attn(**bad)
    if bad.get("causal") == 2:
        d.causal = 2
    assert fwd(lib, d) == code and bwd(lib, d) == code
    assert lib.pq_self_attn_bwd_workspace_bytes(C.byref(d), 4) == 0


def test_attention_arguments(lib):
    d = attn()
    assert fwd(lib, d, T=0) == 0 and fwd(lib, attn(n_seqs=0)) == 0 and bwd(lib, d, T=0) == 0
    assert fwd(lib, d, T=-1) == -1 and fwd(lib, d, T=(1 << 29) + 1) == -2 and fwd(lib, attn(n_heads=64, n_kv_heads=1), T=1 << 25) == -2
    assert fwd(lib, d, Q=None) == -1 and fwd(lib, d, rs=None) == -1 and fwd(lib, d, lse=None) == -1
    assert fwd(lib, d, qs=254) == -2 and fwd(lib, d, ks=129) == -2 and fwd(lib, d, vs=(1 << 23) + 2) == -2
    assert fwd(lib, d, O=C.c_void_p(0x1004)) == -2
    need = lib.pq_self_attn_bwd_workspace_bytes(C.byref(d), 4)
    assert need > 0 and bwd(lib, d, n=C.c_size_t(need - 1)) == -4
    assert bwd(lib, d, dQ=fake) == -1 and bwd(lib, d, dK=fake) == -1 and fwd(lib, d, O=fake) == -1        # in place
    assert bwd(lib, d, ws=None) == -1 and bwd(lib, d, dO=None) == -1 and bwd(lib, d, dqs=255) == -2


def test_attention_workspace(lib):
    """Room for lse and delta, and for a tile's pieces where there are few tiles with much work; no sequences need no more."""
    def size(T, **k):
        return lib.pq_self_attn_bwd_workspace_bytes(C.byref(attn(**k)), T)
    assert size(1 << 20, n_seqs=0) <= (1 << 20) * 64 + 512
    long, cut = dict(n_heads=32, n_kv_heads=8, d_head=64), 8192 * 8 * 2 * 64 * 4
    assert size(8192, **long) == 8192 * 32 * 8 + 3 * cut + 256                                             # 520 tiles, 4 heads of 129 stages
    assert size(8192, window=100, **long) == 8192 * 32 * 8 + 256                                           # a tile's rows are 4 stages
    assert size(8192, n_heads=32, n_kv_heads=32, d_head=64) == 8192 * 32 * 8 + 256


def tensors(n=300, **k):
    t = pq.AdamWTensor(0x1000, 0x2000, None, 0x3000, 0x4000, None, None, None, n)
    for a, b in k.items():
        setattr(t, a, b)
    return (pq.AdamWTensor * 1)(t)


def adamw(**k):
    d = pq.AdamWDesc(1, 0, 0, 0, 0, 0, 0.9, 0.999, 1e-8)
    for a, b in k.items():
        setattr(d, a, b)
    return d


@pytest.mark.parametrize("desc,t,code", [
    (dict(n_tensors=-1), {}, -1), (dict(param_dtype=2), {}, -3), (dict(grad_dtype=5), {}, -3), (dict(state_kind=2), {}, -1), (dict(beta1=1.0), {}, -1),
    (dict(beta2=-0.1), {}, -1), (dict(eps=0.0), {}, -1), (dict(eps=float("nan")), {}, -1), (dict(has_masters=1), dict(master=0x5000), -3),
    (dict(has_masters=2), {}, -1), (dict(has_values=1), {}, -1),
    ({}, dict(n=-1), -1), ({}, dict(param=None), -1), ({}, dict(grad=None), -1), ({}, dict(m=None), -1), ({}, dict(param=0x1008), -2),
    (dict(state_kind=1), {}, -1), (dict(state_kind=1), dict(steps=0x5004), -2), ({}, dict(master=0x5000), -1), ({}, dict(n=(1 << 40) + 1), -1),
    (dict(param_dtype=1, has_masters=1), {}, -1), (dict(state_kind=1), dict(steps=0x5000, m_values=0x6000), -1)])
def test_optimizer_tensors(lib, desc, t, code):
    d, arr = adamw(**desc), tensors(**t)
    assert lib.pq_adamw_plan_bytes(C.byref(d), arr) == 0
    buf = (C.c_uint64 * 64)()
    assert lib.pq_adamw_plan(C.byref(d), arr, buf, C.sizeof(buf)) == code


def test_optimizer_plans(lib):
    d, arr = adamw(), tensors(n=3000)
    n = lib.pq_adamw_plan_bytes(C.byref(d), arr)
    buf = (C.c_uint64 * (n // 8))()
    assert n % 8 == 0 and lib.pq_adamw_plan(C.byref(d), arr, buf, n) == 0
    assert lib.pq_adamw_plan(C.byref(d), arr, buf, n - 1) == -4 and lib.pq_adamw_plan(C.byref(d), arr, None, n) == -1
    words = n // 3 // 8                                               # three pieces of up to 1024 elements
    assert [buf[words * i + words - 1] for i in range(3)] == [1024, 1024, 952]
    assert [buf[words * i] for i in range(3)] == [0x1000, 0x2000, 0x3000]
    step = lambda plan=fake, n=n, s=fake, d=d: lib.pq_adamw_step(C.byref(d), plan, n, s, None)
    assert step(plan=None) == -1 and step(s=None) == -1 and step(n=n - 1) == -4 and step(n=0) == -4 and step(s=C.c_void_p(0x1004)) == -2
    assert step(plan=C.c_void_p(0x1008)) == -2 and step(d=adamw(beta1=2.0)) == -1
    assert lib.pq_adamw_read(C.byref(d), fake, n, None) == -1          # fp32 states
    assert lib.pq_adamw_read(C.byref(adamw(state_kind=1)), fake, n, None) == -1
    assert lib.pq_adamw_plan_bytes(C.byref(adamw()), tensors(n=0)) > 0   # nothing to do is no error


def test_binding_refuses_before_the_library_is_asked():
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    d = attn()
    rs = torch.tensor([0, 2, 4], dtype=torch.int32)
    with pytest.raises(pq.PQError, match="one GPU"):
        pq.self_attn_fwd(d, bf(4, 4, 64), bf(4, 2, 64), bf(4, 2, 64), rs, bf(4, 4, 64), torch.zeros(4, 4))
    with pytest.raises(pq.PQError, match="as many rows"):
        pq.self_attn_fwd(d, bf(4, 4, 64), bf(3, 2, 64), bf(4, 2, 64), rs, bf(4, 4, 64), torch.zeros(4, 4))
    with pytest.raises(pq.PQError, match="shape"):
        pq.self_attn_fwd(d, bf(4, 4, 64), bf(4, 4, 64), bf(4, 2, 64), rs, bf(4, 4, 64), torch.zeros(4, 4))
    with pytest.raises(pq.PQError, match="contiguous bf16"):
        pq.self_attn_fwd(d, bf(4, 4, 64), bf(4, 2, 64), bf(4, 2, 64), rs, torch.zeros(4, 4, 64), torch.zeros(4, 4))
    with pytest.raises(pq.PQError, match="lse"):
        pq.self_attn_fwd(d, bf(4, 4, 64), bf(4, 2, 64), bf(4, 2, 64), rs, bf(4, 4, 64), torch.zeros(4, 3))
    r = pq.make_rope_desc(4, 2, 64, 2)
    with pytest.raises(pq.PQError, match="one GPU"):
        pq.rope(r, bf(4, 4, 64), bf(4, 2, 64), torch.zeros(32, dtype=torch.float64), bf(4, 4, 64), bf(4, 2, 64), row_start=rs)
    with pytest.raises(pq.PQError, match="low"):
        pq.rope_freqs(64, low=2.0, high=1.0, device="cpu")
    p, g = [torch.zeros(300)], [torch.zeros(300)]
    with pytest.raises(pq.PQError, match="one GPU"):
        pq.AdamWTensors(p, g)
    with pytest.raises(pq.PQError, match="without tensors"):
        pq.AdamWTensors([], [])
    with pytest.raises(pq.PQError, match="together"):
        pq.AdamWTensors(p, g, m=p)


def test_frequencies():
    f = pq.rope_freqs(8, base=100.0, device="cpu")
    assert f.dtype is torch.float64 and torch.allclose(f * 2 * torch.pi, torch.tensor([100.0 ** (-i / 4) for i in range(4)], dtype=torch.float64), rtol=1e-14)
    assert torch.equal(pq.rope_freqs(8, factor=4.0, device="cpu"), pq.rope_freqs(8, device="cpu") / 4)
    parts, plain = pq.rope_freqs(64, factor=8.0, original_len=4096, device="cpu"), pq.rope_freqs(64, device="cpu")
    turns = 4096 * plain
    assert torch.equal(parts[turns >= 32], plain[turns >= 32]) and torch.equal(parts[turns <= 1], plain[turns <= 1] / 8)
    between = (turns > 1) & (turns < 32)
    assert between.any() and (parts[between] < plain[between]).all() and (parts[between] > plain[between] / 8).all()


def test_oracle_gradients_against_differences():
    import numpy as np
    r = np.random.default_rng(0)
    q, k, v, do = (r.standard_normal((9, 4)) for _ in range(4))
    seen = to.seen_by(9, window=5)
    o, lse, _ = to.self_attention(q, k, v, seen, 0.4)
    grads = to.self_attention_gradients(do, q, k, v, lse, seen, 0.4)[:3]
    f = lambda *x: (to.self_attention(*x, seen, 0.4)[0] * do).sum()
    for n, g in enumerate(grads):
        for at in np.ndindex(9, 4):
            e = np.zeros((9, 4))
            e[at] = 1e-5
            up, down = (f(*[x + (s * e if m == n else 0) for m, x in enumerate((q, k, v))]) for s in (1, -1))
            assert abs((up - down) / 2e-5 - g[at]) < 1e-8
