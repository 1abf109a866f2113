"""Rotary positions against the definition in fp64.

An output is u = a cos - b sin.  In fp32: sine and cosine of the reduced angle off by 2^-23 (angle 2^-25 relative, polynomial 2 roundings), times
the scale (2^-24), two products and a sum (2^-24 each): at most 5 * 2^-24 * 2 of |a| + |b| times the scale; then one rounding to the type."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as ao
from oracle import training_oracle as to
from paper_2602_22592_amd import binding as pq

pytestmark = pytest.mark.gpu
t32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32).cuda()


def rows_of(x, dtype, gap):
    T, h, d = x.shape
    buf = torch.full((T, h * d + gap), 7.0, dtype=dtype, device="cuda")
    buf[:, :h * d] = torch.from_numpy(np.ascontiguousarray(x.reshape(T, h * d), np.float32)).cuda().to(dtype)
    return buf[:, :h * d].unflatten(1, (h, d))


CASES = {
    "token": dict(rows=[1, 1, 1], lens=[1, 777, 100000], H=4, Hk=2, d=64, rot=64, no_start=True),
    "whole": dict(rows=[5, 0, 70], lens=None, H=4, Hk=4, d=128, rot=128),
    "behind": dict(rows=[5, 1, 70], lens=[5, 1001, 9000], H=4, Hk=2, d=128, rot=128),
    "part": dict(rows=[33], lens=[40], H=2, Hk=1, d=128, rot=32),
    "odd_part": dict(rows=[33], lens=[40], H=2, Hk=1, d=90, rot=46),
    "d90": dict(rows=[40, 9], lens=[40, 9], H=3, Hk=3, d=90, rot=90),
    "d2": dict(rows=[9], lens=[9], H=3, Hk=1, d=2, rot=2),
    "d80": dict(rows=[17], lens=[170], H=5, Hk=1, d=80, rot=80),
    "d256": dict(rows=[130], lens=[1300], H=2, Hk=1, d=256, rot=256),
    "no_keys": dict(rows=[12], lens=[12], H=2, Hk=0, d=64, rot=64),
    "inverse": dict(rows=[50], lens=[5000], H=2, Hk=1, d=64, rot=64, inverse=True, scale=1.25),
    "far": dict(rows=[3], lens=[2 ** 30], H=2, Hk=1, d=64, rot=64),
    "strided": dict(rows=[40], lens=[90], H=2, Hk=1, d=64, rot=64, gap=8),
    "strided_odd": dict(rows=[40], lens=[90], H=2, Hk=1, d=64, rot=64, gap=2),
    "others": dict(rows=[8, 9], lens=[90, 9], H=2, Hk=1, d=64, rot=64, before=2, behind=3),
    "many": dict(rows=[i % 4 for i in range(300)], lens=[i % 4 + i for i in range(300)], H=1, Hk=1, d=64, rot=64),
    "tall": dict(rows=[5000], lens=[5000], H=1, Hk=1, d=32, rot=32),
}


@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("name", CASES)
def test_against_the_definition(name, dtype, layout):
    c = dict(dict(gap=0, before=0, behind=0, inverse=False, scale=1.0, no_start=False), **CASES[name])
    rows, lens, d, half = c["rows"], c["lens"] or c["rows"], c["d"], c["rot"] // 2
    T = c["before"] + sum(rows) + c["behind"]
    r = np.random.default_rng(3)
    draw = lambda h: (ao.bf16 if dtype is torch.bfloat16 else np.float32)(r.standard_normal((T, h, d)))
    q, k = draw(c["H"]), draw(c["Hk"]) if c["Hk"] else None
    positions = np.concatenate([np.arange(n - m, n) for m, n in zip(rows, lens)]) if rows else []
    freqs = pq.rope_freqs(c["rot"], base=10000.0, factor=4.0, original_len=64)
    starts = None if c["no_start"] else t32(c["before"] + np.concatenate([[0], np.cumsum(rows)]))
    desc = pq.make_rope_desc(c["H"], c["Hk"], d, len(rows), rot_dim=c["rot"], layout=pq.PQ_ROPE_HALF if layout == "half" else pq.PQ_ROPE_PAIRS,
                             inverse=c["inverse"], scale=c["scale"])
    dl = None if c["lens"] is None else t32(lens)
    Q, K = rows_of(q, dtype, c["gap"]), None if k is None else rows_of(k, dtype, c["gap"])
    Qr = rows_of(np.full(q.shape, 7.0), dtype, 0)
    Kr = None if k is None else rows_of(np.full(k.shape, 7.0), dtype, c["gap"])
    pq.rope(desc, Q, K, freqs, Qr, Kr, row_start=starts, lens=dl)
    inside = slice(c["before"], c["before"] + sum(rows))
    pairs = (np.arange(half), np.arange(half) + half) if layout == "half" else (2 * np.arange(half), 2 * np.arange(half) + 1)
    u = torch.finfo(dtype).eps / 2
    for x, y in ((q, Qr), (k, Kr)):
        if x is None:
            continue
        got = y.float().cpu().numpy().astype(np.float64)
        want = to.rope(x[inside], freqs.cpu().numpy(), positions, layout, c["inverse"], c["scale"])
        tol = u * np.abs(want)
        both = 10 * 2.0 ** -24 * c["scale"] * (np.abs(x[inside][..., pairs[0]]) + np.abs(x[inside][..., pairs[1]])) * (1 + u)
        tol[..., pairs[0]] += both
        tol[..., pairs[1]] += both
        assert (np.abs(got[inside] - want) <= tol).all(), np.abs(got[inside] - want).max()
        assert (got[inside][..., c["rot"]:] == x[inside][..., c["rot"]:]).all()
        assert (got[:c["before"]] == 7).all() and (got[inside.stop:] == 7).all()
    # in place
    pq.rope(desc, Q, K, freqs, Q, K, row_start=starts, lens=dl)
    assert torch.equal(Q[inside], Qr[inside]) and (k is None or torch.equal(K[inside], Kr[inside]))


def test_the_inverse_is_the_gradient():
    """<rope(x), y> = <x, inverse(y)>: in fp32, each side 6 roundings an element."""
    desc, back = (pq.make_rope_desc(4, 0, 64, 1, rot_dim=48, scale=1.5, inverse=i) for i in (False, True))
    g = torch.Generator().manual_seed(1)
    x, y = (torch.randn((40, 4, 64), generator=g).cuda() for _ in range(2))
    rs, ln, fr = t32([0, 40]), t32([1000]), pq.rope_freqs(48)
    a, b = torch.empty_like(x), torch.empty_like(y)
    pq.rope(desc, x, None, fr, a, None, rs, ln)
    pq.rope(back, y, None, fr, b, None, rs, ln)
    left, right = (a.double() * y.double()).sum(), (x.double() * b.double()).sum()
    size = (a.double() * y.double()).abs().sum() + (x.double() * b.double()).abs().sum()
    assert abs(left - right) <= 10 * 2.0 ** -24 * 2 * size
    # .. and the difference quotient of a linear map, exact but for rounding
    e = torch.zeros_like(x)
    e[7, 2, 5] = 1.0
    c = torch.empty_like(x)
    pq.rope(desc, e, None, fr, c, None, rs, ln)
    assert abs((c.double() * y.double()).sum() - b[7, 2, 5].double()) <= 20 * 2.0 ** -24 * 1.5 * y[7, 2].abs().double().sum()
