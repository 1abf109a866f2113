"""Rotary positions and attention over packed rows refuse outputs that share memory with inputs or with each other: their workgroups read and write
in no order.  (No GPU needed.)"""
import random

import pytest

import training_calls as tc

FAR = 1 << 32                                   # (addresses that nothing here reaches)
H, HK, D = 2, 1, 8


def call(fn, at, T=4, stride={}, dtype=1):
    """The call's arguments and the bytes of its buffers: {name: set of offsets}; buffers that `at` does not place lie far apart from each other."""
    at = dict(at)
    place = lambda name: at.setdefault(name, FAR * (1 + sorted(NAMES[fn]).index(name)))
    size = 4 if dtype == 0 else 2
    heads = lambda name: H if name in ("Q", "O", "dO", "dQ", "Qr") else HK
    row = lambda name: stride.get(name, heads(name) * D)
    p, s = (lambda name: ["p", place(name)]), (lambda name: ["l", row(name)])
    if fn == "pq_rope":
        args = [tc.rope_desc(H, HK, D), p("Q"), s("Q"), p("K"), s("K"), ["i", dtype], ["i", T], p("freqs"), p("row_start"), p("lens"), p("Qr"), s("Qr"),
                p("Kr"), s("Kr"), tc.NULL]
    elif fn == "pq_self_attn_fwd":
        args = [tc.attn_desc(H, HK, D), p("Q"), s("Q"), p("K"), s("K"), p("V"), s("V"), ["i", T], p("row_start"), p("O"), p("lse"), tc.NULL]
    else:
        args = [tc.attn_desc(H, HK, D), p("dO"), p("Q"), s("Q"), p("K"), s("K"), p("V"), s("V"), p("O"), p("lse"), ["i", T], p("row_start"), p("dQ"), s("dQ"),
                p("dK"), s("dK"), p("dV"), s("dV"), p("ws"), ["n", 512], tc.NULL]
    flat = dict(freqs=D // 2 * 8, row_start=2 * 4, lens=4, lse=T * H * 4, ws=256)            # (lse and delta of up to 16 rows: 256 bytes)
    taken = {}
    for name in NAMES[fn]:
        a = place(name)
        taken[name] = set(range(a, a + flat[name])) if name in flat else {
            x for i in range(T) for x in range(a + i * row(name) * size, a + (i * row(name) + heads(name) * D) * size)}
    return [fn] + args, taken


NAMES = {"pq_rope": ("Q", "K", "freqs", "row_start", "lens", "Qr", "Kr"), "pq_self_attn_fwd": ("Q", "K", "V", "row_start", "O", "lse"),
         "pq_self_attn_bwd": ("dO", "Q", "K", "V", "O", "lse", "row_start", "dQ", "dK", "dV", "ws")}
WRITTEN = {"pq_rope": ("Qr", "Kr"), "pq_self_attn_fwd": ("O", "lse"), "pq_self_attn_bwd": ("dQ", "dK", "dV", "ws")}
IN_PLACE = {("Qr", "Q"), ("Kr", "K")}


@pytest.mark.parametrize("fn", NAMES)
def test_equal_addresses(fn):
    calls, want = [], []
    for w in WRITTEN[fn]:
        for other in NAMES[fn]:
            if other != w:
                calls.append(call(fn, {w: 0x1000, other: 0x1000})[0])
                want.append(0 if (w, other) in IN_PLACE else -1)
    calls.append(call(fn, {})[0])
    want.append(0)
    got = tc.run(calls)
    assert [g[0] for g in got] == want, [(c[0], g) for c, g, w in zip(calls, got, want) if g[0] != w]
    assert all(bool(g[2]) == (g[0] == 0) for g in got)               # (nothing is launched by a refused call)
    assert all("overlap" in g[1] for g in got if g[0])


@pytest.mark.parametrize("fn", NAMES)
def test_any_two_buffers_near_each_other(fn):
    """Against the sets of their bytes: rows between each other's rows are no overlap, a shared byte is one."""
    r = random.Random(7)
    calls, want, kinds = [], [], {True: 0, False: 0}
    while len(calls) < 1200:
        w, other = r.choice(WRITTEN[fn]), r.choice(NAMES[fn])
        if w == other or (w, other) in IN_PLACE:
            continue
        T = r.choice((1, 2, 3, 7, 16))
        same = r.choice((None, 24, 32, 40, 64))
        stride = {n: same or 2 * r.randint(8, 30) for n in NAMES[fn]}
        for n in ("O", "dO"):
            stride.pop(n, None)
        c, taken = call(fn, {w: 0x100000, other: 0x100000 + 16 * r.randint(-70, 70)}, T=T, stride=stride, dtype=r.choice((0, 1)) if fn == "pq_rope" else 1)
        bad = bool(taken[w] & taken[other])
        kinds[bad] += 1
        calls.append(c)
        want.append(-1 if bad else 0)
    assert min(kinds.values()) > 100
    got = tc.run(calls)
    assert [g[0] for g in got] == want, [(c, g) for c, g, x in zip(calls, got, want) if g[0] != x][:3]


def test_rope_in_place_with_neighbouring_heads():
    """Queries and keys in one buffer, turned where they are, and moved by a head's width."""
    one = dict(stride=dict(Q=48, K=48, Qr=48, Kr=48))
    base, keys = 0x100000, 0x100000 + H * D * 2
    ok, _ = call("pq_rope", dict(Q=base, K=keys, Qr=base, Kr=keys), **one)
    bad, _ = call("pq_rope", dict(Q=base, K=keys, Qr=base + 16, Kr=keys), **one)
    swapped, _ = call("pq_rope", dict(Q=base, K=keys, Kr=base), **one)
    other, _ = call("pq_rope", dict(Q=base, K=keys, Qr=base), stride=dict(Q=48, K=48, Qr=50, Kr=48))
    assert [g[0] for g in tc.run([ok, bad, swapped, other])] == [0, -1, -1, -2]


def test_rows_of_one_long_buffer():
    """2^20 rows of four tensors between each other, and one of them moved onto the last row of another."""
    def rope(Kr):
        at = [1 << 40, (1 << 40) + 32, (1 << 40) + 64, Kr]
        far = [["p", (1 << 50) + 4096 * i] for i in range(3)]
        return ["pq_rope", tc.rope_desc(H, HK, D), ["p", at[0]], ["l", 64], ["p", at[1]], ["l", 64], ["i", 1], ["i", 1 << 20], *far, ["p", at[2]], ["l", 64],
                ["p", at[3]], ["l", 64], tc.NULL]
    got = tc.run([rope((1 << 40) + 96), rope((1 << 40) + (1 << 20) * 128 - 128), rope((1 << 40) + (1 << 20) * 128)])
    assert [g[0] for g in got] == [0, -1, 0]
