"""The largest calls: a launch has fewer than 2^32 threads, 256 a workgroup, and what wants more is refused where it can be seen.  (No GPU needed.)"""
import ctypes as C

import training_calls as tc
from paper_2602_22592_amd import binding as pq

MOST = (1 << 24) - 1                            # workgroups
P = [["p", (1 << 44) * i] for i in range(1, 14)]


def rope(T, heads=32, d=90):
    n = ["l", heads * d]
    return ["pq_rope", tc.rope_desc(heads, heads, d, d), P[0], n, P[1], n, ["i", 1], ["i", T], P[2], P[3], P[4], P[5], n, P[6], n, tc.NULL]


def forward(T, n_seqs, heads=64):
    n = ["l", heads * 8]
    return ["pq_self_attn_fwd", tc.attn_desc(heads, heads, 8, n_seqs), P[0], n, P[1], n, P[2], n, ["i", T], P[3], P[4], P[5], tc.NULL]


def backward(T, n_seqs, heads=64):
    n = ["l", heads * 8]
    return ["pq_self_attn_bwd", tc.attn_desc(heads, heads, 8, n_seqs), P[0], P[1], n, P[2], n, P[3], n, P[4], P[5], ["i", T], P[6], P[7], n, P[8], n, P[9], n, P[10],
            ["n", 1 << 40], tc.NULL]


def test_positions():
    """A row a workgroup where rows are long and no multiple of 16 bytes."""
    assert [g[0] for g in tc.run([rope(MOST), rope(MOST + 1), rope(1 << 29)])] == [0, -2, -2]


def test_attention():
    """(rows / 128 + sequences) heads."""
    T, most = 1 << 18, MOST // 64 - (1 << 18) // 128
    got = tc.run([forward(T, most), forward(T, most + 1), backward(T, most), backward(T, most + 1)])
    assert [g[0] for g in got] == [0, -2, 0, -2]
    size = [["pq_self_attn_bwd_workspace_bytes", tc.attn_desc(64, 64, 8, n), ["i", T]] for n in (most, most + 1)]
    got = tc.run(size)
    assert got[0][0] > 0 and got[1][0] == 0 and "too many" in got[1][1]


def test_optimizer():
    """2048 elements a workgroup."""
    lib = pq.lib()
    t = (pq.AdamWTensor * 1)(pq.AdamWTensor(0x1000, 0x2000, None, 0x3000, 0x4000, None, None, None, MOST * 2048))
    d = pq.AdamWDesc(1, 0, 0, 0, 0, 0, 0.9, 0.999, 1e-8)
    n = lib.pq_adamw_plan_bytes(C.byref(d), t)
    assert n > 0 and n % MOST == 0
    t[0].n += 1
    assert lib.pq_adamw_plan_bytes(C.byref(d), t) == 0 and b"too many" in lib.pq_last_error_string()
    assert lib.pq_adamw_plan(C.byref(d), t, (C.c_uint64 * 64)(), 512) == -2
    one = n // MOST
    assert lib.pq_adamw_step(C.byref(d), C.c_void_p(0x1000), n + one, C.c_void_p(0x1000), None) == -4
