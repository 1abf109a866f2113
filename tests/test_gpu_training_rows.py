"""Rows of no sequence in training: as many as a step's row_start says, whatever the steps before it left in the buffers."""
import numpy as np
import pytest
import torch

from paper_2602_22592_amd import binding as pq
from paper_2602_22592_amd import workloads as wl
from paper_2602_22592_amd.stack import AttentionCore, Stack

pytestmark = pytest.mark.gpu
t32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32).cuda()
dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda().to(torch.bfloat16)
NAMES = ("Wq", "Wk", "Wv", "Wo", "W_up", "W_gate", "W_down", "Up", "Gate", "Down", "Wr")
T, D, F, E, R, H, HK = 128, 64, 96, 2, 8, 2, 1


class Steps:
    """A stack of two layers over two sequences, and a step's inputs."""

    def __init__(self, case):
        layers = [dict(w, Wk=w["Wk"][:HK * D // H], Wv=w["Wv"][:HK * D // H]) for w in case["layers"]]
        self.weights = [{n: dev(w[n]) for n in NAMES} for w in layers]
        self.grads = [dict({n: torch.empty(w[n].shape, dtype=torch.float32, device="cuda") for n in NAMES}, dab=torch.empty(2, device="cuda")) for w in layers]
        self.core = AttentionCore(T, H, HK, D // H, 2, freqs=pq.rope_freqs(D // H))
        self.stack = Stack(2, T, D, F, E, R, 1, [w["alpha"] for w in layers], [w["beta"] for w in layers], core=self.core)

    def run(self, x, dY, rows):
        out = self.stack.forward(x, self.weights, rows).clone()
        return out, self.stack.backward(dY, self.weights, self.grads, rows).clone()

    def left(self):
        """Everything that a step leaves and the next product reads."""
        st = self.stack
        return {**{f"{l}.{n}": g[n].clone() for l, g in enumerate(self.grads) for n in g}, "dq": st.dq, "dk": st.dkv[0], "dv": st.dkv[1],
                **{f"{l}.o": ly["core"]["o"] for l, ly in enumerate(st.layers)}}


def _case():
    c = wl.stack_case(9, 2, T, D, F, E, R, vocab=100)
    return c, dev(c["table"][c["ids"]]), dev(c["dY"])


@pytest.mark.parametrize("second", [[0, 50, 100], [20, 20, 90], [0, 0, 0], [128, 128, 128]])
def test_a_step_with_fewer_rows_than_the_one_before(second):
    """As a stack that never saw another row_start, bit by bit."""
    c, x, dY = _case()
    a, b = Steps(c), Steps(c)
    a.run(x, dY, t32([0, 60, 128]))
    got, want = a.run(x, dY, t32(second)), b.run(x, dY, t32(second))
    for p, q in zip(got, want):
        assert torch.isfinite(q).all() and torch.equal(p, q)
    for (name, p), q in zip(a.left().items(), b.left().values()):
        assert torch.isfinite(q).all() and torch.equal(p, q), name


def test_captured_steps_take_a_new_row_start():
    c, x, dY = _case()
    a, rows = Steps(c), t32([0, 60, 128])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a.run(x, dY, rows)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.stack.forward(x, a.weights, rows)
        a.stack.backward(dY, a.weights, a.grads, rows)
    for starts in ([0, 60, 128], [10, 40, 90], [0, 1, 2], [30, 128, 128]):
        rows.copy_(t32(starts))
        graph.replay()
        torch.cuda.synchronize()
        b = Steps(c)                                                 # (one that never saw another row_start)
        b.run(x, dY, t32(starts))
        torch.cuda.synchronize()
        for (name, p), q in zip(a.left().items(), b.left().values()):
            assert torch.isfinite(q).all() and torch.equal(p, q), (starts, name)


def test_a_core_clears_what_it_is_given():
    """Output and gradients full of NaN, as memory that nobody has written may be."""
    core = AttentionCore(T, H, HK, D // H, 2, freqs=pq.rope_freqs(D // H))
    s = core.saved()
    for n in "qkv":
        s[n].normal_()
    for n in ("o", "lse"):
        s[n].fill_(float("nan"))
    rows, outside = t32([10, 40, 90]), torch.ones(T, dtype=torch.bool, device="cuda")
    outside[10:90] = False
    m = core.forward(s, rows)
    assert torch.isfinite(m).all() and (m[outside] == 0).all() and (m[~outside] != 0).any(1).all()
    grads = [torch.full((T, h * D // H), float("nan"), dtype=torch.bfloat16, device="cuda") for h in (H, HK, HK)]
    core.backward(torch.randn((T, H, D // H), device="cuda").bfloat16(), s, rows, *grads)
    for g in grads:
        assert torch.isfinite(g).all() and (g[outside] == 0).all()
    assert (grads[2][~outside] != 0).any(1).all()


def test_alpha_and_beta_are_those_of_the_descriptors_at_the_call():
    """What nothing in the stack trains: whoever does writes them into the layers' descriptors."""
    c, x, dY = _case()
    rows, a = t32([0, 60, 128]), Steps(c)
    before = a.run(x, dY, rows)[0]
    for w, ly in zip(c["layers"], a.stack.layers):
        w["alpha"], w["beta"] = 1.5 * w["alpha"], 0.5 * w["beta"]
        ly["ffn_desc"].alpha, ly["ffn_desc"].beta = w["alpha"], w["beta"]
    b = Steps(c)
    got, want = a.run(x, dY, rows), b.run(x, dY, rows)
    assert not torch.equal(got[0], before)
    for p, q in zip(got, want):
        assert torch.equal(p, q)
    for (name, p), q in zip(a.left().items(), b.left().values()):
        assert torch.equal(p, q), name
