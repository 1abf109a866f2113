"""The loads from memory straight to LDS that attention over packed rows writes as assembly: what the compiler, which does not look inside, made around
them, read from the library's own code.  (No GPU needed.)"""
import os
import re

import pytest

from paper_2602_22592_amd import binding as pq
from test_staged_stores import OBJDUMP, disassemble


def _scalars(operand):
    m = re.match(r"s\[(\d+):(\d+)\]$", operand)
    if m:
        return set(range(int(m[1]), int(m[2]) + 1))
    m = re.match(r"s(\d+)$", operand)
    return {int(m[1])} if m else set()


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no disassembler")
def test_registers_of_direct_loads(tmp_path):
    """m0, the LDS address, is set by the blocks and used by nothing else.  One wait state from m0 to the load, and five from a vector instruction that writes
    the scalar registers of its base, which the compiler does not keep in front of assembly."""
    if not os.path.exists(pq.LIB_PATH):
        from paper_2602_22592_amd.build import build
        build(verbose=False)
    loads = 0
    for name, code in disassemble(pq.LIB_PATH, ["self_forward_kernel", "self_query_kernel", "self_token_kernel"], tmp_path / "code.o").items():
        for i, line in enumerate(code):
            if not line.startswith("global_load_lds"):
                own = line.startswith("s_mov_b32 m0, s") and any(x.startswith("global_load_lds") for x in code[i + 1:i + 3])
                assert own or not re.search(r"\bm0\b|movrel|sendmsg|gws|\blds\b|buffer_load", line), (name, code[max(i - 4, 0):i + 4])
                continue
            loads += 1
            base, states, m0 = _scalars(line.split(",")[1].strip().split(" ")[0]), 0, None
            assert len(base) == 2, line
            for before in reversed(code[max(i - 8, 0):i]):
                op, _, rest = before.partition(" ")
                written = rest.split(",")[0].strip()
                if m0 is None and written == "m0":
                    m0 = states
                assert not (op.startswith("v_") and _scalars(written) & base and states < 5), (name, code[i - 8:i + 1])
                states += int(rest, 0) + 1 if op == "s_nop" else 1
            assert m0 is not None and m0 >= 1, (name, code[i - 8:i + 1])
    assert loads > 100
