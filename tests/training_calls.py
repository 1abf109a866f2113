"""The host side of the training calls without a GPU: what a call returns, and what it launches.

`run(calls)` makes the calls in a child process whose HIP runtime is host_launches.c: a launch is counted and does nothing.  A call is [function,
[type, value], ...]: "d" a descriptor of whole numbers and floats (by their Python types), "p" an address (0: NULL), "i" int32, "l" int64, "n" size_t.
The result is one [returned, error, kernels] per call."""
import ctypes as C
import json
import os
import struct
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
LIB = os.path.join(os.path.dirname(HERE), "paper_2602_22592_amd", "libpquant.so")
NULL = ["p", 0]


def run(calls):
    with tempfile.TemporaryDirectory() as tmp:
        shim = os.path.join(tmp, "libhost_launches.so")
        subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-o", shim, os.path.join(HERE, "host_launches.c")], check=True)
        res = subprocess.run([sys.executable, os.path.abspath(__file__), shim, LIB], input=json.dumps(calls), text=True, capture_output=True, check=False)
    assert res.returncode == 0, res.stderr
    return json.loads(res.stdout)


def rope_desc(n_heads=2, n_kv_heads=1, d_head=8, rot_dim=8, layout=0, inverse=0, n_seqs=1, scale=1.0):
    return ["d", [n_heads, n_kv_heads, d_head, rot_dim, layout, inverse, n_seqs, scale]]


def attn_desc(n_heads=2, n_kv_heads=1, d_head=8, n_seqs=1, causal=1, window=0, scale=0.5):
    return ["d", [n_heads, n_kv_heads, d_head, n_seqs, causal, window, scale]]


def _child(shim_path, lib_path):
    shim = C.CDLL(shim_path, mode=C.RTLD_GLOBAL)
    shim.trace_name.restype = C.c_char_p
    lib = C.CDLL(lib_path)
    lib.pq_last_error_string.restype = C.c_char_p
    kinds = {"p": lambda x: C.c_void_p(x or None), "i": C.c_int32, "l": C.c_int64, "n": C.c_size_t,
             "d": lambda x: C.create_string_buffer(b"".join(struct.pack("f" if isinstance(v, float) else "i", v) for v in x))}
    out = []
    for name, *args in json.load(sys.stdin):
        shim.trace_reset()
        f = getattr(lib, name)
        f.restype = C.c_size_t if name.endswith("_bytes") else C.c_int
        rc = f(*[kinds[k](x) for k, x in args])
        failed = rc == 0 if name.endswith("_bytes") else rc != 0
        out.append([rc, lib.pq_last_error_string().decode() if failed else "", [shim.trace_name(i).decode() for i in range(shim.trace_count())]])
    json.dump(out, sys.stdout)


if __name__ == "__main__":
    _child(sys.argv[1], sys.argv[2])
