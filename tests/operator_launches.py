"""What a call of the operators on tokens enqueues, seen without a GPU (launch_recorder.py): sizes and strides, which the entry points read on the host, are
given as lists.  Floating arguments are left out: they travel in registers of their own."""
from __future__ import annotations

import json
import subprocess
import sys

import launch_recorder

_CHILD = """
import ctypes, json, struct, sys
shim = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
lib = ctypes.CDLL(sys.argv[2])
shim.shim_launches.restype = ctypes.c_char_p
out = []
for name, args in json.load(sys.stdin):
    shim.shim_clear()
    fn = getattr(lib, name)
    fn.restype = ctypes.c_size_t if name.endswith("_bytes") else ctypes.c_int
    rc = fn(*[ctypes.c_char_p(struct.pack("%dq" % len(a), *a)) if isinstance(a, list) else ctypes.c_size_t(a & (2 ** 64 - 1)) for a in args])
    out.append([rc, [[int(x) for x in line.split(" ", 3)[:2]] + [line.split(" ", 3)[3]] for line in shim.shim_launches().decode().splitlines()]])
print(json.dumps(out))
"""


def shape(rows, total, heads, dk, dv, q=0, k=0, v=0):
    """A tcuscan_attention_shape_t of dense arrays."""
    q, k, v = q or heads, k or heads, v or heads
    return [rows, total, heads, dk, dv, q, k, v, q * dk, dk, k * dk, dk, v * dv, dv, heads * dv, dv, q * dk, dk, k * dk, dk, v * dv, dv]


def launches(shim: str, calls):
    """calls: [(entry point, [integers and lists of them])].  Returns for each (result, [(kernel, workgroups, threads of one)])."""
    done = subprocess.run([sys.executable, "-c", _CHILD, shim, launch_recorder.LIB], input=json.dumps(calls), capture_output=True, text=True, timeout=120)
    assert done.returncode == 0, done.stderr
    return [(rc, [(launch_recorder._plain(name), grid, block) for grid, block, name in rows]) for rc, rows in json.loads(done.stdout)]
