"""What calls launch, without a GPU: a child process whose HIP runtime is tests/launch_spy.c runs a piece of Python and gives
back the launches and the LDS that was asked for.  Pointers handed to the calls are never used."""
from __future__ import annotations

import json
import os
import re
import subprocess
import sys
import tempfile
from collections import namedtuple

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)

Launch = namedtuple("Launch", "kernel grid threads lds")
Attr = namedtuple("Attr", "kernel lds")

PRELUDE = """
import ctypes, json, sys
sys.path[:0] = [{root!r}, {here!r}]
spy = ctypes.CDLL({spy!r}, mode=ctypes.RTLD_GLOBAL)
spy.spy_text.restype = ctypes.c_char_p
from paper_2506_17286_amd import binding as B
def events():
    t = spy.spy_text().decode()
    spy.spy_clear()
    return t
FAKE, R = 1 << 20, ctypes.byref
out = []
"""


def run(code: str):
    """Runs `code` (which has B, FAKE, R and events() and appends to `out`) and returns `out`."""
    with tempfile.TemporaryDirectory() as tmp:
        lib = os.path.join(tmp, "spy.so")
        subprocess.run(["gcc", "-shared", "-fPIC", "-O1", "-o", lib, os.path.join(HERE, "launch_spy.c")], check=True, capture_output=True, text=True)
        # no device is visible to the child: should a launch reach a real runtime, it fails there
        env = dict(os.environ, HIP_VISIBLE_DEVICES="-1", ROCR_VISIBLE_DEVICES="-1")
        script = PRELUDE.format(root=ROOT, here=HERE, spy=lib) + code + "\nprint('OUT ' + json.dumps(out))\n"
        p = subprocess.run([sys.executable, "-c", script], capture_output=True, text=True, timeout=300, env=env)
    assert p.returncode == 0, (p.stdout + p.stderr)[-3000:]
    return json.loads(p.stdout.rsplit("OUT ", 1)[1])


def parse(text: str):
    got = []
    for line in text.splitlines():
        what, name, *n = line.split()
        n = [int(v) for v in n]
        got.append(Attr(name, n[0]) if what == "attr" else Launch(name, tuple(n[:3]), n[3], n[4]))
    return got


def attention_kernel(name: str):
    """(type, key bytes, latent columns, cut, edge) of an 8-bit attention kernel's (mangled) name, or None"""
    m = re.search(r"mx_attn_kernelI(f|DF16b|u6__bf16)Li(\d+)ELi(\d+)ELi\d+ELi\d+ELb([01])ELb([01])E", name)
    return (("f32" if m[1] == "f" else "bf16"), int(m[2]), int(m[3]), m[4] == "1", m[5] == "1") if m else None
