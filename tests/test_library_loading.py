"""The operators' argument types are known whichever way the library was loaded first (without them ctypes hands structures over by value and cuts sizes to 32 bits)."""
import os
import subprocess
import sys

import pytest

import paper_2401_15077_amd as pkg

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("first", ["pkg.load_library(need_gpu_runtime=False)", "pkg.load_library()", "None"])
def test_operators_are_declared(first):
    if not os.path.exists(pkg.LIB_PATH):
        from paper_2401_15077_amd import build
        build.build()
    code = f"""
import ctypes
import paper_2401_15077_amd as pkg
import torch
first = {first}
from paper_2401_15077_amd import operators as ops
lib = ops._library()
assert first is None or lib is first
for name in ("eagle_rope_plan_init", "eagle_rope", "eagle_chunk_attention_workspace", "eagle_chunk_attention", "eagle_apply_logit_rules", "eagle_set_rope", "eagle_set_attention",
             "eagle_set_logit_rules"):
    assert getattr(lib, name).argtypes, name
assert lib.eagle_chunk_attention_workspace.restype is ctypes.c_size_t
"""
    done = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-1500:]
