"""The package under a torch without a type of packed e2m1 codes."""
import os
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")

import test_attention_abi as t  # noqa: E402

b = t.b              # the fixture that builds and loads the binding

WITHOUT = """
import torch
if hasattr(torch, "float4_e2m1fn_x2"):
    del torch.float4_e2m1fn_x2
import paper_2410_06270_amd as mc
assert mc.pack_sizes(2, 256, 512, [2, 3], 64)
assert mc.kv_page_bytes(16, 2, 64) == 4096 and mc.kv_page_bytes(16, 2, 64, torch.float8_e4m3fn) == 2048
for other in (None, torch.uint8, torch.float16):
    try:
        mc.kv_page_bytes(16, 2, 64, other)
    except AssertionError:
        continue
    raise SystemExit("%s was taken for a cache's type" % other)
print("whole")
"""


def test_import_without_a_4_bit_type(b):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", WITHOUT], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip().endswith("whole"), r.stderr[-2000:]


def test_types_of_a_cache(b):
    assert b.kv_page_bytes(16, 2, 64, torch.bfloat16) == 4096
    if hasattr(torch, "float4_e2m1fn_x2"):
        assert b.kv_page_bytes(16, 2, 64, torch.float4_e2m1fn_x2) == 1088
