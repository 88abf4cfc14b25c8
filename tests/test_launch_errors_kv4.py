"""A failed launch of the 4-bit cache's calls is reported, and what depends on it
is not launched: the same stub of the HIP runtime as for the other calls."""

import os
import shutil
import subprocess
import sys

import pytest

from tests.test_launch_errors import ROOT, STUB

CHILD = r"""
import ctypes, sys
stub = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
from paper_2606_04446_amd import d2sd
P = ctypes.c_void_p(1 << 20)
cache = d2sd.Kv4Pointers(*(1 << 20,) * 4)
attn = lambda **kw: d2sd.AttnArgs(**{**dict(
    batch=2, num_qo_heads=8, num_kv_heads=2, head_dim=128, page_size=16, dtype=d2sd.BF16, stage=d2sd.STAGE_CASCADE,
    total_nodes=40, max_nodes=20, max_ctx_len=30000, num_pages=2048, max_pages=2000, mask_words=1, q=1 << 20, page_table=1 << 20,
    ctx_len=1 << 20, k_tree=1 << 20, v_tree=1 << 20, node_indptr=1 << 20, anc_mask=1 << 20, out=1 << 20, lse=None), **kw})
def attend(**kw):
    a = attn(**kw)
    n = ctypes.c_size_t()
    assert d2sd._ws_size_kv4(ctypes.byref(a), ctypes.byref(n)) == d2sd.OK
    return d2sd._cascade_kv4(ctypes.byref(a), ctypes.byref(cache), P, n.value, None)
calls = {
    "append": (2, lambda: d2sd._append_kv4(2, 2, 128, 16, d2sd.BF16, 64, 32, 100, P, 300, 200, P, P, P, P, ctypes.byref(cache), None)),
    "append, few rows": (1, lambda: d2sd._append_kv4(2, 2, 128, 16, d2sd.BF16, 64, 32, 100, P, 30, 20, P, P, P, P, ctypes.byref(cache), None)),
    "commit": (1, lambda: d2sd._commit_kv4(2, 8, 2, 128, 16, d2sd.BF16, 64, 32, 100, P, 40, P, P, P, P, P, P, ctypes.byref(cache), None)),
    "read": (1, lambda: d2sd._read_kv4(2, 2, 128, 16, d2sd.BF16, 64, 32, P, 30, 20, None, P, ctypes.byref(cache), P, P, None)),
    "attention": (2, attend), "attention, fp32": (2, lambda: attend(dtype=d2sd.F32)),
    "attention, short contexts": (1, lambda: attend(max_ctx_len=100)),
    "attention, short contexts cut": (2, lambda: attend(max_ctx_len=500, kv_split=64)),
    "attention, tree alone": (1, lambda: attend(stage=d2sd.STAGE_TREE)),
}
for name, (launches, call) in calls.items():
    for n in range(launches + 1):
        stub.stub_reset(n)
        got = (call(), stub.stub_launches())
        assert got == ((d2sd.OK, launches) if n == 0 else (d2sd.ERR_HIP, n)), (name, n, got)
print("ok")
"""


@pytest.mark.skipif(shutil.which("gcc") is None, reason="needs a C compiler")
def test_a_failed_launch_is_reported(tmp_path):
    src, lib = tmp_path / "stub.c", tmp_path / "libstub.so"
    src.write_text(STUB)
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(lib), str(src)], check=True)
    r = subprocess.run([sys.executable, "-c", CHILD, str(lib)], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip().endswith("ok"), r.stdout + r.stderr[-2000:]
