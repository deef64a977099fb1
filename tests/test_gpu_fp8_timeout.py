"""The wind-down of the attention over a cache in 8 bits: with every wait a single test (the library's short-wait build, in a child
process) both kernels give up, report it, wait out their own copies and MMAs and return, and the context stays usable.  Nothing
faults and nothing waits for what never comes: the warps of a row leave together."""
import json
import os
import subprocess
import sys

import pytest
import torch

from paper_2606_31315_gb300 import _build

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = r"""
import json, sys
sys.path.insert(0, sys.argv[1])
import torch
from paper_2606_31315_gb300 import _build
_build.LIB = _build.TEST_LIB            # the short-wait build only
import paper_2606_31315_gb300 as bp
out = []
for ctx, new, hq, hkv, d, seqs in ((0, 700, 32, 8, 128, 1), (5000, 1, 32, 8, 128, 1), (100, 300, 8, 2, 64, 3), (2000, 20, 8, 2, 64, 40),
                                   (300, 16, 32, 8, 128, 100)):
    n = ctx + new
    pages = -(-n // 64)
    cache = [torch.randn(seqs * pages * 64, hkv, d, device="cuda").to(torch.float8_e4m3fn) for _ in range(2)]
    scale = [torch.full((seqs * pages, hkv), 127, dtype=torch.uint8, device="cuda") for _ in range(2)]
    table = torch.arange(seqs * pages, device="cuda", dtype=torch.int32).view(seqs, pages)
    q = torch.randn(seqs * new, hq, d, device="cuda").to(torch.bfloat16)
    cu = [torch.arange(seqs + 1, device="cuda", dtype=torch.int32) * x for x in (new, n)]
    ws = bp.workspace(bp.chunk_attention_workspace_size(seqs, seqs * new, hq, hkv, d), "cuda")
    bp.chunk_attention_paged_fp8(q, cache[0], scale[0], cache[1], scale[1], *cu, table, 64, new, n, ws=ws)
    out.append(bp.get_status(ws))
x = torch.arange(1 << 20, device="cuda", dtype=torch.float64)
print(json.dumps({"status": out, "context_ok": float(x.sum()) == float((1 << 20) * ((1 << 20) - 1) // 2)}))
"""


def test_expired_waits_report_timeout_and_leave_the_context_usable():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    _build.build()
    res = subprocess.run([sys.executable, "-c", CHILD, ROOT], capture_output=True, text=True, timeout=600)
    assert res.returncode == 0, res.stderr[-3000:]
    got = json.loads([ln for ln in res.stdout.splitlines() if ln.startswith("{")][-1])
    assert got == {"status": [5] * 5, "context_ok": True}, got  # BP_ERR_TIMEOUT
