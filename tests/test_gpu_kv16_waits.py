"""The 16-bit attention's diagnostic makes waits run out; it does not say by itself that they did.

A child process sets SWITCHSD_DIAG_ATTENTION_GIVE_UP=1, which keeps the products from being issued: the warps that wait for them
run out of time.  Where there is nothing to wait for (no row has new tokens), nothing runs out, and the statuses say so; a
launch whose rows are all there says SWITCHSD_ROW_TIMEOUT."""
import json
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = r"""
import json, sys
sys.path.insert(0, sys.argv[1])
import torch
import paper_2609_20186_gb300 as fw
torch.manual_seed(0)
out = []
i32 = dict(dtype=torch.int32, device="cuda")
B, T, n, D, Hq, Hkv, page = 6, 9, 700, 128, 8, 2, 32
blocks = -(-n // page)
cache = torch.randn(B * blocks, 2, Hkv, page, D, device="cuda").to(torch.bfloat16)
table = torch.arange(B * blocks, **i32).view(B, blocks)
q = torch.randn(B, T, Hq, D, device="cuda").to(torch.bfloat16)
lens = torch.full((B,), n - T, **i32)
for new in ([0] * B, [0, -1, T + 1, 0, 0, 0], [T] * B):
    o, status = torch.full_like(q, 7.0), torch.full((B,), 77, **i32)
    fw.switchsd_kv16_attention(q, cache, table, lens, torch.tensor(new, **i32), o, status=status)
    torch.cuda.synchronize()
    out.append(dict(status=status.tolist(), zero=not o.any().item()))
print(json.dumps(out))
"""


def test_only_waits_that_ran_out_are_reported():
    env = {**os.environ, "SWITCHSD_DIAG_ATTENTION_GIVE_UP": "1"}
    r = subprocess.run([sys.executable, "-c", CHILD, ROOT], env=env, capture_output=True, text=True, timeout=600, cwd=ROOT)
    assert r.returncode == 0, r.stderr[-2000:]
    nothing, bad, late = json.loads(r.stdout.strip().splitlines()[-1])
    assert nothing["status"] == [0] * 6 and nothing["zero"]
    assert bad["status"] == [0, 2, 2, 0, 0, 0] and bad["zero"]
    assert late["status"] == [3] * 6
