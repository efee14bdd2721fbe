"""The 16-bit attention's bounded waits, made to run out without any fault.

Every on-chip wait of the kernel is bounded; a warp whose wait ran out goes to the end, the copies and products in flight are
still waited for (bounded), and every row's status says SWITCHSD_ROW_TIMEOUT.  A child process sets
SWITCHSD_DIAG_ATTENTION_GIVE_UP=1: all warps but the fetching one and that of the runs then give up before their first wait, and
these two run out of time on rings that nobody empties.  The process goes on: without the variable the same calls give results.
"""
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
out = {}
i32 = dict(dtype=torch.int32, device="cuda")
for name, (B, T, n, D) in {"many": (70, 9, 1500, 128), "few": (2, 9, 150, 64), "one token": (3, 1, 900, 128), "chunk": (3, 300, 2500, 64)}.items():
    Hq, Hkv, page = 8, 2, 32
    blocks = -(-n // page)
    cache = torch.randn(B * blocks, 2, Hkv, page, D, device="cuda").to(torch.bfloat16)
    table = torch.arange(B * blocks, **i32).view(B, blocks)
    q = torch.randn(B, T, Hq, D, device="cuda").to(torch.bfloat16)
    lens, new = torch.full((B,), n - T, **i32), torch.full((B,), T, **i32)
    lens[1] = -1  # a bad row beside the good ones
    o = torch.empty_like(q)
    status = torch.full((2, B), 77, **i32)
    for i in range(2):
        fw.switchsd_kv16_attention(q, cache, table, lens, new, o, status=status[i])
    torch.cuda.synchronize()
    out[name] = dict(status=status.tolist(), sum=o.double().abs().sum().item())
c = fw.KVCache(2, 1, layers=2, heads=1, dim=64, pages=9, max_len=64, page=16, dtype=torch.bfloat16)
x = torch.randn(2, 1, 3, 64, device="cuda").to(torch.bfloat16)
c.map(torch.tensor([20, 3], **i32), torch.tensor([1, 1], **i32))
c.append(1, x[:, :, 1:2], x[:, :, 2:])
c.attend(1, x[:, :, :1].contiguous(), torch.empty_like(x[:, :, :1].contiguous()))
out["cache"] = c.attend_status.tolist()
print(json.dumps(out))
"""


def _child(env_extra):
    env = {k: v for k, v in os.environ.items() if k != "SWITCHSD_DIAG_ATTENTION_GIVE_UP"}
    r = subprocess.run([sys.executable, "-c", CHILD, ROOT], env={**env, **env_extra}, capture_output=True, text=True, timeout=600, cwd=ROOT)
    assert r.returncode == 0, r.stderr[-2000:]
    return json.loads(r.stdout.strip().splitlines()[-1])


def test_waits_that_run_out_say_so_in_every_row():
    late, plain = _child({"SWITCHSD_DIAG_ATTENTION_GIVE_UP": "1"}), _child({})
    for name in ("many", "few", "one token", "chunk"):
        assert all(s == 3 for leg in late[name]["status"] for s in leg), (name, late[name]["status"])
        for leg in plain[name]["status"]:
            assert leg == [2 if b == 1 else 0 for b in range(len(leg))], name
        assert plain[name]["sum"] > 0
    assert late["cache"] == [[0, 0], [3, 3]] and plain["cache"] == [[0, 0], [0, 0]]
