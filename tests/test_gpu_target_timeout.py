"""The many-row attention's bounded waits, made to run out without any fault.

Every on-chip wait of the kernel is bounded; when one runs out its warps go on without waiting, the copies and products in
flight are still waited for (bounded), the partial results are marked, and every row's status says SWITCHSD_ROW_TIMEOUT.  A
child process sets SWITCHSD_DIAG_ATTENTION_GIVE_UP=1: the consuming warps then give up before their first wait, and the fetching
warp runs out of time on the ring that nobody empties.  The process goes on: the next calls give what they give without it.
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
for name, (B, T, n) in {"many": (70, 9, 1500), "few": (2, 9, 150), "one token": (3, 1, 900)}.items():
    Hq, Hkv, D, page = 8, 2, 128, 32
    blocks = -(-n // page)
    i32 = dict(dtype=torch.int32, device="cuda")
    cache = torch.zeros(B * blocks, Hkv, fw.switchsd_kv4_bytes(page, D), dtype=torch.uint8, device="cuda")
    table = torch.arange(B * blocks, **i32).view(B, blocks)
    slots = (table[:, :, None] * page + torch.arange(page, **i32)).reshape(B, -1)[:, :n].contiguous()
    x = torch.randn(2, B, n, Hkv, D, device="cuda").to(torch.bfloat16)
    fw.switchsd_kv4_append(x[0], x[1], slots, cache, page=page)
    q = torch.randn(B, T, Hq, D, device="cuda").to(torch.bfloat16)
    lens, new = torch.full((B,), n - T, **i32), torch.full((B,), T, **i32)
    lens[1] = -1  # a bad row beside the good ones
    o = torch.empty_like(q)
    status = torch.full((2, B), 77, **i32)
    for i in range(2):
        fw.switchsd_kv4_attention(q, cache, table, lens, new, o, page=page, status=status[i])
    torch.cuda.synchronize()
    out[name] = dict(status=status.tolist(), sum=o.double().abs().sum().item())
print(json.dumps(out))
"""


def _child(env_extra):
    env = dict(os.environ)
    env.pop("SWITCHSD_DIAG_ATTENTION_GIVE_UP", None)
    env.update(env_extra)
    r = subprocess.run([sys.executable, "-c", CHILD, ROOT], env=env, capture_output=True, text=True, timeout=600, cwd=ROOT)
    assert r.returncode == 0, r.stderr[-2000:]
    return json.loads(r.stdout.strip().splitlines()[-1])


def test_waits_that_run_out_say_so_in_every_row():
    late, plain = _child({"SWITCHSD_DIAG_ATTENTION_GIVE_UP": "1"}), _child({})
    for name in ("many", "few"):
        assert all(s == 3 for leg in late[name]["status"] for s in leg), late[name]["status"]
    for out, names in ((late, ["one token"]), (plain, ["many", "few", "one token"])):
        for name in names:
            for leg in out[name]["status"]:
                assert [s for s in leg] == [2 if b == 1 else 0 for b in range(len(leg))]
    assert late["one token"] == plain["one token"]


CACHE = r"""
import json, sys
sys.path.insert(0, sys.argv[1])
import torch
import paper_2609_20186_gb300 as fw
torch.manual_seed(0)
B, T, H, Hq, D = 3, 9, 1, 4, 64
i32 = dict(dtype=torch.int32, device="cuda")
c = fw.KVCache(B, T, layers=3, heads=H, dim=D, pages=5, max_len=64, page=16)
x = torch.randn(B, T, Hq + 2 * H, D, device="cuda").to(torch.bfloat16)
o = torch.empty(B, T, Hq, D, dtype=x.dtype, device="cuda")
c.map(torch.tensor([3, 60, 0], **i32), torch.tensor([9, 9, 1], **i32))  # the second row asks for five pages: one too many
for layer in (0, 2):
    c.append(layer, x[:, :, Hq:Hq + H], x[:, :, Hq + H:])
    c.attend(layer, x[:, :, :Hq], o)
print(json.dumps(dict(map=c.status.tolist(), attend=c.attend_status.tolist())))
"""


def test_a_caches_layers_keep_their_statuses():
    def child(env_extra):
        env = {k: v for k, v in os.environ.items() if k != "SWITCHSD_DIAG_ATTENTION_GIVE_UP"}
        r = subprocess.run([sys.executable, "-c", CACHE, ROOT], env={**env, **env_extra}, capture_output=True, text=True, timeout=600, cwd=ROOT)
        assert r.returncode == 0, r.stderr[-2000:]
        return json.loads(r.stdout.strip().splitlines()[-1])
    assert child({}) == dict(map=[0, 1, 0], attend=[[0, 2, 0], [0, 0, 0], [0, 2, 0]])
    assert child({"SWITCHSD_DIAG_ATTENTION_GIVE_UP": "1"}) == dict(map=[0, 1, 0], attend=[[3, 3, 3], [0, 0, 0], [3, 3, 3]])
