"""The 16-bit attention's runs of one unit among longer ones, again and again.

A tile of up to 128 query rows is worked on by two groups of warps that exchange their maxima and sums at a run's end; in a run
of one unit of 128 keys the second group has nothing to do, and comes to the exchange while the first one may be late in the one
before.  Contexts of one to five units in alternation make the CTAs' ranges such sequences: every launch is compared bit for bit
with the first, which is compared with 64 bits (tolerances of test_gpu_kv16.py)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["bfloat16", "float16"])
@pytest.mark.parametrize("T,G,D", [(1, 4, 128), (1, 8, 64), (17, 4, 128), (17, 7, 64), (9, 16, 128)])
def test_short_contexts_in_alternation(T, G, D, name):
    import torch
    import paper_2609_20186_gb300 as fw
    dtype = getattr(torch, name)
    torch.manual_seed(T * D + G)
    rng = np.random.default_rng(T)
    B, H, page = 700, 4, 32
    i32 = dict(dtype=torch.int32, device="cuda")
    lens = np.where(np.arange(B) % 2 == 0, rng.integers(1, 110, B), rng.integers(130, 600, B))
    lens[::7] = rng.integers(100, 600, len(lens[::7]))
    new = rng.integers(1, T + 1, B)
    blocks = -(-(600 + T) // page)
    table = torch.randperm(B * blocks, device="cuda").to(torch.int32).view(B, blocks)
    cache = torch.randn(B * blocks, 2, H, page, D, device="cuda").to(dtype)
    tl, tn = torch.tensor(lens, **i32), torch.tensor(new, **i32)
    q = torch.randn(B, T, H * G, D, device="cuda").to(dtype)
    out, first, status = torch.empty_like(q), torch.empty_like(q), torch.zeros(B, **i32)
    fw.switchsd_kv16_attention(q, cache, table, tl, tn, first, status=status)
    differ = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(300):
        fw.switchsd_kv16_attention(q, cache, table, tl, tn, out, status=status)
        differ += (out.view(torch.int16) != first.view(torch.int16)).sum() + (status != 0).sum()
    assert int(differ) == 0
    e = 2.0 ** -11 if name == "float16" else 2.0 ** -8
    for b in range(B):
        n, m = int(lens[b]), int(new[b])
        kv = cache[table[b].long()].permute(1, 2, 0, 3, 4).reshape(2, H, -1, D)[:, :, :n + m].double()
        x = torch.einsum("thgd,hjd->htgj", q[b, :m].double().view(m, H, G, D), kv[0]) * D ** -0.5
        hidden = torch.arange(n + m, device="cuda") > n + torch.arange(m, device="cuda")[:, None]
        p = torch.softmax(x.masked_fill(hidden[None, :, None], float("-inf")), -1)
        want, mag = (torch.einsum("htgj,hjd->thgd", p, v).reshape(m, H * G, D) for v in (kv[1], kv[1].abs()))
        off = (first[b, :m].double() - want).abs() - (e * want.abs() + (e + 2.0 ** -10) * mag)
        assert off.max() <= 0 and not first[b, m:].any(), b
