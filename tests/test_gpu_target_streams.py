"""Calls on a stream that is given, not the current one: what they take from torch for themselves is ordered by that stream, and
work on the current stream while they wait or run does not reach their results."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

CYCLES = 20_000_000  # some ten milliseconds


def _inputs(name):
    """call(out, stream) of an operator, and fresh outputs."""
    import torch
    import paper_2609_20186_gb300 as fw
    from paper_2609_20186_gb300 import binding as bd
    torch.manual_seed(0)
    i32 = dict(dtype=torch.int32, device="cuda")
    if name in ("attention", "drafts"):
        B, T, Hq, Hkv, D, page = 4, 1 if name == "attention" else 9, 8, 2, 128, 32
        n = 3000
        blocks = -(-n // page)
        cache = torch.zeros(B * blocks, Hkv, fw.switchsd_kv4_bytes(page, D), dtype=torch.uint8, device="cuda")
        table = torch.arange(B * blocks, **i32).view(B, blocks)
        slots = (table[:, :, None] * page + torch.arange(page, **i32)).reshape(B, -1)[:, :n].contiguous()
        x = torch.randn(2, B, n, Hkv, D, device="cuda").to(torch.bfloat16)
        fw.switchsd_kv4_append(x[0], x[1], slots, cache, page=page)
        q = torch.randn(B, T, Hq, D, device="cuda").to(torch.bfloat16)
        lens, new = torch.full((B,), n - T, **i32), torch.full((B,), T, **i32)
        return (lambda o, s: fw.switchsd_kv4_attention(q, cache, table, lens, new, o, page=page, stream=s)), lambda: torch.empty_like(q)
    if name == "logits":
        B, T, V, cap = 8, 5, 32000, 4096
        x = torch.randn(B, T, V, device="cuda")
        ctx, lens = torch.randint(0, V, (B, cap), **i32), torch.full((B,), cap, **i32)
        rep = torch.full((B,), 1.3, device="cuda")
        return (lambda o, s: fw.switchsd_logits(x, ctx_tokens=ctx, ctx_lens=lens, rep=rep, out=o, stream=s)), lambda: torch.empty_like(x)
    ctx, lens = torch.randint(0, 50, (4, 8192), **i32), torch.full((4,), 8000, **i32)
    return (lambda o, s: bd.switchsd_copy_labels(ctx, lens, o, stream=s)), lambda: torch.zeros(4, 8192, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("name", ["attention", "drafts", "logits", "labels"])
def test_a_call_on_another_stream_keeps_its_workspace(name, monkeypatch):
    import torch
    call, fresh = _inputs(name)
    want = fresh()
    call(want, None)
    side, taken, real = torch.cuda.Stream(), [], torch.empty

    def empty(*a, **k):
        t = real(*a, **k)
        taken.append((torch.cuda.current_stream().cuda_stream, t.numel()))
        return t
    torch.cuda.synchronize()
    got = fresh()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(CYCLES)
    with monkeypatch.context() as m:
        m.setattr(torch, "empty", empty)
        call(got, side)
    assert len(taken) == 1 and taken[0][0] == side.cuda_stream
    for _ in range(300):  # before and while the call runs: blocks of its workspace's size, filled
        torch.empty(taken[0][1], dtype=torch.uint8, device="cuda").fill_(0xff)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_a_cache_on_its_own_stream():
    """Appends, attention and reads of a cache with a stream of its own, with the current stream busy, and the cache dropped
    before its calls are done."""
    import torch
    import paper_2609_20186_gb300 as fw
    torch.manual_seed(0)
    B, T, H, Hq, D, n = 3, 64, 2, 4, 128, 192
    i32 = dict(dtype=torch.int32, device="cuda")
    x = torch.randn(3, B, T, Hq + 2 * H, D, device="cuda").to(torch.bfloat16)
    new = torch.full((B,), T, **i32)
    lens = [torch.full((B,), T * i, **i32) for i in range(3)]

    def go(stream):
        cache = fw.KVCache(B, T, layers=1, heads=H, dim=D, pages=B * (n // 16), max_len=n, page=16, stream=stream)
        taken = [t.data_ptr() for t in (cache.data, cache.workspace)]
        if stream is not None:
            with torch.cuda.stream(stream):
                torch.cuda._sleep(CYCLES)
        outs = []
        for i in range(3):
            cache.map(lens[i], new)
            cache.append(0, x[i][:, :, Hq:Hq + H], x[i][:, :, Hq + H:])
            outs.append(cache.attend(0, x[i][:, :, :Hq], torch.empty(B, T, Hq, D, dtype=x.dtype, device="cuda")))
            outs.extend(cache.read(0, cache.slots))
        sizes = [cache.data.numel(), cache.workspace.numel()]
        del cache
        for _ in range(200):
            for m in sizes:
                t = torch.empty(m, dtype=torch.uint8, device="cuda").fill_(0xff)
                assert stream is None or t.data_ptr() not in taken or stream.query()
        if stream is not None:
            torch.cuda.current_stream().wait_stream(stream)
        return outs
    want = go(None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = go(side)
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    assert np.isfinite(got[0].float().cpu().numpy()).all()
