"""switchsd_logprobs with more than three and more than twelve positions an SM, which CTAs of 256 and of 128 threads take: several
batches of loads a CTA, bounds that are raised on the way, every element type.  All positions are compared with 64 bits.

Tolerances.  A thread's sum has at most 8 additions a batch in a chain, 2 that join them, one a batch (64 batches at the most)
and 10 joins of threads: 84 roundings of 2^-24; a weight is off by 2^-21 of itself (2^-22 the instruction, the rest its
argument's); a new maximum scales a sum by a factor off by 2^-22, and 16 of these count (in rows that rise without end what was
before is gone after one).  So S by 2^-21 + 84 2^-24 + 16 2^-22 < 2^-16.6 of itself, the sum of weights times logarithms alike,
and their quotient, at most ln V, by twice that.  lse and log probabilities: besides, 2^-22 of themselves."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
S = 2.0 ** -16.6


@pytest.mark.parametrize("top", [0, 5, 9, 20, 32])
@pytest.mark.parametrize("name", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("B,T,V,lead", [(2, 240, 70001, 3), (5, 380, 70001, 1), (4, 500, 33333, 0)])
def test_many_positions(B, T, V, lead, name, top):
    import torch
    import paper_2609_20186_gb300 as fw
    dtype = getattr(torch, name)
    torch.manual_seed(B * T + V)
    inf, low = float("inf"), torch.finfo(dtype).min
    buf = torch.full((lead + B * (T * (V + 1) + 3),), float("nan"), dtype=dtype, device="cuda")
    x = buf[lead:].as_strided((B, T, V), (T * (V + 1) + 3, V + 1, 1))
    at = torch.arange(V, device="cuda")
    for b in range(B):
        y = torch.randn(T, V, device="cuda") * 2
        y.scatter_add_(1, torch.randint(0, V, (T, 8), device="cuda"), torch.rand(T, 8, device="cuda") * 12)
        y[0], y[1], y[2], y[3], y[4] = at / 97.0, -at / 97.0, 3.25, low, -inf  # each one a new best, none, all alike, all but one, nothing
        y[3, 777] = 1.0
        y[5] = torch.round(torch.randn(V, device="cuda"))
        y[6].masked_fill_(torch.rand(V, device="cuda") < 0.999, -inf)
        y[7].masked_fill_(torch.rand(V, device="cuda") < 0.999, low)
        y[8].masked_fill_(torch.rand(V, device="cuda") < 0.5, float("nan"))
        y[9] = float("nan")
        y[10] = torch.floor(at / 1000.0)  # rising, many alike
        y[11, :-40], y[12, 40:] = -inf, -inf
        x[b] = y.to(dtype)
    new = torch.randint(13, T + 1, (B,), device="cuda")
    new[0] = T
    temps = torch.tensor([0.7, 0.0, 1.0, 1.25, 0.55][:B], device="cuda")
    tokens = torch.randint(-1, V + 1, (B, T), device="cuda").to(torch.int32)
    f32 = dict(dtype=torch.float32, device="cuda")
    o = dict(entropy=torch.full((B, T), 77.0, **f32), lse=torch.full((B, T), 77.0, **f32), logprob=torch.full((B, T), 77.0, **f32), prob=torch.full((B, T), 77.0, **f32))
    if top:
        o.update(top_ids=torch.full((B, T, top), 77, dtype=torch.int32, device="cuda"), top_logprobs=torch.full((B, T, top), 77.0, **f32))
    again = {k: v.clone() for k, v in o.items()}
    call = dict(tokens=tokens, new_lens=new.to(torch.int32) - 1, new_add=1, temperature=temps)
    fw.switchsd_logprobs(x, **call, **o)
    fw.switchsd_logprobs(x, **call, **again)
    assert all(torch.equal(o[k], again[k]) for k in o)
    ln_v = float(np.log(V))
    for b in range(B):
        n = int(new[b])
        assert (o["entropy"][b, n:] == 0).all() and (o["lse"][b, n:] == -inf).all() and (o["logprob"][b, n:] == -inf).all() and (o["prob"][b, n:] == 0).all()
        if top:
            assert (o["top_ids"][b, n:] == -1).all() and (o["top_logprobs"][b, n:] == -inf).all()
        for t0 in range(0, n, 64):
            t1 = min(n, t0 + 64)
            z = x[b, t0:t1].double() + 0.0
            z = torch.where(z.isnan(), -inf, z)
            order = torch.sort(z, dim=1, descending=True, stable=True)
            none = order.values[:, :1] == -inf
            if temps[b] == 0:
                lp = torch.full_like(z, -inf).scatter_(1, order.indices[:, :1], 0.0).masked_fill(none, -inf)
                lse, entropy = order.values[:, 0], torch.zeros(t1 - t0, dtype=torch.float64, device="cuda")
            else:
                w = z / temps[b].double()
                lse = torch.logsumexp(w, 1)
                lp = (w - torch.where(none, 0.0, lse[:, None])).masked_fill(z == -inf, -inf)
                entropy = -torch.where(lp == -inf, 0.0, lp * lp.exp()).sum(1)
            lp = torch.where(lp < -3.5e38, -inf, lp)  # beyond binary32, which the outputs are held in

            def near(got, want, off):
                got = got.double()
                return bool(((got == want) | ((got - want).abs() <= off)).all())
            assert near(o["lse"][b, t0:t1], lse, S + 2.0 ** -22 * lse.abs()), (b, t0)
            assert near(o["entropy"][b, t0:t1], entropy, S + (2 * S + 2.0 ** -20) * ln_v), (b, t0)
            token = tokens[b, t0:t1].long()
            inside = (token >= 0) & (token < V)
            want = torch.where(inside, lp.gather(1, token.clamp(0, V - 1)[:, None])[:, 0], -inf)
            assert near(o["logprob"][b, t0:t1], want, S + 2.0 ** -22 * want.abs()), (b, t0)
            size = torch.where(want == -inf, 0.0, want.abs())
            assert near(o["prob"][b, t0:t1], want.exp(), (2 * S + 2.0 ** -21 * size) * want.exp() + 2.0 ** -126), (b, t0)
            if top:
                gone = order.values[:, :top] == -inf
                ids = torch.where(gone, -1, order.indices[:, :top])
                assert torch.equal(o["top_ids"][b, t0:t1].long(), ids), (b, t0)
                want = torch.where(gone, -inf, lp.gather(1, order.indices[:, :top]))
                assert near(o["top_logprobs"][b, t0:t1], want, S + 2.0 ** -22 * want.abs()), (b, t0)
