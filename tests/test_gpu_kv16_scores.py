"""The 16-bit attention of scores of any size, on tiles of one token, a draft and 256 query rows.

Where a row's largest score is the largest by more than its sum's rounding (128 exact products in binary32, 2^-23 each:
2^-16 sum |q k|; 2^-14 sum |q| max |k| is taken) and 24 besides, the others' weights are below 2^10 e^-24 in all, and the result
is its value, off by the weight's rounding and its own: (2 e + e^2) |v|, e = 2^-8 (bf16) or 2^-11 (f16), and the others'
2^10 e^-24 |v| < 2^-16."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _fw():
    import paper_2609_20186_gb300 as fw
    return fw


def _setup(B, H, D, n, page, dtype, k, v):
    """A cache of rows that share their keys and values [H, n, D], each in pages of its own."""
    import torch
    blocks = -(-n // page)
    table = torch.randperm(B * blocks, device="cuda").to(torch.int32).view(B, blocks)
    cache = torch.zeros(B * blocks, 2, H, page, D, dtype=dtype, device="cuda")
    kv = torch.zeros(2, H, blocks * page, D, dtype=dtype, device="cuda")
    kv[0, :, :n], kv[1, :, :n] = k, v
    cache[table.long()] = kv.view(2, H, blocks, page, D).permute(2, 0, 1, 3, 4)
    return cache, table


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("name,by", [("bfloat16", "queries"), ("bfloat16", "scale"), ("float16", "scale")])
@pytest.mark.parametrize("T,G,D", [(1, 4, 128), (5, 8, 128), (1, 16, 64), (40, 8, 64), (34, 8, 128)])
def test_scores_of_any_size(T, G, D, name, by, sign):
    """Scores of 2^18 to 2^90, all of one sign, over several units of a CTA: binary32 numbers lie up to 2^66 apart there."""
    import torch
    dtype, e = getattr(torch, name), 2.0 ** -11 if name == "float16" else 2.0 ** -8
    torch.manual_seed(T * G + D)
    B, H, n, page = 90, 2, 900, 64
    k, v = ((torch.randn(H, n, D, device="cuda") * s + o).to(dtype) for s, o in ((1, 0.5), (40, 0)))
    cache, table = _setup(B, H, D, n, page, dtype, k, v)
    lens, new = torch.full((B,), n - T, dtype=torch.int32, device="cuda"), torch.full((B,), T, dtype=torch.int32, device="cuda")
    base = sign * torch.randn(B, T, H * G, D, device="cuda").abs()
    unseen = (torch.arange(n, device="cuda") > n - T + torch.arange(T, device="cuda")[:, None])[None, :, None, None]
    for up in (18, 22, 23, 24, 25, 26, 28, 30, 34, 40, 60, 90):
        q = (base * 2.0 ** (up if by == "queries" else 0)).to(dtype)
        scale = float(np.float32(0.09 * 2.0 ** (up if by == "scale" else 0)))
        out, status = torch.empty_like(q), torch.zeros(B, dtype=torch.int32, device="cuda")
        _fw().switchsd_kv16_attention(q, cache, table, lens, new, out, scale=scale, status=status)
        assert not status.any() and out.isfinite().all(), up
        x = torch.einsum("bthgd,hjd->bthgj", q.double().view(B, T, H, G, D), k.double()).masked_fill(unseen, float("-inf"))
        best = x.topk(2, -1)
        apart = 2.0 ** -14 * q.double().abs().sum(-1).view(B, T, H, G) * k.double().abs().amax() + 24 / scale
        sure = best.values[..., 0] - best.values[..., 1] > apart
        assert sure.double().mean() > 0.5
        want = v.double()[torch.arange(H, device="cuda")[None, None, :, None], best.indices[..., 0]]
        off = (out.double().view_as(want) - want).abs() - (2 * e + e * e) * want.abs()
        assert off[sure].max() <= 2.0 ** -16, up


@pytest.mark.parametrize("name", ["bfloat16", "float16"])
@pytest.mark.parametrize("T,G,D", [(1, 4, 128), (5, 8, 64), (40, 8, 128)])
def test_large_scores_of_some_rows_from_some_key_on(T, G, D, name):
    """Every third head's queries are of ordinary size, and the scores of the others before the 500th key.  (The ordinary ones:
    tolerances of test_gpu_kv16.py.)"""
    import torch
    dtype, e = getattr(torch, name), 2.0 ** -11 if name == "float16" else 2.0 ** -8
    torch.manual_seed(T + D)
    B, H, n, page = 90, 2, 1100, 32
    k, v = ((torch.randn(H, n, D, device="cuda") * s + o).to(dtype) for s, o in ((1, 0.5), (4, 0)))
    up, down = (2.0 ** 30, 2.0 ** -30) if name == "bfloat16" else (2.0 ** 14, 2.0 ** -12)  # (f16: what its numbers reach, and the scale)
    scale = float(np.float32(0.09)) if name == "bfloat16" else float(np.float32(0.09 * 2.0 ** 12))
    k[:, :500] *= down
    cache, table = _setup(B, H, D, n, page, dtype, k, v)
    lens, new = torch.full((B,), n - T, dtype=torch.int32, device="cuda"), torch.full((B,), T, dtype=torch.int32, device="cuda")
    q = torch.randn(B, T, H * G, D, device="cuda").abs()
    plain = torch.arange(H * G, device="cuda") % 3 == 0
    q[:, :, ~plain] *= up
    if name == "float16":
        q[:, :, plain] *= 2.0 ** -12
    q = q.clamp(max=torch.finfo(dtype).max).to(dtype)  # (4 * 2^14 is no f16 number)
    out, status = torch.empty_like(q), torch.zeros(B, dtype=torch.int32, device="cuda")
    _fw().switchsd_kv16_attention(q, cache, table, lens, new, out, scale=scale, status=status)
    assert not status.any() and out.isfinite().all()
    unseen = (torch.arange(n, device="cuda") > n - T + torch.arange(T, device="cuda")[:, None])[None, :, None, None]
    x = torch.einsum("bthgd,hjd->bthgj", q.double().view(B, T, H, G, D), k.double()).masked_fill(unseen, float("-inf"))
    best = x.topk(2, -1)
    apart = 2.0 ** -14 * q.double().abs().sum(-1).view(B, T, H, G) * k.double().abs().amax() + 24 / scale
    sure = (best.values[..., 0] - best.values[..., 1] > apart) & ~plain.view(H, G)
    assert sure.double().mean() > 0.3
    want = v.double()[torch.arange(H, device="cuda")[None, None, :, None], best.indices[..., 0]]
    off = (out.double().view_as(want) - want).abs() - (2 * e + e * e) * want.abs()
    assert off[sure].max() <= 2.0 ** -16
    p = torch.softmax(x * scale, -1)
    want, mag = (torch.einsum("bthgj,hjd->bthgd", p, y.double()).reshape(B, T, H * G, D)[:, :, plain] for y in (v, v.abs()))
    off = (out.double()[:, :, plain] - want).abs() - (e * want.abs() + (e + 2.0 ** -10) * mag)
    assert off.max() <= 0


@pytest.mark.parametrize("base", [24, 25, 26, 27, 28])
@pytest.mark.parametrize("T,G", [(1, 4), (33, 8)])
def test_half_weights_stay_in_range(T, G, base):
    """f16 weights of scores near 2^24 to 2^28 in binary logarithms, where 15 more than the reference is no number: every unit's
    largest score lies one to three of their steps (at most 16) above the last one's, and all but these far below.  The result
    lies between the smallest and the largest value, and is the last one's where that is 2^10 steps ahead."""
    import torch
    torch.manual_seed(base)
    rng = np.random.default_rng(base)
    B, H, D, page, n = 80, 2, 64, 64, 1280
    step = 2 ** (base - 23)
    scale = float(np.float32(np.log(2)))  # times log2 e: 1, rounded to binary32
    q = torch.zeros(B, T, H * G, D, dtype=torch.float16, device="cuda")
    q[..., 0], q[..., 1] = 2.0 ** (base - 14), float(step)
    for last in (False, True):
        k = torch.zeros(H, n, D, dtype=torch.float16, device="cuda")
        k[..., 0] = -2.0 ** 14
        tops = np.arange(0, n - T, 128) + rng.integers(0, 100, len(range(0, n - T, 128)))
        k[:, tops, 0] = 2.0 ** 14
        k[:, tops, 1] = torch.from_numpy(np.cumsum(rng.integers(1, max(2, min(4, 17 // step + 1)), len(tops)))).to(k)
        if last:
            k[:, tops[-1], 1] += 1024
        v = (torch.rand(H, n, D, device="cuda") + 1).to(torch.float16)
        cache, table = _setup(B, H, D, n, page, torch.float16, k, v)
        i32 = dict(dtype=torch.int32, device="cuda")
        out, status = torch.empty_like(q), torch.zeros(B, **i32)
        _fw().switchsd_kv16_attention(q, cache, table, torch.full((B,), n - T, **i32), torch.full((B,), T, **i32), out, scale=scale, status=status)
        assert not status.any() and (out >= 0.999).all() and (out <= 2.002).all()  # (weights and results rounded, 2^-11 each)
        if last:
            want = v[:, tops[-1]].double()[None, None, :, None]
            assert ((out.double().view(B, T, H, G, D) - want).abs() <= (2.0 ** -10 + 2.0 ** -22) * want).all()


@pytest.mark.parametrize("name", ["bfloat16"])
@pytest.mark.parametrize("T,G", [(1, 4), (40, 8)])
def test_scales_of_any_size(T, G, name):
    """Small scales of large products, subnormal ones among them, of either sign: the scores are of ordinary size.  (Sums off by
    2^-16 sum |q k|, 2^-10 of a score; a subnormal scale has 2^-12 of itself; then as in test_gpu_kv16.py.)"""
    import torch
    torch.manual_seed(T)
    B, H, D, n, page = 5, 2, 64, 700, 64
    k = torch.randn(H, n, D, device="cuda").to(torch.bfloat16)
    v = torch.randn(H, n, D, device="cuda").to(torch.bfloat16)
    cache, table = _setup(B, H, D, n, page, torch.bfloat16, k * 2.0 ** 58, v)
    lens, new = torch.full((B,), n - T, dtype=torch.int32, device="cuda"), torch.full((B,), T, dtype=torch.int32, device="cuda")
    q = torch.randn(B, T, H * G, D, device="cuda").to(torch.bfloat16)
    unseen = (torch.arange(n, device="cuda") > n - T + torch.arange(T, device="cuda")[:, None])[None, :, None, None]
    x = torch.einsum("bthgd,hjd->bthgj", q.double().view(B, T, H, G, D), k.double())
    lifted = (q.float() * 2.0 ** 63).to(torch.bfloat16)
    for factor in (0.1, -0.1, 1e-4, -1e-4):  # (of 2^-121)
        p = torch.softmax((x * factor).masked_fill(unseen, float("-inf")), -1)
        want, mag = (torch.einsum("bthgj,hjd->bthgd", p, y.double()) for y in (v, v.abs()))
        out, scale = torch.empty_like(q), float(np.float32(factor * 2.0 ** -121))
        assert abs(scale / (factor * 2.0 ** -121) - 1) < 2.0 ** -12
        _fw().switchsd_kv16_attention(lifted, cache, table, lens, new, out, scale=scale)
        off = (out.double().view_as(want) - want).abs() - (2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -9) * mag)
        assert off.max() <= 0, factor
