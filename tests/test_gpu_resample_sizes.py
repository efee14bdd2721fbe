"""switchsd_resample where logits over temperatures are large, and where masks leave nothing to bound the search by: the token is
binary64's (sampling_ref.py), whatever binary32 can tell apart there."""
import numpy as np
import pytest

from tests import sampling_ref as ref

pytestmark = pytest.mark.gpu


def _call(x, name, draft, temps, seeds, ctx, *, lse=None, xq=None, q_lse=None):
    """Every row's draft of one token is rejected; the token appended in its place."""
    import torch
    import paper_2609_20186_gb300 as fw
    dtype = dict(bf16=torch.bfloat16, f32=torch.float32)[name]
    B, V = x.shape
    f32 = lambda a: None if a is None else torch.from_numpy(np.asarray(a, np.float32)).cuda()
    logits = torch.from_numpy(np.asarray(x, np.float32)).cuda().to(dtype)[:, None].expand(B, 2, V)
    q = None if xq is None else torch.from_numpy(np.asarray(xq, np.float32)).cuda().to(dtype)[:, None]
    one, out = torch.ones(B, 1, device="cuda"), torch.full((B, 2), 77, dtype=torch.int32, device="cuda")
    status = torch.full((B,), 77, dtype=torch.int32, device="cuda")
    fw.switchsd_resample(logits, torch.from_numpy(np.asarray(draft, np.int32)).cuda()[:, None], torch.ones(B, dtype=torch.int32, device="cuda"), one * 0, one * 0.5, out,
                         seeds=torch.from_numpy(np.asarray(seeds, np.int64)).cuda(), ctx_lens=torch.from_numpy(np.asarray(ctx, np.int32)).cuda(), temperature=f32(temps),
                         lse=None if lse is None else f32(lse)[:, None].expand(B, 2).contiguous(), q_logits=q, q_lse=None if q_lse is None else f32(q_lse)[:, None], status=status)
    assert not status.any() and (out[:, 1] == -1).all()
    return out[:, 0].cpu().numpy()


def _rows(x, temps, seeds, ctx, **kw):
    each = lambda b: {k: (v[b] if isinstance(v, np.ndarray) else v) for k, v in kw.items()}
    return np.array([ref.token(x[b], temps[b], int(seeds[b]), int(ctx[b]), **each(b)) for b in range(len(x))])


@pytest.mark.parametrize("at,T,spread", [(1e5, 0.7, 2.0), (-1e5, 0.7, 2.0), (60.0, 4e-4, 1e-3), (3e6, 1.0, 4.0), (-40.0, 1e-3, 3e-3)])
def test_residuals_of_large_logits(at, T, spread):
    """A drafter's rows whose logits over the temperature lie near 4e4 to 3e6, where binary32's numbers are up to 1/4 apart."""
    rng = np.random.default_rng(int(abs(at)))
    B, V = 4000, 150
    x = np.float32(at + rng.standard_normal((B, V)) * spread).astype(np.float64)
    xq = np.float32(x + rng.standard_normal((B, V)) * spread * 0.3).astype(np.float64)
    temps = np.full(B, np.float32(T), np.float64)
    lse, q_lse = (np.float32([ref.logprobs(y[b], temps[b])[2] for b in range(B)]).astype(np.float64) for y in (x, xq))
    seeds, ctx = rng.integers(-2**63, 2**63 - 1, B), rng.integers(0, 10000, B)
    got = _call(x, "f32", np.zeros(B), temps, seeds, ctx, lse=lse, xq=xq, q_lse=q_lse)
    with np.errstate(over="ignore", invalid="ignore"):
        want = _rows(x, temps, seeds, ctx, lse=lse, lq=xq, q_lse=q_lse)
    assert np.array_equal(got, want), (np.argwhere(got != want)[:5], (got != want).sum())


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1e-30, 1e-37, 2e-38, 1e-40, 2.0 ** -149])
def test_temperatures_next_to_zero(T, name):
    """Logits over temperatures beyond binary32's range: the largest logit that may be drawn, of equal ones the one that binary64
    finds, and the smallest where the draws are lost in its rounding; of negative, positive and mixed logits."""
    rng = np.random.default_rng(int(-np.log2(T)))
    B, V = 12, 5003
    x = np.abs(rng.standard_normal((B, V))) * 9 + 1
    x[:4] *= -1
    x[4:8] *= np.where(rng.random((4, V)) < 0.5, -1, 1)
    x[3:5] = np.round(x[3:5])  # (many equal ones)
    x = ((np.float32(x).view(np.uint32) & 0xffff0000).view(np.float32) if name == "bf16" else np.float32(x)).astype(np.float64)
    temps, seeds, ctx = np.full(B, np.float32(T), np.float64), np.arange(B) * 3 - 5, np.arange(B)
    draft = x.argmax(1)
    got = _call(x, name, draft, temps, seeds, ctx)
    assert np.array_equal(got, _rows(x, temps, seeds, ctx, skip=draft))


@pytest.mark.parametrize("drafter", [False, True])
@pytest.mark.parametrize("name,V,B", [("f32", 200003, 2), ("f32", 60000, 90), ("bf16", 262144, 3), ("bf16", 131072, 170)])
def test_masks_that_leave_no_early_token(name, V, B, drafter):
    """Logits of -inf but for the last third of every eighth of the vocabulary (what a CTA takes, or a part of it): thousands of
    tokens without a bound to go by, more than the list of those to be worked out holds."""
    rng = np.random.default_rng(V + B)
    some = min(B, 3)
    x = np.float32(rng.standard_normal((some, V)) * 2)
    xq = np.float32(x + rng.standard_normal((some, V)) * 0.7)
    if name == "bf16":
        x, xq = ((y.view(np.uint32) & 0xffff0000).view(np.float32) for y in (x, xq))
    eighth = -(-V // 8)
    x[:, np.arange(V) % eighth < 2 * eighth // 3] = -np.inf
    x, xq = (np.float64(y)[np.arange(B) % some] for y in (x, xq))
    temps, seeds, ctx = np.full(B, np.float32(0.8), np.float64), np.arange(B) % some, np.zeros(B, int)
    draft, kw, weights = x.argmax(1), {}, {}
    if drafter:
        lse, q_lse = (np.float32([ref.logprobs(y[b], temps[b])[2] for b in range(some)]).astype(np.float64)[np.arange(B) % some] for y in (x, xq))
        kw, weights = dict(lse=lse, xq=xq, q_lse=q_lse), dict(lse=lse[:some], lq=xq[:some], q_lse=q_lse[:some])
    else:
        weights = dict(skip=draft[:some])
    got = _call(x, name, draft, temps, seeds, ctx, **kw)
    assert np.array_equal(got, _rows(x[:some], temps, seeds, ctx, **weights)[np.arange(B) % some])


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("T,spread", [(0.01, 8.0), (0.01, 1.0), (0.05, 6.0), (0.003, 0.6)])
def test_residuals_of_low_temperatures(T, spread, name):
    """All of p and q on one token each, often the same one: what is left there is lse's rounding, or nothing, and the other tokens'
    p is no binary64 number, or one of few bits."""
    rng = np.random.default_rng(int(T * 1e4 + spread))
    B, V = 4000, 30
    x = np.float32(rng.standard_normal((B, V)) * spread)
    xq = np.float32(x + rng.standard_normal((B, V)) * spread * 0.3)
    x, xq = ((np.float64((y.view(np.uint32) & 0xffff0000).view(np.float32)) if name == "bf16" else np.float64(y)) for y in (x, xq))
    xq[::7, ::3] = -np.inf
    temps = np.full(B, np.float32(T), np.float64)
    lse, q_lse = (np.float32([ref.logprobs(y[b], temps[b])[2] for b in range(B)]).astype(np.float64) for y in (x, xq))
    seeds, ctx = rng.integers(-2**63, 2**63 - 1, B), rng.integers(0, 10000, B)
    got = _call(x, name, np.zeros(B), temps, seeds, ctx, lse=lse, xq=xq, q_lse=q_lse)
    want = _rows(x, temps, seeds, ctx, lse=lse, lq=xq, q_lse=q_lse)
    assert np.array_equal(got, want), (np.argwhere(got != want)[:5], (got != want).sum())
