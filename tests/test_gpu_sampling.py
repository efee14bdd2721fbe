"""switchsd_logprobs and switchsd_resample on the GPU, against plain implementations in 64 bits (sampling_ref.py).

Tokens are compared exactly.  Tolerances of the log probabilities: z = (l - max) / temperature is rounded twice
(2^-23 of it), its exponential is off by 2^-21 of it (2^-22 the instruction, the rest z's), a sum of V weights in parts of at
most 2^9 additions a thread and 12 joins by (2^9 + 12) 2^-24 at the worst, 2^-14.9: so ln S by 2^-14.5, a log probability by
that and 2^-22 of itself, the entropy by twice that and 2^-20 of ln V; lse by that and 2^-22 of itself.
"""
import numpy as np
import pytest

from tests import sampling_ref as ref
from tests.target_ref import bf16_round

pytestmark = pytest.mark.gpu


def _fw():
    import paper_2609_20186_gb300 as fw
    return fw


def _cuda(a, dtype):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


def _i32(a):
    import torch
    return _cuda(np.asarray(a, np.int64), torch.int32)


def _f32(a):
    import torch
    return _cuda(np.asarray(a, np.float64), torch.float32)


def _dtype(name):
    import torch
    return dict(bf16=torch.bfloat16, f16=torch.float16, f32=torch.float32)[name]


def _round(x, name):
    with np.errstate(over="ignore"):
        return bf16_round(x) if name == "bf16" else x.astype(np.float16 if name == "f16" else np.float32).astype(np.float64)


def _logits(rng, shape, name, spread=2.0):
    x = rng.standard_normal(shape) * spread
    flat = x.reshape(-1, shape[-1])
    for row in flat:
        row[rng.integers(0, shape[-1], 4)] += rng.uniform(0, 12, 4)
    return _round(x, name)


def _placed(x, name, lead=0, pad=0):
    """[B, T, V] as a view with its own strides, `lead` elements into its memory."""
    import torch
    B, T, V = x.shape
    buf = torch.full((lead + B * (T * (V + pad) + 3),), float("nan"), dtype=_dtype(name), device="cuda")
    y = buf[lead:].as_strided((B, T, V), (T * (V + pad) + 3, V + pad, 1))
    y.copy_(_cuda(x, torch.float64))
    return y


def _outputs(B, T, K, top):
    import torch
    f = dict(dtype=torch.float32, device="cuda")
    o = dict(entropy=torch.full((B, T), 77.0, **f), lse=torch.full((B, T), 77.0, **f), status=torch.full((B,), 77, dtype=torch.int32, device="cuda"))
    if K:
        o.update(logprob=torch.full((B, K), 77.0, **f), prob=torch.full((B, K), 77.0, **f))
    if top:
        o.update(top_ids=torch.full((B, T, top), 77, dtype=torch.int32, device="cuda"), top_logprobs=torch.full((B, T, top), 77.0, **f))
    return o


LOG_S = 2.0 ** -14.5


def _check(o, x, new, temps, tokens, top):
    B, T, V = x.shape
    g = {k: v.double().cpu().numpy() for k, v in o.items()}
    for b in range(B):
        ok = 0 <= new[b] <= T
        assert g["status"][b] == (0 if ok else 2)
        for t in range(T):
            here = ok and t < new[b]
            lp, entropy, lse, order = ref.logprobs(x[b, t], temps[b]) if here else (np.full(V, -np.inf), 0.0, -np.inf, [])
            lp = np.where(lp < -3.5e38, -np.inf, lp)  # beyond binary32, which the outputs are held in
            if lse == -np.inf:
                assert g["lse"][b, t] == -np.inf and g["entropy"][b, t] == 0
            else:
                assert abs(g["lse"][b, t] - lse) <= LOG_S + 2.0 ** -22 * abs(lse), (b, t)
                assert abs(g["entropy"][b, t] - entropy) <= 2 * LOG_S + 2.0 ** -20 * np.log(V + 1), (b, t)
            if tokens is not None and t < tokens.shape[1]:
                want = lp[tokens[b, t]] if 0 <= tokens[b, t] < V else -np.inf
                got, prob = g["logprob"][b, t], g["prob"][b, t]
                assert got == want if want == -np.inf else abs(got - want) <= LOG_S + 2.0 ** -22 * abs(want), (b, t)
                assert abs(prob - np.exp(want)) <= (2 * LOG_S + 2.0 ** -21 * (abs(want) if want > -np.inf else 0)) * np.exp(want) + 2.0 ** -126
            if top:
                ids = (order + [-1] * top)[:top]
                assert g["top_ids"][b, t].tolist() == ids, (b, t)
                for i, v in enumerate(ids):
                    want, got = (lp[v] if v >= 0 else -np.inf), g["top_logprobs"][b, t, i]
                    assert got == want if want == -np.inf else abs(got - want) <= LOG_S + 2.0 ** -22 * abs(want), (b, t, i)


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("B,T,V,K,top,lead,pad", [(1, 1, 1, 1, 1, 0, 0), (2, 3, 7, 3, 8, 1, 0), (3, 2, 100, 1, 32, 5, 1), (1, 1, 128256, 1, 20, 0, 0),
                                                  (5, 4, 1000, 3, 0, 3, 5), (2, 40, 5003, 40, 5, 7, 2), (1, 2, 262144, 2, 32, 0, 0), (90, 5, 9001, 4, 3, 2, 1)])
def test_logprobs(B, T, V, K, top, lead, pad, name):
    """Sizes, alignments, strides, ragged rows, temperatures with 0 among them, tokens outside the vocabulary."""
    import torch
    rng = np.random.default_rng(B * T + V)
    x = _logits(rng, (B, T, V), name)
    new = rng.integers(0, T + 1, B)
    new[-1] = T
    temps = rng.uniform(0.3, 2.0, B).astype(np.float32)
    temps[::4] = 0 if B > 1 else 0.7
    tokens = rng.integers(-1, V + 1, (B, K)) if K else None
    if K:
        tokens[:, 0] = x[:, 0].argmax(1)
    o = _outputs(B, T, K, top)
    _fw().switchsd_logprobs(_placed(x, name, lead, pad), tokens=_i32(tokens) if K else None, new_lens=_i32(new - 1), new_add=1, temperature=_f32(temps), **o)
    _check(o, x, new, temps.astype(np.float64), tokens, top)


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_logprobs_of_masks_and_ties(name):
    """Nothing left, one token, masks of -inf and of the type's lowest value, equal logits, NaN, logits in rising and falling
    order (every one a new best), bad lengths."""
    import torch
    rng = np.random.default_rng(2)
    V, top = 20011, 32
    low = torch.finfo(_dtype(name)).min
    rows = [np.full(V, -np.inf), np.full(V, np.nan), np.full(V, -np.inf), np.full(V, low), np.zeros(V), np.full(V, 3.25), np.arange(V) / 97.0, -np.arange(V) / 97.0,
            rng.standard_normal(V), rng.standard_normal(V), rng.standard_normal(V), np.round(rng.standard_normal(V)), np.where(np.arange(V) % 2 > 0, -0.0, 0.0)]
    rows[2][777] = -3e4
    rows[3][[5, 19999]] = 1.0
    rows[8][rng.random(V) < 0.999] = -np.inf
    rows[9][rng.random(V) < 0.999] = low
    rows[10][rng.random(V) < 0.5] = np.nan
    x = np.stack([_round(r, name) for r in rows])[:, None]
    B = len(rows)
    for temps in (np.ones(B), np.zeros(B), np.full(B, 0.01)):
        o, tokens = _outputs(B, 1, 1, top), np.full((B, 1), 777)
        _fw().switchsd_logprobs(_placed(x, name, 3), tokens=_i32(tokens), temperature=_f32(temps), **o)
        _check(o, x, [1] * B, np.float32(temps).astype(np.float64), tokens, top)
    o, new = _outputs(B, 1, 1, top), np.ones(B, int)
    new[:4] = (-1, 2, 0, 1)
    _fw().switchsd_logprobs(_placed(x, name), tokens=_i32(tokens), new_lens=_i32(new), **o)
    _check(o, x, new, np.ones(B), tokens, top)


def test_logprobs_of_infinity_and_bad_temperatures():
    import torch
    x = torch.randn(4, 1, 3000, device="cuda")
    x[0, 0, 17] = float("inf")
    o, nan = _outputs(4, 1, 1, 2), float("nan")
    _fw().switchsd_logprobs(x, tokens=_i32([[17], [5], [5], [5]]), temperature=_f32([1.0, -1.0, np.inf, np.nan]), **o)
    assert o["lse"][0, 0] == float("inf") and o["lse"][1:].isnan().all() and o["entropy"].isnan().all() and o["logprob"].isnan().all()
    assert o["top_ids"][0, 0, 0] == 17 and o["top_ids"][1, 0, 0] == x[1, 0].argmax() and nan != nan
    _fw().switchsd_logprobs(x, tokens=_i32([[17], [5], [5], [5]]), temperature=_f32([0.0] * 4), **o)
    assert o["logprob"][0, 0] == 0 and o["lse"][0, 0] == float("inf") and o["entropy"][0, 0] == 0


def test_logprobs_outputs_one_at_a_time():
    """Every output alone is what it is among the others, and the others' memory is left."""
    import torch
    rng = np.random.default_rng(4)
    x = _placed(_logits(rng, (3, 4, 6000), "bf16"), "bf16")
    tokens, temps = _i32(rng.integers(0, 6000, (3, 4))), _f32([0.0, 1.0, 0.6])
    full = _outputs(3, 4, 4, 7)
    _fw().switchsd_logprobs(x, tokens=tokens, temperature=temps, **full)
    for name in ("logprob", "prob", "entropy", "lse", "top_ids", "top_logprobs"):
        o = _outputs(3, 4, 4, 7)
        _fw().switchsd_logprobs(x, tokens=tokens, temperature=temps, **{name: o[name]})
        assert torch.equal(o[name], full[name]), name


def test_logits_beyond_32_bits():
    import torch
    rng = np.random.default_rng(9)
    V, far = 40000, 2**31 + 24
    buf = torch.empty(2 * far + 2 * V, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((2, 2, V), (far, far, 1))
    y = _logits(rng, (2, 2, V), "bf16")
    y[1, 0] = y[0, 1]  # (the same memory)
    x.copy_(_cuda(y, torch.float64))
    o, tokens = _outputs(2, 2, 2, 5), rng.integers(0, V, (2, 2))
    _fw().switchsd_logprobs(x, tokens=_i32(tokens), **o)
    _check(o, y, [2, 2], np.ones(2), tokens, 5)
    out = torch.zeros(2, 2, dtype=torch.int32, device="cuda")
    zero = torch.zeros(2, 1, device="cuda")
    _fw().switchsd_resample(x, _i32([[5], [5]]), _i32([1, 1]), zero + 1, zero, out, seeds=torch.tensor([1, 2], device="cuda"), ctx_lens=_i32([7, 9]))
    assert out.cpu().tolist() == [[-1, ref.token(y[b, 1], 1.0, b + 1, 7 + 2 * b + 1, )] for b in range(2)]


# --- the appended token -------------------------------------------------------------------------------------------
def _resample(x, name, draft, n, p, u, seeds, ctx, temps=None, lse=None, q=None, xq=None, q_lse=None, mode=None, lead=0, pad=0):
    import torch
    B, T, V = x.shape
    out, status = torch.full((B, T), 77, dtype=torch.int32, device="cuda"), torch.full((B,), 77, dtype=torch.int32, device="cuda")
    _fw().switchsd_resample(_placed(x, name, lead, pad), _i32(draft), _i32(n), _f32(p), _f32(u), out, seeds=_cuda(np.asarray(seeds, np.int64), torch.int64),
                            ctx_lens=_i32(ctx), temperature=None if temps is None else _f32(temps), lse=None if lse is None else _f32(lse),
                            q_draft=None if q is None else _f32(q), q_logits=None if xq is None else _placed(xq, name, lead + 1, pad),
                            q_lse=None if q_lse is None else _f32(q_lse), mode=None if mode is None else _i32(mode), status=status)
    return out.cpu().numpy(), status.cpu().numpy()


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("B,T,V,drafter,lead,pad", [(1, 1, 1, False, 0, 0), (6, 2, 9, True, 1, 0), (40, 5, 100, True, 0, 1), (9, 3, 5003, False, 3, 2), (30, 4, 3001, True, 5, 1),
                                                    (1, 2, 128256, False, 0, 0), (2, 2, 152064, True, 0, 0), (200, 1, 2000, False, 0, 0), (1, 1, 262144, False, 1, 0)])
def test_resample(B, T, V, drafter, lead, pad, name):
    """Every row's one token and nothing else, of copied drafts, a drafter's and none, over temperatures and alignments."""
    rng = np.random.default_rng(B + V)
    k = T - 1
    x = _logits(rng, (B, T, V), name)
    temps = rng.uniform(0.3, 1.5, B).astype(np.float32).astype(np.float64)
    if B > 1:
        temps[::5] = 0
    n = rng.integers(0, T, B)
    seeds, ctx = rng.integers(-2**63, 2**63 - 1, B), rng.integers(0, 2**31 - 1 - T, B)
    u = rng.random((B, k)).astype(np.float32)
    draft = x[:, :k].argmax(2) if k else np.zeros((B, 0), int)
    p, q, lse, q_lse, xq = np.zeros((B, k)), np.ones((B, k)), np.zeros((B, T)), np.zeros((B, k)), None
    mode = rng.integers(0, 3, B)
    if drafter:
        xq = _round(x[:, :k] + rng.standard_normal((B, k, V)) * 0.7, name)
    for b in range(B):
        for t in range(T):
            lse[b, t] = np.float32(ref.logprobs(x[b, t], temps[b])[2])
            if t < k:
                p[b, t] = np.float32(0.6)
                if drafter:
                    q_lse[b, t] = np.float32(ref.logprobs(xq[b, t], temps[b])[2])
                    q[b, t] = 1.0 if mode[b] == 1 else np.float32(0.7)
    got, status = _resample(x, name, draft, n, p, u, seeds, ctx, temps, lse, q if drafter else None, xq, q_lse if drafter else None, mode if drafter else None, lead, pad)
    assert not status.any()
    want = np.full((B, T), -1)
    for b in range(B):
        a = ref.accepted(p[b], q[b], u[b], n[b])
        kw = {}
        if a < n[b]:
            kw = dict(lse=lse[b, a], lq=xq[b, a], q_lse=q_lse[b, a]) if drafter and mode[b] != 1 else dict(skip=draft[b, a])
        want[b, a] = ref.token(x[b, a], temps[b], int(seeds[b]), int(ctx[b]) + a, **kw)
    assert np.array_equal(got, want), np.argwhere(got != want)


def test_resample_at_its_edges():
    """Nothing left, one token left, only the rejected one left, residuals that vanish, NaN, equal logits, infinities, bad
    lengths and temperatures, logits in rising order, a T of which one is allowed."""
    rng = np.random.default_rng(6)
    V = 4001
    inf, nan = np.inf, np.nan
    rows = [np.full(V, -inf), np.full(V, -inf), np.full(V, -inf), rng.standard_normal(V), rng.standard_normal(V), np.full(V, 2.0), np.arange(V) / 7.0,
            rng.standard_normal(V), rng.standard_normal(V), rng.standard_normal(V), rng.standard_normal(V), np.full(V, nan), rng.standard_normal(V) * 1e4]
    rows[1][99] = 1.0
    rows[2][50] = 1.0                     # the rejected token alone
    rows[4][rng.random(V) < 0.5] = nan
    rows[7][3] = inf
    B = len(rows)
    x = np.stack([_round(r, "f32") for r in rows])[:, None].repeat(2, 1)
    draft = np.full((B, 1), 50)
    n, temps = np.ones(B, int), np.ones(B)
    n[8], n[9], temps[10] = -1, 2, nan
    p, u = np.zeros((B, 1)), np.full((B, 1), 0.5)
    seeds, ctx = np.arange(B) * 7 - 20, np.arange(B)
    got, status = _resample(x, "f32", draft, n, p, u, seeds, ctx, temps)
    want = [[ref.token(x[b, 0], 1.0, int(seeds[b]), int(ctx[b]), skip=50), -1] for b in range(B)]
    for b in (8, 9, 10):
        want[b] = [-1, -1]
    want[7] = [3, -1]
    assert got.tolist() == want and status.tolist() == [2 if b in (8, 9) else 0 for b in range(B)]
    # p = q everywhere but for roundings, exactly, and p > q at one token only
    x = np.stack([rng.standard_normal(V)] * 3).astype(np.float32).astype(np.float64)[:, None].repeat(2, 1)
    xq = x[:, :1].copy()
    xq[2, 0] += 1.0
    xq[2, 0, 1234] = -5.0
    lse = np.array([[np.float32(ref.logprobs(x[b, 0], 1.0)[2])] * 2 for b in range(3)])
    q_lse = lse[:, :1].copy()
    q_lse[0] = np.nextafter(np.float32(q_lse[0]), np.float32(100))
    q_lse[2] = np.float32(ref.logprobs(x[2, 0], 1.0)[2])
    got, _ = _resample(x, "f32", draft[:3], np.ones(3, int), p[:3], u[:3], seeds[:3], ctx[:3], None, lse, np.ones((3, 1)), xq, q_lse)
    assert got[:, 0].tolist() == [ref.token(x[b, 0], 1.0, int(seeds[b]), int(ctx[b]), lse=lse[b, 0], lq=xq[b, 0], q_lse=q_lse[b, 0]) for b in range(3)] and got[2, 0] == 1234


def test_resample_follows_the_distribution():
    """Over many seeds every token comes as often as its weight says: a chi-squared statistic of 19 degrees of freedom below
    the 1e-6 quantile's 63 (the seeds are fixed; another generator would leave it so for all but one in a million)."""
    import torch
    rng = np.random.default_rng(8)
    V, B = 20, 60000
    l = _round(rng.standard_normal(V) * 1.5, "f32")
    lq = _round(rng.standard_normal(V) * 1.5, "f32")
    lse, q_lse = (np.float32(ref.logprobs(a, 1.0)[2]) for a in (l, lq))
    x, xq = _f32(l).expand(B, 2, V), _f32(lq).expand(B, 1, V)
    ones, out = torch.ones(B, 1, device="cuda"), torch.empty(B, 2, dtype=torch.int32, device="cuda")
    seeds, ctx = torch.arange(B, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    draft = torch.full((B, 1), 3, dtype=torch.int32, device="cuda")
    for kw, w in ((dict(), np.exp(l)), (dict(lse=_f32(np.full((B, 2), lse)), q_logits=xq, q_lse=_f32(np.full((B, 1), q_lse))), np.maximum(np.exp(l - lse) - np.exp(lq - q_lse), 0))):
        if not kw:
            w[3] = 0
        _fw().switchsd_resample(x, draft, torch.ones(B, dtype=torch.int32, device="cuda"), ones * 0, ones * 0.5, out, seeds=seeds, ctx_lens=ctx, **kw)
        count = np.bincount(out[:, 0].cpu().numpy(), minlength=V)
        expect = w / w.sum() * B
        assert not count[w == 0].any()
        assert ((count - expect)[w > 0] ** 2 / expect[w > 0]).sum() < 63
        assert (out[:, 1] == -1).all()


def test_a_step_at_temperature():
    """A verification step as it is used: probabilities of the drafts, the appended token, the verification; twice in a
    captured graph on other inputs."""
    import torch
    from paper_2609_20186_gb300 import binding as bd
    rng = np.random.default_rng(12)
    B, k, V, cap = 12, 4, 700, 64
    g, i32 = dict(device="cuda"), dict(dtype=torch.int32, device="cuda")
    logits, ctx, lens = torch.zeros(B, k + 1, V, dtype=torch.bfloat16, **g), torch.zeros(B, cap, **i32), torch.zeros(B, **i32)
    draft, n, temps, u, seeds = torch.zeros(B, k, **i32), torch.zeros(B, **i32), torch.zeros(B, **g), torch.zeros(B, k, **g), torch.zeros(B, dtype=torch.int64, **g)
    p, token, accept = torch.zeros(B, k, **g), torch.zeros(B, k + 1, **i32), torch.zeros(B, **i32)

    def step():
        bd.switchsd_logprobs(logits, tokens=draft, new_lens=n, new_add=1, temperature=temps, prob=p)
        bd.switchsd_resample(logits, draft, n, p, u, token, seeds=seeds, ctx_lens=lens, temperature=temps)
        bd.switchsd_verify_sampled(draft, p, u, token, accept, draft_len=n, ctx_tokens=ctx, ctx_lens=lens)
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        x = _logits(rng, (B, k + 1, V), "bf16")
        d, m, L = x[:, :k].argmax(2), rng.integers(0, k + 1, B), rng.integers(1, cap - k - 1, B)
        T, w, s = rng.choice([0.0, 0.5, 1.0], B), rng.random((B, k)).astype(np.float32), rng.integers(-2**63, 2**63 - 1, B)
        for dst, src in ((logits, _cuda(x, torch.bfloat16)), (draft, _i32(d)), (n, _i32(m)), (lens, _i32(L)), (temps, _f32(T)), (u, _f32(w)), (seeds, _cuda(s, torch.int64))):
            dst.copy_(src)
        graph.replay()
        probs = p.cpu().numpy()
        for b in range(B):
            a = ref.accepted(probs[b], np.ones(k), w[b], m[b])
            want = ref.token(x[b, a], T[b], int(s[b]), int(L[b]) + a, **(dict(skip=d[b, a]) if a < m[b] else {}))
            assert int(accept[b]) == a and int(lens[b]) == L[b] + a + 1
            assert ctx[b, L[b]:L[b] + a + 1].tolist() == d[b, :a].tolist() + [want]


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("B,T", [(3, 50), (8, 57), (3, 153), (152, 12), (19, 97)])
def test_logprobs_of_many_positions(B, T, name):
    """Numbers of positions on both sides of those where other CTAs take them, a vocabulary that none divides evenly."""
    rng = np.random.default_rng(B + T)
    V, top = 4099, 7
    x = _logits(rng, (B, T, V), name)
    new = rng.integers(0, T + 1, B)
    new[0] = T
    temps = np.float32(0.9) + np.zeros(B, np.float32)
    tokens = rng.integers(0, V, (B, T))
    o = _outputs(B, T, T, top)
    _fw().switchsd_logprobs(_placed(x, name, 3, 1), tokens=_i32(tokens), new_lens=_i32(new), temperature=_f32(temps), **o)
    _check(o, x, new, temps.astype(np.float64), tokens, top)


def test_resample_of_rows_with_unlike_alignments():
    """A drafter's rows that are aligned otherwise than the target's, at every offset between them, over more than one CTA a
    row."""
    rng = np.random.default_rng(3)
    B, T, V = 4, 2, 20011
    x = _logits(rng, (B, T, V), "bf16")
    xq = _round(x[:, :1] + rng.standard_normal((B, 1, V)) * 0.7, "bf16")
    draft, ones = x[:, :1].argmax(2), np.ones((B, 1))
    lse = np.array([[np.float32(ref.logprobs(x[b, t], 1.0)[2]) for t in range(T)] for b in range(B)], np.float64)
    q_lse = np.array([[np.float32(ref.logprobs(xq[b, 0], 1.0)[2])] for b in range(B)], np.float64)
    seeds, ctx = rng.integers(0, 2**62, B), rng.integers(0, 1000, B)
    for lead in range(8):
        got, status = _resample(x, "bf16", draft, np.ones(B, int), 0.5 * ones, ones, seeds, ctx, np.ones(B), lse, ones, xq, q_lse, np.zeros(B, int), lead, lead)
        assert not status.any()
        for b in range(B):
            want = ref.token(x[b, 0], 1.0, int(seeds[b]), int(ctx[b]), lse=lse[b, 0], lq=xq[b, 0], q_lse=q_lse[b, 0])
            assert got[b].tolist() == [want, -1], (lead, b)
