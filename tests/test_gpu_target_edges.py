"""The operators of include/switchsd_target.h at the edges of what their header takes: counts of pages that no map wrote,
against the plain implementations in 64 bits (target_ref.py)."""
import numpy as np
import pytest

from tests import target_ref as ref

pytestmark = pytest.mark.gpu


def _fw():
    import paper_2609_20186_gb300 as fw
    return fw


def _i32(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


# --- block tables and slot maps -----------------------------------------------------------------------------------
@pytest.mark.parametrize("B", [4, 70, 130, 170, 200, 300, 1100])
@pytest.mark.parametrize("bad", [-1, -2, -5, -2**31, 9, 2**31 - 1])
def test_map_leaves_rows_with_a_bad_count_of_pages_alone(B, bad):
    """A row whose held lies outside [0, blocks] keeps it, gets no slots, and moves no page: the pool's count, list and
    tables are those of a step that skips the row.  B: clusters of 1, 3, 5, 6, 7 and 8 CTAs."""
    import torch
    fw = _fw()
    T, page, blocks = 3, 16, 8
    rng = np.random.default_rng(B)
    pages = B * blocks
    free = rng.permutation(pages).astype(np.int32)
    st = ref.MapState(B, blocks, free)
    table, held = torch.full((B, blocks), -1, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    fl, fc = _i32(free), _i32([pages])
    rows = [1, B // 2, B - 1]
    for step in range(3):
        lens, new = rng.integers(0, page * blocks - T, B), rng.integers(0, T + 1, B)
        wl = lens.copy()
        good = held.clone()
        if step == 1:
            held[rows] = bad
            wl[rows] = -1                        # how the plain form leaves a row out
        before = held.clone()
        slots, status = torch.full((B, T), 7, dtype=torch.int32, device="cuda"), torch.full((B,), 7, dtype=torch.int32, device="cuda")
        fw.switchsd_kv_map(_i32(lens), _i32(new), table, held, fl, fc, slots, page=page, status=status)
        want_slots, want_status = st.step(wl.tolist(), new.tolist(), T, page)
        wt, wh, wf, wc = st.arrays()
        assert int(fc.cpu()[0]) == wc
        assert np.array_equal(fl.cpu().numpy(), wf)
        assert np.array_equal(table.cpu().numpy(), wt)
        assert np.array_equal(status.cpu().numpy(), want_status)
        assert np.array_equal(slots.cpu().numpy(), want_slots)
        if step == 1:
            assert torch.equal(held[rows], before[rows])
            held[rows] = good[rows]              # mended by the caller: the next step has every page
        assert np.array_equal(held.cpu().numpy(), wh)
    everything = np.concatenate([wf[:wc], wt[wt >= 0]])
    assert np.array_equal(np.sort(everything), np.arange(pages))  # no page lost, none held twice


@pytest.mark.parametrize("B,T", [(1, 2**31 - 1), (33, (2**31 - 1) // 33)])
def test_map_of_the_longest_step(B, T):
    """B * T just below 2^31: the slots' last places."""
    import torch
    fw = _fw()
    page, blocks, n = 256, 4, 700
    table, held = torch.full((B, blocks), -1, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    fl, fc = _i32(np.arange(B * blocks)), _i32([B * blocks])
    slots, status = torch.full((B, T), 7, dtype=torch.int32, device="cuda"), torch.full((B,), 7, dtype=torch.int32, device="cuda")
    fw.switchsd_kv_map(_i32(np.full(B, 100)), _i32(np.full(B, n)), table, held, fl, fc, slots, page=page, status=status)
    assert not status.any() and (held == 4).all()
    p = torch.arange(100, 100 + n, device="cuda")
    assert torch.equal(slots[:, :n].long(), table.long()[:, p // page] * page + p % page)
    for b in range(B):
        assert (slots[b, n:] == -1).all()


@pytest.mark.parametrize("B,add,alias", [(5, 0, False), (40, 1, False), (300, 1, True), (1030, -2, False)])
def test_map_says_what_it_granted(B, add, alias):
    """granted is new_lens for the rows with slots and -1 - new_add for the others: bad lengths, too many blocks, no pages."""
    import torch
    fw = _fw()
    rng = np.random.default_rng(B)
    T, page, blocks = 9, 16, 10
    pages = max(2, int(B * blocks * 0.35))
    free = rng.permutation(pages).astype(np.int32)
    st = ref.MapState(B, blocks, free)
    table, held = torch.full((B, blocks), -1, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    fl, fc = _i32(free), _i32([pages])
    refused = 0
    for step in range(4):
        lens, new = rng.integers(0, page * blocks - T, B), rng.integers(0, T + 1, B)
        lens[1], new[2], lens[3] = -4, T + 1, page * blocks
        new[3] = max(new[3], 1)
        given, status = _i32(new - add), torch.full((B,), 7, dtype=torch.int32, device="cuda")
        granted = given if alias else torch.full((B,), 77, dtype=torch.int32, device="cuda")
        slots = torch.full((B, T), 7, dtype=torch.int32, device="cuda")
        fw.switchsd_kv_map(_i32(lens), given, table, held, fl, fc, slots, page=page, new_add=add, status=status, granted=granted)
        want_slots, want_status = st.step(lens.tolist(), new.tolist(), T, page)
        assert np.array_equal(slots.cpu().numpy(), want_slots) and np.array_equal(status.cpu().numpy(), want_status)
        assert np.array_equal(granted.cpu().numpy(), np.where(want_status == 0, new - add, -1 - add))
        assert np.array_equal(table.cpu().numpy(), st.arrays()[0])
        refused += int((want_status == 1).sum())
    assert refused > 4 or B < 40  # (more than the row whose blocks are too few: the pool was short too)


@pytest.mark.parametrize("T", [3, 9])  # 12 and 36 query rows a key head
def test_a_row_without_pages_sits_the_step_out(T):
    """The pool is short of pages for one row, in whose last page an earlier step left a rejected draft: its attention is
    zeros and not those tokens', its logits name no token, the verification leaves its context; the other row goes on, and
    so does the first once the pool has pages."""
    import torch
    fw = _fw()
    torch.manual_seed(T)
    B, H, Hq, D, page, V, k = 2, 1, 4, 128, 16, 50, T - 1
    cache = fw.KVCache(B, T, layers=1, heads=H, dim=D, pages=4, max_len=200, page=page, lens_add=-1, new_add=1)
    i32 = dict(dtype=torch.int32, device="cuda")
    ctx = torch.randint(0, V, (B, 200), **i32)
    hist = [[], []]

    def step(lens, vlen):
        """One step; the rows' keys and values join `hist` where they got slots."""
        x = torch.randn(B, T, Hq + 2 * H, D, device="cuda").to(torch.bfloat16)
        cl, vl = _i32(lens), _i32(vlen)
        cache.map(cl, vl)
        vl.copy_(cache.new)
        cache.append(0, x[:, :, Hq:Hq + H], x[:, :, Hq + H:])
        out = cache.attend(0, x[:, :, :Hq], torch.full((B, T, Hq, D), 9.0, dtype=torch.bfloat16, device="cuda"))
        best = torch.full((B, T), 77, **i32)
        fw.switchsd_logits(torch.randn(B, T, V, device="cuda"), ctx_tokens=ctx, ctx_lens=cl, new_lens=vl, new_add=1, argmax=best)
        acc, status = torch.full((B,), 77, **i32), torch.full((B,), 77, **i32)
        before = ctx.clone()
        fw.switchsd_verify(torch.zeros(B, k, **i32), best, acc, draft_len=vl, ctx_tokens=ctx, ctx_lens=cl, status=status)
        xs = x.double().cpu().numpy()
        got = out.double().cpu().numpy()
        for b in range(B):
            n = lens[b] - 1
            del hist[b][n:]
            if cache.status[b] != 0:
                assert cache.new[b] == -2 and (got[b] == 0).all()
                assert (best[b] == -1).all() and acc[b] == -1 and status[b] == 2
                assert torch.equal(ctx[b], before[b]) and cl[b] == lens[b]
                continue
            assert cache.new[b] == vlen[b] and acc[b] >= 0 and status[b] == 0 and cl[b] == lens[b] + acc[b] + 1
            for t in range(vlen[b] + 1):
                hist[b].append([ref.dequantise(*ref.quantise(xs[b, t, lo:lo + H])) for lo in (Hq, Hq + H)])
            ks, vs = (np.array([h[i] for h in hist[b]]) for i in range(2))
            want, mag = ref.attention(xs[b:b + 1, :, :Hq], [ks], [vs], [n], [vlen[b] + 1], float(np.float32(D ** -0.5)))
            tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -10 * mag
            assert np.all(np.abs(got[b:b + 1] - want) <= tol)
        return cache.status.cpu().tolist()
    goal = (14, 40)
    while [len(h) for h in hist] != list(goal):      # (a row that is there already writes its last token again)
        have = [len(h) for h in hist]
        assert step([min(n, g - 1) + 1 for n, g in zip(have, goal)], [max(0, min(k, g - n - 1)) for n, g in zip(have, goal)]) == [0, 0]
    assert int(cache.free_count) == 0
    assert step([15, 40], [1, 0]) == [0, 0]          # the first row's one page is full; its last token is rejected
    assert step([16, 40], [1, 0]) == [1, 0]          # and needs a second page, which there is not
    assert step([16, 31], [1, 0]) == [0, 0]          # the second row gave one back


# --- attention ----------------------------------------------------------------------------------------------------
def _bf16(x):
    import torch
    return torch.from_numpy(np.asarray(x, np.float64)).to(torch.bfloat16).cuda()


def _filled(rng, n, Hkv, D, page):
    """A cache with n random tokens of one row in order of its pages; its table, and the keys and values it holds."""
    import torch
    fw = _fw()
    blocks = -(-n // page)
    cache = torch.full((blocks, Hkv, fw.switchsd_kv4_bytes(page, D)), 0xff, dtype=torch.uint8, device="cuda")
    k, v = ref.bf16_round(rng.standard_normal((n, Hkv, D))), ref.bf16_round(rng.standard_normal((n, Hkv, D)))
    fw.switchsd_kv4_append(_bf16(k[None]), _bf16(v[None]), _i32(np.arange(n)[None]), cache, page=page)
    return cache, _i32(np.arange(blocks)[None]), ref.dequantise(*ref.quantise(k)), ref.dequantise(*ref.quantise(v))


def _near(got, want, mag):
    """bf16's rounding, 2^-8 of the result, and the weights' and the scores', 2^-10 of sum p |v|: as in test_gpu_target.py."""
    tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -10 * mag
    assert np.all(np.abs(got - want) <= tol), float(np.nanmax(np.abs(got - want) / tol))


@pytest.mark.parametrize("T", [1, 2, 5])  # tiles of 8, 16 and 128 query rows
@pytest.mark.parametrize("up,odd", [(0, 24), (0, -30), (20, "inf"), (20, "nan")])
def test_attention_of_a_head_goes_by_its_own_queries(T, up, odd):
    """One head's queries 2^24 above, and 2^30 below, the others' of its tile, or with an infinity or a NaN among
    them: the others' results are what they are without it."""
    import torch
    fw = _fw()
    rng = np.random.default_rng(T)
    Hq, D, page, n = 8, 128, 32, 200
    cache, table, k, v = _filled(rng, n, 1, D, page)
    q = ref.bf16_round(rng.standard_normal((1, T, Hq, D))) * 2.0 ** up
    if isinstance(odd, int):
        q[:, :, 3] *= 2.0 ** odd
    else:
        q[:, :, 3, 17] = float(odd)
    scale = float(np.float32(D ** -0.5 * 2.0 ** -up))
    out = torch.empty(1, T, Hq, D, dtype=torch.bfloat16, device="cuda")
    fw.switchsd_kv4_attention(_bf16(q), cache, table, _i32([n - T]), _i32([T]), out, page=page, scale=scale)
    got = out.double().cpu().numpy()
    rest = [h for h in range(Hq) if h != 3]
    want, mag = ref.attention(q[:, :, rest], [k], [v], [n - T], [T], scale)
    _near(got[:, :, rest], want, mag)
    if isinstance(odd, str):
        assert np.isnan(got[:, :, 3]).all()
    elif odd < 0:  # its scores are all but equal
        want, mag = ref.attention(q[:, :, 3:4], [k], [v], [n - T], [T], scale)
        _near(got[:, :, 3:4], want, mag)
    else:          # one key has all of the weight: the largest score's, far above every rounding of the scores
        x = np.einsum("td,nd->tn", q[0, :, 3], k[:, 0])
        for t in range(T):
            x[t, n - T + t + 1:] = -np.inf
            best = np.sort(x[t])
            if best[-1] - best[-2] > 2.0 ** -14 * np.abs(q[0, t, 3]).sum() * np.abs(k).max():
                assert np.all(np.abs(got[0, t, 3] - v[np.argmax(x[t]), 0]) <= 2.0 ** -8 * np.abs(v[np.argmax(x[t]), 0]))


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("T", [1, 2, 5])  # tiles of 8, 16 and 128 query rows
def test_attention_of_scores_of_any_size(T, sign):
    """Scores of 2^20 to 2^90, where binary32 numbers lie up to 2^66 apart: where the largest is the largest by far more than
    the sums' rounding, its value is the result.  (A score's error is below 2^-14 sum |q| max |k|: 128 products, 2^-23 each.)"""
    import torch
    fw = _fw()
    rng = np.random.default_rng(T)
    Hq, D, page, n = 8, 128, 32, 600
    cache = torch.full((-(-n // page), 1, fw.switchsd_kv4_bytes(page, D)), 0xff, dtype=torch.uint8, device="cuda")
    k, v = ref.bf16_round(rng.standard_normal((n, 1, D)) + 0.5), ref.bf16_round(rng.standard_normal((n, 1, D)) * 40)
    fw.switchsd_kv4_append(_bf16(k[None]), _bf16(v[None]), _i32(np.arange(n)[None]), cache, page=page)
    table, k, v = _i32(np.arange(-(-n // page))[None]), ref.dequantise(*ref.quantise(k)), ref.dequantise(*ref.quantise(v))
    for up in (18, 22, 23, 24, 25, 26, 28, 30, 40, 90):
        # (the largest of many scores that are all positive, or all negative)
        q = ref.bf16_round(sign * np.abs(rng.standard_normal((1, T, Hq, D)))) * 2.0 ** up
        out = torch.empty(1, T, Hq, D, dtype=torch.bfloat16, device="cuda")
        fw.switchsd_kv4_attention(_bf16(q), cache, table, _i32([n - T]), _i32([T]), out, page=page, scale=0.09)
        got, sure = out.double().cpu().numpy(), 0
        assert np.isfinite(got).all()
        for t in range(T):
            for h in range(Hq):
                x = k[:n - T + t + 1, 0] @ q[0, t, h]
                order = np.argsort(x)
                if x[order[-1]] - x[order[-2]] > 2.0 ** -14 * np.abs(q[0, t, h]).sum() * np.abs(k).max() + 2.0 ** 9:
                    want = v[order[-1], 0]
                    _near(got[0, t, h], want, np.abs(want))
                    sure += 1
        assert sure >= T * Hq // 2


def test_a_dimension_of_one_may_have_any_stride():
    """Strides that no address goes by: of a batch, a step or a head count of one."""
    import torch
    fw = _fw()
    rng = np.random.default_rng(3)
    D, page, n = 64, 16, 20
    cache, table, k, v = _filled(rng, n, 1, D, page)
    q = ref.bf16_round(rng.standard_normal((1, 1, 1, D)))
    flat = _bf16(q).reshape(-1)
    x = flat.as_strided((1, 1, 1, D), (D + 1, 3 * D + 5, 7, 1))
    out = torch.empty(1, 1, 1, D, dtype=torch.bfloat16, device="cuda")
    fw.switchsd_kv4_attention(x, cache, table, _i32([n - 1]), _i32([1]), out, page=page, scale=0.125)
    want, mag = ref.attention(q, [k], [v], [n - 1], [1], 0.125)
    _near(out.double().cpu().numpy(), want, mag)
    fw.switchsd_kv4_append(x, x, _i32([[3]]), cache, page=page)
    ok, ov = (torch.empty(1, 1, 1, D, dtype=torch.float16, device="cuda") for _ in range(2))
    fw.switchsd_kv4_read(cache, _i32([[3]]), ok, ov, page=page)
    held = ref.dequantise(*ref.quantise(q))
    assert np.array_equal(ok.double().cpu().numpy(), held) and np.array_equal(ov.double().cpu().numpy(), held)


@pytest.mark.parametrize("of", ["key", "value"])
@pytest.mark.parametrize("T,Hq,at", [(1, 4, 0), (2, 8, 1), (9, 4, 8), (9, 4, 3), (40, 4, 17), (9, 4, -5)])  # tiles of 8, 16 and 128 rows, two tiles
def test_attention_of_a_nan_reaches_those_who_see_it(T, Hq, at, of):
    """A NaN in the second group of 64 of the key or the value of new token `at` (-5: of a cached one): the tokens before it
    are as without it, it and those after it get NaN -- a value's in its 64 dimensions at least."""
    import torch
    fw = _fw()
    rng = np.random.default_rng(T + at)
    D, page, n = 128, 16, 300
    blocks = -(-n // page)
    cache = torch.full((blocks, 1, fw.switchsd_kv4_bytes(page, D)), 0xff, dtype=torch.uint8, device="cuda")
    k, v = ref.bf16_round(rng.standard_normal((n, 1, D))), ref.bf16_round(rng.standard_normal((n, 1, D)))
    kn, vn = k.copy(), v.copy()
    (kn if of == "key" else vn)[n - T + at, 0, 70] = np.nan
    fw.switchsd_kv4_append(_bf16(kn[None]), _bf16(vn[None]), _i32(np.arange(n)[None]), cache, page=page)
    k, v = ref.dequantise(*ref.quantise(k)), ref.dequantise(*ref.quantise(v))
    q = ref.bf16_round(rng.standard_normal((1, T, Hq, D)))
    out = torch.empty(1, T, Hq, D, dtype=torch.bfloat16, device="cuda")
    fw.switchsd_kv4_attention(_bf16(q), cache, _i32(np.arange(blocks)[None]), _i32([n - T]), _i32([T]), out, page=page, scale=0.09)
    got = out.double().cpu().numpy()
    want, mag = ref.attention(q, [k], [v], [n - T], [T], 0.09)
    first = max(at, 0)
    _near(got[:, :first], want[:, :first], mag[:, :first])
    assert np.isnan(got[:, first:, :, 64 if of == "value" else 0:]).all()
    if of == "value" and T * Hq <= 16:
        _near(got[:, first:, :, :64], want[:, first:, :, :64], mag[:, first:, :, :64])


@pytest.mark.parametrize("T,Hq,Hkv,D", [(1, 4, 2, 64), (5, 8, 2, 128)])
def test_attention_of_more_rows_than_threads(T, Hq, Hkv, D):
    """1500 ragged rows, some without new tokens, some of bad lengths: a thread looks up several; and twice the same, bit for
    bit."""
    import torch
    fw = _fw()
    rng = np.random.default_rng(D)
    B, page = 1500, 16
    lens, new = rng.integers(0, 70, B), rng.integers(0, T + 1, B)
    lens[::7] = 0
    need = -(-(lens + new) // page)
    blocks, pages = int(need.max()), int(need.sum())
    table, ids, at = np.full((B, blocks), -1), rng.permutation(pages), 0
    for b in range(B):
        table[b, :need[b]] = ids[at:at + need[b]]
        at += need[b]
    most = int((lens + new).max())
    k, v = ref.bf16_round(rng.standard_normal((B, most, Hkv, D))), ref.bf16_round(rng.standard_normal((B, most, Hkv, D)))
    p = np.arange(most)
    slots = np.where(p < (lens + new)[:, None], np.take_along_axis(table, np.minimum(p // page, blocks - 1)[None].repeat(B, 0), 1) * page + p % page, -1)
    cache = torch.full((pages, Hkv, fw.switchsd_kv4_bytes(page, D)), 0xff, dtype=torch.uint8, device="cuda")
    fw.switchsd_kv4_append(_bf16(k), _bf16(v), _i32(slots), cache, page=page)
    k, v = ref.dequantise(*ref.quantise(k)), ref.dequantise(*ref.quantise(v))
    q = ref.bf16_round(rng.standard_normal((B, T, Hq, D)))
    given = lens.copy()
    given[5::50] = -1
    outs = []
    for _ in range(2):
        out, status = torch.full((B, T, Hq, D), 9.0, dtype=torch.bfloat16, device="cuda"), torch.full((B,), 9, dtype=torch.int32, device="cuda")
        fw.switchsd_kv4_attention(_bf16(q), cache, _i32(table), _i32(given), _i32(new), out, page=page, scale=0.1, status=status)
        outs.append(out)
    assert torch.equal(outs[0], outs[1])
    assert np.array_equal(status.cpu().numpy(), np.where(given < 0, 2, 0))
    want, mag = ref.attention(q, [x[:n] for x, n in zip(k, lens + new)], [x[:n] for x, n in zip(v, lens + new)], lens, np.where(given < 0, 0, new), 0.1)
    _near(outs[0].double().cpu().numpy(), want, mag)


@pytest.mark.parametrize("T", [1, 2, 5])  # tiles of 8, 16 and 128 query rows
def test_attention_of_scores_far_below_zero(T):
    """All scores near -2^115, which is still a score: the largest takes it all."""
    import torch
    fw = _fw()
    rng = np.random.default_rng(T)
    Hq, D, page, n = 4, 64, 16, 500
    cache = torch.full((-(-n // page), 1, fw.switchsd_kv4_bytes(page, D)), 0xff, dtype=torch.uint8, device="cuda")
    k, v = ref.bf16_round(np.abs(rng.standard_normal((n, 1, D))) + 1), ref.bf16_round(rng.standard_normal((n, 1, D)))
    fw.switchsd_kv4_append(_bf16(k[None]), _bf16(v[None]), _i32(np.arange(n)[None]), cache, page=page)
    k, v = ref.dequantise(*ref.quantise(k)), ref.dequantise(*ref.quantise(v))
    q = ref.bf16_round(-np.abs(rng.standard_normal((1, T, Hq, D))) - 0.5) * 2.0 ** 108
    out = torch.empty(1, T, Hq, D, dtype=torch.bfloat16, device="cuda")
    fw.switchsd_kv4_attention(_bf16(q), cache, _i32(np.arange(-(-n // page))[None]), _i32([n - T]), _i32([T]), out, page=page, scale=1.0)
    got, sure = out.double().cpu().numpy(), 0
    for t in range(T):
        for h in range(Hq):
            x = k[:n - T + t + 1, 0] @ q[0, t, h]
            assert -2.0 ** 117 < x.min() and x.max() < -2.0 ** 113
            order = np.argsort(x)
            if x[order[-1]] - x[order[-2]] > 2.0 ** -14 * np.abs(q[0, t, h]).sum() * np.abs(k).max():
                _near(got[0, t, h], v[order[-1], 0], np.abs(v[order[-1], 0]))
                sure += 1
    assert sure >= T * Hq // 2
