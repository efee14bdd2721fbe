"""The operators of include/switchsd_target.h on the GPU, against plain implementations in 64 bits (target_ref.py).

Whole numbers, codes, scales and what the cache stands for are compared exactly.  Tolerances of the attention, from its
roundings: the output's (8 significant bits, 2^-8 of it, for bf16, 2^-11 for f16), the weights' 11 bits (2^-12 of each term, so at most that
of sum p |v|) and binary32 sums of at most 128 products in a score (their error times the score's size stays below 2^-12
for these inputs): 2^-8 |o| (or 2^-11 |o|) + 2^-10 sum p |v|.
"""
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
@pytest.mark.parametrize("B,T,page,blocks,room", [(1, 1, 16, 9, 1.0), (7, 5, 16, 40, 0.5), (33, 17, 64, 12, 0.4), (300, 9, 32, 30, 0.45),
                                                  (1025, 3, 16, 12, 0.5), (2500, 33, 256, 8, 0.5), (6, 700, 128, 90, 0.6)])
def test_map_follows_the_lengths(B, T, page, blocks, room):
    import torch
    fw = _fw()
    rng = np.random.default_rng(B + T)
    pages = max(2, int(B * blocks * room))
    free = rng.permutation(pages).astype(np.int32)
    st = ref.MapState(B, blocks, free)
    table, held = torch.full((B, blocks), -1, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    fl, fc = _i32(free), _i32([pages])
    lens = np.zeros(B, np.int64)
    for step in range(6):
        kind = rng.random(B)
        lens = np.where(kind < 0.2, 0, np.where(kind < 0.5, rng.integers(0, page * blocks + 1, B), np.minimum(lens + rng.integers(0, T + 1, B), page * blocks)))
        new = rng.integers(0, T + 1, B)
        new[kind < 0.1] = 0
        if step == 3:
            lens[0], new[-1] = -1, T + 1            # bad rows keep what they hold
        if step == 4:
            lens[B // 2] = page * blocks            # asks for more than a row's table has
            new[B // 2] = 1
        slots, status = torch.full((B, T), 7, dtype=torch.int32, device="cuda"), torch.full((B,), 7, dtype=torch.int32, device="cuda")
        # the lengths arrive shifted, as a context's do
        fw.switchsd_kv_map(_i32(lens + 1), _i32(new - 1), table, held, fl, fc, slots, page=page, lens_add=-1, new_add=1, status=status)
        want_slots, want_status = st.step(lens.tolist(), new.tolist(), T, page)
        wt, wh, wf, wc = st.arrays()
        assert np.array_equal(status.cpu().numpy(), want_status)
        assert int(fc.cpu()[0]) == wc
        assert np.array_equal(held.cpu().numpy(), wh)
        assert np.array_equal(table.cpu().numpy(), wt)
        assert np.array_equal(fl.cpu().numpy(), wf)
        assert np.array_equal(slots.cpu().numpy(), want_slots)
        lens = np.maximum(lens, 0)
    everything = np.concatenate([wf[:wc], wt[wt >= 0]])
    assert np.array_equal(np.sort(everything), np.arange(pages))  # no page lost, none held twice


# --- the cache ----------------------------------------------------------------------------------------------------
def _values(rng, shape, f16):
    """Values of many sizes, with whole groups of special ones, rounded to the type."""
    x = rng.standard_normal(shape) * np.exp(rng.normal(0, 2, shape[:-1]))[..., None]
    flat = x.reshape(-1, shape[-1])
    n = len(flat)
    flat[0 % n] = 0
    flat[3 % n] = 2.0 ** -23 * rng.standard_normal(shape[-1])        # scales among f16's smallest
    flat[5 % n, :64] = np.linspace(-8, 7.0, 64)                       # a scale of exactly 1
    flat[7 % n, :64] = rng.integers(-16, 15, 64) * 0.5                # ties
    flat[9 % n, :64] = -np.abs(flat[9 % n, :64])
    flat[11 % n] = 50000.0 * np.sign(flat[11 % n])
    if not f16:
        flat[13 % n] = 3e9 * np.sign(flat[13 % n])                    # beyond the largest scale: saturates
    return x.astype(np.float16).astype(np.float64) if f16 else ref.bf16_round(x)


def _tensor(x, f16):
    import torch
    return torch.from_numpy(np.asarray(x, np.float64)).to(torch.float16 if f16 else torch.bfloat16).cuda()


@pytest.mark.parametrize("f16", [False, True])
@pytest.mark.parametrize("D,page,H,T", [(128, 16, 3, 1), (64, 32, 2, 5), (128, 64, 1, 17), (64, 16, 5, 40), (128, 128, 2, 9), (64, 256, 1, 33)])
def test_append_then_read(f16, D, page, H, T):
    """Three appends in a row to rows of odd lengths, one of them without new tokens; the values, the bytes' layout, and
    what was in the cache before."""
    import torch
    fw = _fw()
    rng = np.random.default_rng(D + page + T)
    B = 4
    cache = fw.KVCache(B, T, layers=1, heads=H, dim=D, pages=B * (400 // page + 2), max_len=400, page=page)
    lens = rng.integers(0, 3 * page // 2, B)
    lens[1] = 0
    held = {}
    for step in range(3):
        new = rng.integers(1, T + 1, B)
        new[step] = 0
        new[3] = T
        cache.map(_i32(lens), _i32(new))
        slots = cache.slots.cpu().numpy()
        k, v = _values(rng, (B, T, H, D), f16), _values(rng, (B, T, H, D), f16)
        # views of a fused projection: strides of tokens and heads that are not the sizes
        x = torch.zeros(B, T, 3 * H + 1, D, dtype=torch.float16 if f16 else torch.bfloat16, device="cuda")
        x[:, :, 1:H + 1], x[:, :, 2 * H + 1:] = _tensor(k, f16), _tensor(v, f16)
        cache.append(0, x[:, :, 1:H + 1], x[:, :, 2 * H + 1:])
        (kc, ks), (vc, vs) = ref.quantise(k), ref.quantise(v)
        for b in range(B):
            for t in range(new[b]):
                for h in range(H):
                    held[(slots[b, t], h)] = (kc[b, t, h], vc[b, t, h], ks[b, t, h], vs[b, t, h])
        gk, gv = (a.double().cpu().numpy() for a in cache.read(0, cache.slots))
        inside = (np.arange(T) < new[:, None])[..., None, None]
        assert np.array_equal(gk, np.where(inside, ref.dequantise(kc, ks), 0))
        assert np.array_equal(gv, np.where(inside, ref.dequantise(vc, vs), 0))
        lens = lens + new
    raw = cache.data[0].cpu().numpy()
    for (slot, h), want in held.items():
        for got, w in zip(ref.decode_slot(raw, page, D, slot, h), want):
            assert np.array_equal(got, w)


@pytest.mark.parametrize("f16", [False, True])
def test_append_of_nan_and_infinity(f16):
    """A NaN makes its group NaN and leaves the others; an infinity saturates."""
    import torch
    fw = _fw()
    x = np.random.default_rng(0).standard_normal((1, 3, 1, 128))
    x = x.astype(np.float16).astype(np.float64) if f16 else ref.bf16_round(x)
    y = x.copy()
    y[0, 0, 0, 70] = np.nan
    y[0, 1, 0, 3] = np.inf
    y[0, 2, 0, 127] = -np.inf
    cache = torch.zeros(1, 1, fw.switchsd_kv4_bytes(16, 128), dtype=torch.uint8, device="cuda")
    slots = _i32([[0, 1, 2]])
    out = [torch.empty(1, 3, 1, 128, dtype=torch.float16, device="cuda") for _ in range(2)]
    fw.switchsd_kv4_append(_tensor(y, f16), _tensor(y, f16), slots, cache, page=16)
    fw.switchsd_kv4_read(cache, slots, *out, page=16)
    codes, s = ref.quantise(x)
    for o in out:
        g = o.double().cpu().numpy()
        assert np.isnan(g[0, 0, 0, 64:]).all()
        assert np.array_equal(g[0, 0, 0, :64], ref.dequantise(codes, s)[0, 0, 0, :64])
        assert g[0, 1, 0, 3] == 7 * 8128 and (np.delete(g[0, 1, 0, :64], 3) == 0).all()
        assert g[0, 2, 0, 127] == -8 * 8128 and (g[0, 2, 0, 64:127] == 0).all()


# --- attention ----------------------------------------------------------------------------------------------------
def _cache_of(rng, B, H, D, page, lens, new, blocks, garbage=0xff):
    """A cache of pages in random order holding random tokens, everything else filled with `garbage` (0xff: NaN scales).
    Returns the device cache, the table and the rows' keys and values."""
    import torch
    fw = _fw()
    need = [-(-(int(a) + int(n)) // page) for a, n in zip(lens, new)]
    pages = sum(need) + 2
    ids = rng.permutation(pages)
    table = np.full((B, blocks), -1, np.int32)
    at = 0
    for b in range(B):
        table[b, :need[b]] = ids[at:at + need[b]]
        at += need[b]
    cache = torch.full((pages, H, fw.switchsd_kv4_bytes(page, D)), garbage, dtype=torch.uint8, device="cuda")
    ks, vs = [], []
    for b in range(B):
        n = int(lens[b] + new[b])
        k = rng.standard_normal((n, H, D)) * np.where(np.arange(D) % 32 == 5, 4, 1) + np.where(np.arange(D) % 64 == 9, 2, 0)
        v = rng.standard_normal((n, H, D)) * 0.5 * np.exp(rng.normal(0, 1, (n, H, 1)))
        k, v = ref.bf16_round(k), ref.bf16_round(v)
        if n:
            p = np.arange(n)
            slots = table[b][p // page].astype(np.int64) * page + p % page
            fw.switchsd_kv4_append(_tensor(k[None], False), _tensor(v[None], False), _i32(slots[None]), cache, page=page)
        ks.append(ref.dequantise(*ref.quantise(k)))
        vs.append(ref.dequantise(*ref.quantise(v)))
    return cache, table, ks, vs


def _check(got, want, mag, f16):
    tol = (2.0 ** -11 if f16 else 2.0 ** -8) * np.abs(want) + 2.0 ** -10 * mag
    err = np.abs(got - want)
    assert np.all(err <= tol), (float(np.max(err / np.maximum(tol, 1e-30))), np.argwhere(err > tol)[:4])


def _attend(q, cache, table, lens, new, page, f16, scale, **kw):
    import torch
    fw = _fw()
    x = _tensor(q, f16) if isinstance(q, np.ndarray) else q
    out = torch.full(x.shape, 9.0, dtype=x.dtype, device="cuda")
    fw.switchsd_kv4_attention(x, cache, _i32(table), _i32(lens), _i32(new), out, page=page, scale=scale, **kw)
    return out.double().cpu().numpy()


CASES = [
    # Hq, Hkv, D, page, T, lens, new
    (4, 1, 128, 16, 1, [0, 1, 15, 16, 31], [1, 1, 1, 1, 1]),                   # ends of pages, a single key
    (8, 2, 64, 32, 1, [0, 100, 37, 255], [0, 1, 1, 1]),                        # a row without new tokens
    (5, 5, 128, 64, 3, [0, 61, 62, 63, 64, 0], [3, 3, 2, 1, 3, 0]),            # one query head a key head, new tokens over a page's end
    (16, 2, 128, 16, 5, [500, 3, 77], [5, 4, 1]),                              # 40 query rows a key head
    (20, 4, 64, 128, 17, [300, 0, 130], [17, 17, 9]),                          # 85
    (20, 4, 128, 32, 33, [700, 31], [33, 20]),                                 # 165: more than one tile of query rows
    (64, 1, 128, 256, 2, [1000, 255], [2, 1]),                                 # the widest group
    (3, 1, 64, 16, 1, [2049, 5], [1, 1]),                                      # an odd group
    (8, 1, 128, 16, 1, [9000, 40, 1, 3000], [1, 1, 1, 1]),                     # very ragged
    (4, 4, 128, 64, 9, [4000], [9]),                                           # one long row
    (4, 2, 128, 16, 70, [5], [70]),                                            # a prompt's chunk
]


@pytest.mark.parametrize("f16", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c[:5]))
def test_attention(case, f16):
    Hq, Hkv, D, page, T, lens, new = case
    rng = np.random.default_rng(Hq * 1000 + D + T)
    B = len(lens)
    lens, new = np.array(lens), np.array(new)
    blocks = int(-(-(lens + new).max() // page)) + 2
    cache, table, ks, vs = _cache_of(rng, B, Hkv, D, page, lens, new, blocks)
    q = rng.standard_normal((B, T, Hq, D)) * 0.7
    q = q.astype(np.float16).astype(np.float64) if f16 else ref.bf16_round(q)
    scale = float(np.float32(D ** -0.5))
    want, mag = ref.attention(q, ks, vs, lens, new, scale)
    _check(_attend(q, cache, table, lens, new, page, f16, scale), want, mag, f16)


@pytest.mark.parametrize("Hq,Hkv,T,spread", [(4, 4, 1, 1.0), (12, 4, 3, 1.0), (8, 4, 9, 1.0), (8, 4, 9, 6.0), (20, 4, 33, 1.0)])
def test_attention_of_many_units_a_cta(Hq, Hkv, T, spread):
    """Enough keys that a CTA goes over many of an item's units and over several items; with spread queries the running maximum
    keeps rising by more than the kernel lets its reference lag, and weights get small.  (The spread scores carry up to
    2^-24 * 128 of their products' size in error: see the next test.)"""
    rng = np.random.default_rng(T + Hq)
    B, D, page = 6, 64, 32
    lens = np.array([9000, 4100, 7777, 130, 8192, 6001])
    new = np.minimum(np.array([T, max(1, T - 2), T, 1, T, T]), T)
    cache, table, ks, vs = _cache_of(rng, B, Hkv, D, page, lens, new, 300)
    q = ref.bf16_round(rng.standard_normal((B, T, Hq, D)) * 0.7 * spread)
    want, mag = ref.attention(q, ks, vs, lens, new, 0.125)
    big = np.abs(q).sum(-1).max() * max(np.abs(k).max() for k in ks) * 0.125
    _check(_attend(q, cache, table, lens, new, page, False, 0.125), want, mag * (1 + 2 ** 10 * big * 2.0 ** -23 * (spread > 1)), False)


def test_attention_shifted_lengths_strides_and_status():
    """Lengths with lens_add and new_add, queries as a view of a fused projection, and rows with bad lengths among good ones."""
    import torch
    fw = _fw()
    rng = np.random.default_rng(5)
    Hq, Hkv, D, page, T = 8, 2, 128, 16, 4
    lens, new = np.array([20, 33, 7, 0, 90]), np.array([4, 2, 1, 4, 3])
    B = len(lens)
    cache, table, ks, vs = _cache_of(rng, B, Hkv, D, page, lens, new, 6)
    x = torch.from_numpy(rng.standard_normal((B, T, Hq + 2 * Hkv, D))).to(torch.bfloat16).cuda()
    q = x[:, :, :Hq]
    want, mag = ref.attention(q.double().cpu().numpy(), ks, vs, lens, new, 0.05)
    want[2] = want[4] = 0
    bad_l, bad_n = lens + 1, new - 1
    bad_l[2] = -3
    bad_n[4] = T
    status = torch.full((B,), 9, dtype=torch.int32, device="cuda")
    got = _attend(q, cache, table, bad_l, bad_n, page, False, 0.05, lens_add=-1, new_add=1, status=status)
    _check(got, want, mag, False)
    assert status.cpu().tolist() == [0, 0, 2, 0, 2]
    # a row whose tokens do not fit its table
    out = torch.empty(B, T, Hq, D, dtype=torch.bfloat16, device="cuda")
    fw.switchsd_kv4_attention(q, cache, _i32(table), _i32(np.array([20, 33, 7, 0, 94])), _i32(new), out, page=page, status=status)
    assert status.cpu().tolist() == [0, 0, 0, 0, 2] and not out[4].any()


def test_attention_does_not_see_pages_outside_the_pool():
    rng = np.random.default_rng(6)
    Hq, Hkv, D, page, T = 4, 1, 64, 16, 2
    lens, new = np.array([70, 20, 16]), np.array([2, 1, 2])
    cache, table, ks, vs = _cache_of(rng, 3, Hkv, D, page, lens, new, 6)
    seen = [np.ones(int(a + n), bool) for a, n in zip(lens, new)]
    table[0, 1], table[0, 3] = -1, 1 << 30
    seen[0][16:32] = seen[0][48:64] = False
    table[1, :2] = -5
    seen[1][:] = False
    q = ref.bf16_round(rng.standard_normal((3, T, Hq, D)))
    want, mag = ref.attention(q, ks, vs, lens, new, 0.125, seen)
    _check(_attend(q, cache, table, lens, new, page, False, 0.125), want, mag, False)


@pytest.mark.parametrize("T,Hq", [(1, 4), (9, 20)])
def test_attention_of_extreme_values(T, Hq):
    """Scores far apart, values whose scales differ by 2^12 between tokens and by 2^12 between the two groups, a constant
    row of zeros, and a key of NaN that only the last token sees."""
    import torch
    fw = _fw()
    rng = np.random.default_rng(7)
    Hkv, D, page, n = 1, 128, 32, 200
    k, v = rng.standard_normal((n, Hkv, D)), rng.standard_normal((n, Hkv, D))
    v *= np.exp2(rng.integers(-6, 7, (n, 1, 1)))
    v[..., 64:] *= 2.0 ** -12
    v[17] = 0
    k[:, :, :8] *= 6
    k, v = ref.bf16_round(k), ref.bf16_round(v)
    kn = k.copy()
    kn[n - 1, 0, 5] = np.nan
    cache = torch.zeros(7, Hkv, fw.switchsd_kv4_bytes(page, D), dtype=torch.uint8, device="cuda")
    slots = np.arange(n)[None]
    fw.switchsd_kv4_append(_tensor(kn[None], False), _tensor(v[None], False), _i32(slots), cache, page=page)
    kd, vd = ref.dequantise(*ref.quantise(k)), ref.dequantise(*ref.quantise(v))
    lens, new = np.array([n - T]), np.array([T])
    q = ref.bf16_round(rng.standard_normal((1, T, Hq, D)) * 3)
    want, mag = ref.attention(q, [kd], [vd], lens, new, 0.2)
    got = _attend(q, cache, np.arange(7)[None], lens, new, page, False, 0.2)
    assert np.isnan(got[0, T - 1]).all()
    # the scores reach some hundreds here: binary32 sums of 128 products leave up to 2^-24 * 2 * 128 of the largest product
    # sum in each, so the weights carry that much more relative error
    big = np.abs(q[0]).sum(-1).max() * np.abs(kd).max() * 0.2
    mag = mag * (1 + 2 ** 10 * big * 2.0 ** -23)
    _check(got[:, :T - 1], want[:, :T - 1], mag[:, :T - 1], False)


@pytest.mark.parametrize("T,Hq", [(1, 4), (9, 4)])
def test_attention_of_the_largest_scales(T, Hq):
    """Values and keys at every size of a scale up to the largest (8128), 2^-12 apart from key to key in the scores."""
    import torch
    fw = _fw()
    rng = np.random.default_rng(9)
    Hkv, D, page, n = 1, 128, 32, 100
    k, v = rng.standard_normal((n, Hkv, D)), rng.standard_normal((n, Hkv, D))
    size = np.exp2(np.arange(n) % 15)[:, None, None]
    k, v = ref.bf16_round(k * size), ref.bf16_round(v * size)
    k[n // 2], v[n // 3] = 60000, -64000
    k, v = ref.bf16_round(k), ref.bf16_round(v)
    cache = torch.zeros(4, Hkv, fw.switchsd_kv4_bytes(page, D), dtype=torch.uint8, device="cuda")
    fw.switchsd_kv4_append(_tensor(k[None], False), _tensor(v[None], False), _i32(np.arange(n)[None]), cache, page=page)
    kd, vd = ref.dequantise(*ref.quantise(k)), ref.dequantise(*ref.quantise(v))
    lens, new = np.array([n - T]), np.array([T])
    q = ref.bf16_round(rng.standard_normal((1, T, Hq, D)))
    scale = 2.0 ** -20
    want, mag = ref.attention(q, [kd], [vd], lens, new, scale)
    _check(_attend(q, cache, np.arange(4)[None], lens, new, page, False, scale), want, mag, False)


def test_attention_past_32_bit_offsets():
    """The pool's last pages of a cache of more than 4 GiB."""
    import torch
    fw = _fw()
    Hq, Hkv, D, page = 8, 8, 128, 128
    size = fw.switchsd_kv4_bytes(page, D)
    pages = (5 << 30) // (Hkv * size)
    rng = np.random.default_rng(8)
    n = 300
    k, v = ref.bf16_round(rng.standard_normal((n, Hkv, D))), ref.bf16_round(rng.standard_normal((n, Hkv, D)))
    cache = torch.empty(pages, Hkv, size, dtype=torch.uint8, device="cuda")
    cache[-4:] = 0xff
    table = np.array([[pages - 1, pages - 3, pages - 2]])
    p = np.arange(n)
    slots = table[0][p // page].astype(np.int64) * page + p % page
    fw.switchsd_kv4_append(_tensor(k[None], False), _tensor(v[None], False), _i32(slots[None]), cache, page=page)
    q = ref.bf16_round(rng.standard_normal((1, 1, Hq, D)))
    kd, vd = ref.dequantise(*ref.quantise(k)), ref.dequantise(*ref.quantise(v))
    want, mag = ref.attention(q, [kd], [vd], [n - 1], [1], 0.09)
    _check(_attend(q, cache, table, [n - 1], [1], page, False, 0.09), want, mag, False)


def test_attention_on_another_stream_and_in_a_graph():
    """The call on a side stream, and recorded with the map and the append into a graph whose replays follow the lengths."""
    import torch
    fw = _fw()
    B, T, H, Hq, D = 3, 2, 2, 8, 128
    torch.manual_seed(0)
    cache = fw.KVCache(B, T, layers=1, heads=H, dim=D, pages=64, max_len=256, page=16)
    lens, new = _i32([0, 0, 0]), _i32([2, 1, 2])
    x = torch.randn(B, T, Hq + 2 * H, D, device="cuda").to(torch.bfloat16)
    out = torch.empty(B, T, Hq, D, dtype=torch.bfloat16, device="cuda")

    def step():
        cache.map(lens, new)
        cache.append(0, x[:, :, Hq:Hq + H], x[:, :, Hq + H:])
        cache.attend(0, x[:, :, :Hq], out)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    n = [0, 0, 0]
    hist = [[[], []] for _ in range(B)]
    rng = np.random.default_rng(1)
    for it in range(20):
        x.copy_(torch.from_numpy(rng.standard_normal(x.shape)))
        lens.copy_(_i32(n))
        g.replay()
        xs = x.double().cpu().numpy()
        new_h = new.cpu().numpy()
        ks, vs = [], []
        for b in range(B):
            for t in range(new_h[b]):
                hist[b][0].append(ref.dequantise(*ref.quantise(xs[b, t, Hq:Hq + H])))
                hist[b][1].append(ref.dequantise(*ref.quantise(xs[b, t, Hq + H:])))
            ks.append(np.array(hist[b][0]))
            vs.append(np.array(hist[b][1]))
        want, mag = ref.attention(xs[:, :, :Hq], ks, vs, n, new_h, float(np.float32(D ** -0.5)))
        _check(out.double().cpu().numpy(), want, mag, False)
        for b in range(B):  # the last token of a row is rejected now and then
            keep = int(new_h[b]) - int(it % 3 == 0 and new_h[b] == 2)
            drop = int(new_h[b]) - keep
            if drop:
                hist[b][0].pop()
                hist[b][1].pop()
            n[b] += keep


# --- logits -------------------------------------------------------------------------------------------------------
def _logit_inputs(rng, B, T, V, cap, dtype, nbias, masked, drafted=True):
    x = rng.standard_normal((B, T, V)) * 3
    if dtype == "bf16":
        x = ref.bf16_round(x)
    elif dtype == "f16":
        x = x.astype(np.float16).astype(np.float64)
    else:
        x = x.astype(np.float32).astype(np.float64)
    ctx = np.minimum(rng.zipf(1.2, (B, cap)), 4 * V).astype(np.int32) - 3   # some ids outside [0, V)
    draft = rng.integers(0, min(V, 7), (B, max(1, T - 1))).astype(np.int32) if drafted else None
    if drafted:
        draft[0, 0] = -1
    lens = rng.integers(0, cap + 1, B)
    lens[0] = cap
    new = rng.integers(0, T + 1, B)
    new[-1] = T
    r = rng.random((4, B)).astype(np.float32)
    ids = bias = mask = None
    if nbias:
        ids = rng.integers(-2, V + 2, (B, nbias)).astype(np.int32)
        ids[:, -1] = ids[:, 0]                                               # named twice: the last one counts
        bias = (rng.standard_normal((B, nbias)) * 5).astype(np.float32)
        bias[0, 1 % nbias] = np.inf
    if masked:
        mask = rng.integers(-2**31, 2**31, (B, T, (V + 31) // 32 + 1), dtype=np.int64).astype(np.int32)
        mask[0, 0] = 0
    prompt = (lens * r[3]).astype(np.int32)
    return dict(x=x, ctx=ctx, lens=lens, draft=draft, new=new, rep=1 + r[0], freq=r[1], pres=r[2] * 2, prompt=prompt, bias_ids=ids, bias=bias, mask=mask)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("B,T,V,cap,nbias,masked,pad", [(1, 1, 1, 4, 0, False, 0), (3, 2, 5, 8, 3, True, 0), (2, 5, 1000, 64, 9, True, 0),
                                                        (2, 3, 50257, 300, 0, True, 0), (5, 4, 32003, 1200, 33, False, 5), (1, 70, 777, 128, 4, True, 3),
                                                        (40, 2, 4099, 2000, 1, True, 1), (2, 2, 152064, 5000, 300, True, 0)])
def test_logits(dtype, B, T, V, cap, nbias, masked, pad):
    """The processed logits and the greedy tokens: bit for bit those of the formula in binary32, and near those in 64 bits
    (three roundings of values below 2^7, and the type's own)."""
    import torch
    fw = _fw()
    rng = np.random.default_rng(V + T)
    i = _logit_inputs(rng, B, T, V, cap, dtype, nbias, masked)
    tt = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[dtype]
    buf = torch.full((B, T, V + pad), 1000.0, dtype=tt, device="cuda")
    buf[..., :V] = torch.from_numpy(i["x"]).to(tt).cuda()
    x = buf[..., :V]
    out = torch.full((B, T, V), 55.0, dtype=tt, device="cuda")
    argmax, status = torch.full((B, T), 9, dtype=torch.int32, device="cuda"), torch.full((B,), 9, dtype=torch.int32, device="cuda")
    f = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    kw = dict(ctx_tokens=_i32(i["ctx"]), ctx_lens=_i32(i["lens"]), draft=_i32(i["draft"]), new_lens=_i32(i["new"] - 1), new_add=1, rep=f(i["rep"]), freq=f(i["freq"]),
              pres=f(i["pres"]), prompt_lens=_i32(i["prompt"]), bias_ids=f(i["bias_ids"]), bias=f(i["bias"]), mask=f(i["mask"]), status=status)
    fw.switchsd_logits(x, out=out, argmax=argmax, **kw)
    args = [i[n] for n in ("x", "ctx", "lens", "draft", "new", "rep", "freq", "pres", "prompt", "bias_ids", "bias", "mask")]
    want, best = ref.logits(*args, dtype=np.float32)
    exact, _ = ref.logits(*args, dtype=np.float64)
    assert np.array_equal(argmax.cpu().numpy(), best)
    assert (status == 0).all()
    got = out.float().cpu().numpy()
    inside = np.arange(T) < i["new"][:, None]
    assert (got[~inside] == 55.0).all()
    assert np.array_equal(got[inside], torch.from_numpy(want).to(tt).float().numpy()[inside])
    fin = np.isfinite(exact) & inside[..., None]
    own = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}[dtype]
    size = np.abs(exact[fin]) + 2 ** 7
    assert np.all(np.abs(got[fin] - exact[fin]) <= 3 * 2.0 ** -24 * size + own * np.abs(exact[fin]) + 2.0 ** -25)
    # tokens alone, and in place
    again = torch.full((B, T), 9, dtype=torch.int32, device="cuda")
    fw.switchsd_logits(x, argmax=again, **kw)
    assert torch.equal(again, argmax)
    fw.switchsd_logits(x, out=x, **kw)
    assert torch.equal(x[torch.from_numpy(inside).cuda()], out[torch.from_numpy(inside).cuda()])
    assert pad == 0 or (buf[..., V:] == 1000.0).all()


def test_logits_without_a_context_and_special_values():
    """Infinities and NaN: a NaN and -inf are never chosen, masked ones leave nothing behind; ties go to the lowest token."""
    import torch
    fw = _fw()
    V = 300
    x = torch.zeros(1, 6, V, dtype=torch.float32, device="cuda")
    x[0, 0, [7, 200]] = 5.0                                  # a tie
    x[0, 1] = float("nan")
    x[0, 1, 99] = -3.0                                       # NaN around it
    x[0, 2] = float("-inf")
    x[0, 3, 4], x[0, 3, 250] = float("nan"), float("inf")    # both masked
    x[0, 3, 250 - 32] = 1.0
    x[0, 4, 250] = float("inf")
    x[0, 5] = float("nan")
    mask = torch.full((1, 6, 10), -1, dtype=torch.int32, device="cuda")
    m = np.full(10, -1, np.int32)
    for v in (4, 250):
        m[v // 32] = np.int32(np.uint32(m[v // 32].view(np.uint32) & ~np.uint32(1 << (v % 32))).view(np.int32))
    mask[0, 3] = torch.from_numpy(m).cuda()
    out, best = torch.empty_like(x), torch.empty(1, 6, dtype=torch.int32, device="cuda")
    fw.switchsd_logits(x, mask=mask, out=out, argmax=best)
    assert best.cpu().tolist() == [[7, 99, -1, 218, 250, -1]]
    want = x.clone()
    want[0, 3, 4] = want[0, 3, 250] = float("-inf")
    assert torch.equal(out.nan_to_num(123.0, 1e30, -1e30), want.nan_to_num(123.0, 1e30, -1e30))


def test_logits_bad_lengths_leave_the_row_out():
    import torch
    fw = _fw()
    x = torch.randn(4, 2, 100, device="cuda")
    ctx = torch.zeros(4, 8, dtype=torch.int32, device="cuda")
    best, status = torch.full((4, 2), 9, dtype=torch.int32, device="cuda"), torch.full((4,), 9, dtype=torch.int32, device="cuda")
    fw.switchsd_logits(x, ctx_tokens=ctx, ctx_lens=_i32([8, 9, -1, 0]), new_lens=_i32([2, 2, 2, 3]), argmax=best, status=status)
    assert status.cpu().tolist() == [0, 2, 2, 2]
    assert best[0].tolist() == x[0].argmax(-1).tolist() and (best[1:] == -1).all()


def test_operators_refuse_what_they_do_not_take():
    """The binding's and the library's checks on real tensors: types, shapes, strides, alignment, devices."""
    import torch
    fw = _fw()
    B, T, H, D, page = 2, 3, 2, 64, 16
    cache = torch.zeros(4, H, fw.switchsd_kv4_bytes(page, D), dtype=torch.uint8, device="cuda")
    k = torch.zeros(B, T, H, D, dtype=torch.bfloat16, device="cuda")
    slots = torch.zeros(B, T, dtype=torch.int32, device="cuda")
    table, lens, new = torch.zeros(B, 2, dtype=torch.int32, device="cuda"), _i32([0, 0]), _i32([1, 1])
    with pytest.raises(TypeError):
        fw.switchsd_kv4_append(k.float(), k.float(), slots, cache, page=page)
    with pytest.raises(TypeError):
        fw.switchsd_kv4_append(k, k.half(), slots, cache, page=page)
    with pytest.raises(ValueError):
        fw.switchsd_kv4_append(k, k, slots, cache, page=32)
    with pytest.raises(ValueError):
        fw.switchsd_kv4_append(k.transpose(2, 3), k, slots, cache, page=page)
    odd = torch.zeros(B * T * H * (D + 1) + 8, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(RuntimeError):
        fw.switchsd_kv4_append(odd[1:1 + B * T * H * D].view(B, T, H, D), k, slots, cache, page=page)       # not 16-byte aligned
    with pytest.raises(RuntimeError):
        fw.switchsd_kv4_append(odd.as_strided((B, T, H, D), (T * H * (D + 1), H * (D + 1), D + 1, 1)), k, slots, cache, page=page)
    out = torch.empty_like(k)
    with pytest.raises(TypeError):
        fw.switchsd_kv4_attention(k, cache, table.long(), lens, new, out, page=page)
    with pytest.raises(TypeError):
        fw.switchsd_kv4_attention(k, cache, table, lens.cpu(), new, out, page=page)
    with pytest.raises(ValueError):
        fw.switchsd_kv4_attention(k, cache, table, lens, new, out[:, :, :1], page=page)
    q3 = torch.zeros(B, T, 3, D, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(RuntimeError):
        fw.switchsd_kv4_attention(q3, cache, table, lens, new, torch.empty_like(q3), page=page)             # 3 query heads, 2 key heads
    with pytest.raises(ValueError):
        fw.KVCache(1, 1, layers=1, heads=1, dim=96, pages=1, max_len=16)
    x = torch.zeros(B, T, 40, device="cuda")
    with pytest.raises(ValueError):
        fw.switchsd_logits(x, ctx_tokens=table, argmax=slots)
    with pytest.raises(RuntimeError):
        fw.switchsd_logits(x)                                                                               # nothing to write
    with pytest.raises(RuntimeError):
        fw.switchsd_logits(x, argmax=slots, mask=torch.zeros(B, T, 1, dtype=torch.int32, device="cuda"))    # too few words
