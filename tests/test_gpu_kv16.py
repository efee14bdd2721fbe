"""The 16-bit paged cache and its attention on the GPU, against plain implementations in 64 bits.

Append and read are copies, compared bit for bit.  Tolerances of the attention, from its roundings: the output's, at most
half a step (2^-8 of it for bf16, 2^-11 for f16); the weights', the same of each term, so at most that of sum p |v|; f16
weights below 2^-25 of the largest have an absolute error of 2^-36 of it, which 2^14 keys make 2^-22; and binary32 sums of
at most 128 exact products in a score, whose error, 2^-17 of sum |q k| at the worst, stays below 2^-10 for these inputs
(sum |q k| * scale below 100), so 2^-10 of sum p |v| again, and 2^-13 where the scores are of ordinary size:
e |o| + (e + 2^-10) sum p |v|, e = 2^-8 or 2^-11.
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


def _dtype(f16):
    import torch
    return torch.float16 if f16 else torch.bfloat16


def _round(x, f16):
    return np.asarray(x).astype(np.float16).astype(np.float64) if f16 else ref.bf16_round(x)


def _tensor(x, f16):
    import torch
    return torch.from_numpy(np.asarray(x, np.float64)).to(_dtype(f16)).cuda()


def _numpy(t):
    return t.double().cpu().numpy()


# --- append and read ----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("f16", [False, True])
@pytest.mark.parametrize("B,D,page,H,T", [(1, 128, 16, 1, 1), (4, 128, 16, 3, 7), (3, 64, 32, 2, 5), (2, 128, 64, 8, 300), (5, 64, 256, 5, 33), (700, 64, 16, 1, 2)])
def test_append_then_read(f16, B, D, page, H, T):
    """Slots in any order, some outside the pool; views of a fused projection; bits of every kind, and what lies beside."""
    import torch
    fw = _fw()
    rng = np.random.default_rng(D + page + T + B)
    pages = -(-B * T // page) + 2
    slots = rng.permutation(pages * page)[:B * T].reshape(B, T)
    slots[rng.random((B, T)) < 0.2] = -1
    slots[rng.random((B, T)) < 0.05] = pages * page
    before = torch.from_numpy(rng.integers(-2**15, 2**15, (pages, 2, H, page, D)).astype(np.int16)).cuda()
    x = torch.from_numpy(rng.integers(-2**15, 2**15, (B, T, 3 * H + 1, D)).astype(np.int16)).cuda()
    cache = before.clone().view(_dtype(f16))
    k, v = x[:, :, 1:H + 1], x[:, :, 2 * H + 1:]
    fw.switchsd_kv16_append(k.view(_dtype(f16)), v.view(_dtype(f16)), _i32(slots), cache)
    want = before.clone()
    b, t = np.nonzero((slots >= 0) & (slots < pages * page))
    s = slots[b, t]
    want[s // page, 0, :, s % page], want[s // page, 1, :, s % page] = k[b, t], v[b, t]
    assert torch.equal(cache.view(torch.int16), want)
    out = torch.full((2, B, T, H, D), 7, dtype=torch.int16, device="cuda").view(_dtype(f16))
    fw.switchsd_kv16_read(cache, _i32(slots), out[0], out[1])
    want_out = torch.zeros(2, B, T, H, D, dtype=torch.int16, device="cuda")
    want_out[0, b, t], want_out[1, b, t] = k[b, t], v[b, t]
    assert torch.equal(out.view(torch.int16), want_out)


# --- attention ----------------------------------------------------------------------------------------------------
class Setup:
    """Contexts in a paged cache whose every other place is NaN, and the rows' keys and values in 64 bits."""

    def __init__(self, rng, lens, new, Hkv, D, page, f16, T, q_size=0.75, spare=2, first_page=0, pages=None, k_scale=1.0):
        import torch
        self.B, self.T, self.Hkv, self.D, self.page, self.f16 = len(lens), T, Hkv, D, page, f16
        lens, new = np.asarray(lens), np.asarray(new)
        self.lens, self.new = lens, new
        need = [max(0, -(-(max(0, l) + max(0, n)) // page)) for l, n in zip(lens, new)]
        total = sum(need)
        pages = pages or first_page + total + spare
        order = first_page + rng.permutation(pages - first_page)[:total]
        self.table = np.full((self.B, max(need) + 1), -1, np.int64)
        self.k, self.v = [], []
        self.cache = torch.full((pages, 2, Hkv, page, D), float("nan"), dtype=_dtype(f16), device="cuda")
        at = 0
        for b in range(self.B):
            n = max(0, int(lens[b])) + max(0, int(new[b]))
            mine = order[at:at + need[b]]
            at += need[b]
            self.table[b, :need[b]] = mine
            k = rng.standard_normal((n, Hkv, D)) * k_scale
            k[..., 5::32] *= 4
            v = rng.standard_normal((n, Hkv, D)) * 0.5
            self.k.append(_round(k, f16))
            self.v.append(_round(v, f16))
            if n:
                self.put(b, np.arange(n))
        self.q_size = q_size

    def put(self, b, places):
        import torch
        s = torch.from_numpy(self.table[b, places // self.page] * self.page + places % self.page).cuda()
        self.cache[s // self.page, 0, :, s % self.page] = _tensor(self.k[b][places], self.f16)
        self.cache[s // self.page, 1, :, s % self.page] = _tensor(self.v[b][places], self.f16)

    def queries(self, rng, G):
        return _round(rng.standard_normal((self.B, self.T, self.Hkv * G, self.D)) * self.q_size * np.sqrt(128 / self.D), self.f16)

    def attend(self, q, **kw):
        """As views of a fused projection."""
        import torch
        B, T, Hq, D = q.shape
        x = torch.zeros(B, T, Hq + 2 * self.Hkv, D, dtype=_dtype(self.f16), device="cuda")
        x[:, :, :Hq] = _tensor(q, self.f16)
        out = torch.full((B, T, Hq, D), 77.0, dtype=_dtype(self.f16), device="cuda")
        status = torch.full((B,), 77, dtype=torch.int32, device="cuda")
        _fw().switchsd_kv16_attention(x[:, :, :Hq], self.cache, _i32(self.table), _i32(self.lens + 1), _i32(self.new - 2), out, lens_add=-1, new_add=2, status=status, **kw)
        return _numpy(out), status.cpu().numpy()


def _close(got, want, mag, f16):
    e = 2.0 ** -11 if f16 else 2.0 ** -8
    off = np.abs(got - want) - (e * np.abs(want) + (e + 2.0 ** -10) * mag)
    assert np.isfinite(got).all() and off.max() <= 0, (off.max(), np.argwhere(off > 0)[:5])


CASES = [  # lens, new, T, Hkv, G, D, page
    ([0], [1], 1, 1, 1, 128, 16),
    ([0, 1, 15, 16, 17, 31], [1, 1, 1, 0, 1, 1], 1, 2, 4, 128, 16),
    ([127, 128, 129, 126, 255, 256], [1, 1, 1, 1, 0, 1], 1, 1, 8, 64, 32),
    ([2500, 0, 700], [1, 1, 1], 1, 2, 3, 128, 64),
    ([900, 33], [1, 1], 1, 1, 64, 128, 256),
    ([511, 3000], [1, 1], 1, 3, 16, 64, 128),
    ([1000, 5, 129, 0], [17, 1, 9, 3], 17, 2, 4, 128, 32),
    ([300, 2000], [33, 20], 33, 1, 5, 64, 64),
    ([120, 0, 77], [9, 9, 2], 9, 2, 33, 128, 16),
    ([0, 100, 640], [300, 257, 1], 300, 1, 4, 128, 64),
    ([64, 0], [130, 128], 130, 2, 1, 64, 16),
    ([190, 1], [100, 90], 100, 1, 7, 128, 32),
    ([250], [200], 200, 1, 48, 64, 128),
    ([3, 900], [40, 12], 64, 1, 64, 128, 64),
    ([700], [520], 520, 1, 3, 64, 256),
]


@pytest.mark.parametrize("f16", [False, True])
@pytest.mark.parametrize("lens,new,T,Hkv,G,D,page", CASES)
def test_attention(lens, new, T, Hkv, G, D, page, f16):
    rng = np.random.default_rng(T * 1000 + G + D + page)
    s = Setup(rng, lens, new, Hkv, D, page, f16, T)
    q = s.queries(rng, G)
    got, status = s.attend(q)
    want, mag = ref.attention(q, s.k, s.v, lens, new, D ** -0.5)
    _close(got, want, mag, f16)
    assert not status.any()
    for b, n in enumerate(new):
        assert not got[b, n:].any()


@pytest.mark.parametrize("f16", [False, True])
@pytest.mark.parametrize("T,G,D", [(1, 4, 128), (5, 2, 64), (9, 4, 128), (40, 8, 64)])
def test_many_units_a_cta(T, G, D, f16):
    """Long contexts beside short ones: ranges that begin and end inside items, tiles of several rows, and joins."""
    rng = np.random.default_rng(T)
    lens = [20000, 3, 12345, 0, 700, 9000]
    new = [T, T, max(1, T // 2), T, 0, 1]
    s = Setup(rng, lens, new, 2, D, 64, f16, T)
    q = s.queries(rng, G)
    got, status = s.attend(q)
    want, mag = ref.attention(q, s.k, s.v, lens, new, D ** -0.5)
    _close(got, want, mag, f16)
    assert not status.any()


@pytest.mark.parametrize("T,G,D,page", [(17, 4, 128, 32), (1, 8, 128, 16), (130, 2, 128, 64), (40, 4, 64, 256)])
def test_long_ranges(T, G, D, page):
    """Some hundred units a CTA, again and again: tiles of keys and values that arrive in any order.  (The reference by torch,
    in 64 bits.)"""
    import torch
    fw = _fw()
    torch.manual_seed(T)
    B, H, L = 40, 8, 9000 if T < 100 else 3000
    i32 = dict(dtype=torch.int32, device="cuda")
    blocks = -(-(L + T) // page)
    table = torch.randperm(B * blocks, device="cuda").to(torch.int32).view(B, blocks)
    cache = torch.randn(B * blocks, 2, H, page, D, device="cuda").to(torch.bfloat16)
    lens = torch.linspace(L // 3, L, B, device="cuda").to(torch.int32)
    new = (torch.arange(B, **i32) * 7 % T) + 1
    q = torch.randn(B, T, H * G, D, device="cuda").to(torch.bfloat16)
    out, first, status = torch.empty_like(q), torch.empty_like(q), torch.zeros(B, **i32)
    for i in range(60):
        fw.switchsd_kv16_attention(q, cache, table, lens, new, out, status=status)
        if i == 0:
            first.copy_(out)
        assert torch.equal(out, first) and not status.any()
    for b in range(0, B, 3):
        n, m = int(lens[b]), int(new[b])
        kv = cache[table[b].long()].permute(1, 2, 0, 3, 4).reshape(2, H, -1, D)[:, :, :n + m].double()
        x = torch.einsum("thgd,hjd->htgj", q[b, :m].double().view(m, H, G, D), kv[0]) * D ** -0.5
        p = torch.softmax(x.masked_fill((torch.arange(n + m, device="cuda") > n + torch.arange(m, device="cuda")[:, None])[None, :, None], float("-inf")), -1)
        want, mag = (torch.einsum("htgj,hjd->thgd", p, v).reshape(m, H * G, D) for v in (kv[1], kv[1].abs()))
        off = (out[b, :m].double() - want).abs() - (2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -10) * mag)
        assert off.max() <= 0 and not out[b, m:].any()


def test_many_rows():
    """More rows than threads of a CTA, most of them short."""
    rng = np.random.default_rng(5)
    B = 1500
    lens, new = rng.integers(0, 40, B), rng.integers(0, 4, B)
    s = Setup(rng, lens, new, 1, 64, 16, False, 3)
    q = s.queries(rng, 2)
    got, status = s.attend(q)
    want, mag = ref.attention(q, s.k, s.v, lens, new, 0.125)
    _close(got, want, mag, False)
    assert not status.any()


@pytest.mark.parametrize("T,G", [(1, 4), (9, 4), (70, 8)])
def test_rows_and_pages_that_are_left_out(T, G):
    """Bad lengths: zeros and a status; pages outside the pool: not seen, all of a row's too."""
    rng = np.random.default_rng(3)
    lens, new = [300, 40, 200, 90, 10], [T, T, T, T, T]
    s = Setup(rng, lens, new, 2, 128, 32, False, T)
    blocks = s.table.shape[1]
    seen = [np.ones(l + n, bool) for l, n in zip(lens, new)]
    for b, p, bad in ((0, 2, -1), (0, 5, 10**6), (2, 0, s.cache.shape[0])):
        s.table[b, p] = bad
        seen[b][32 * p:32 * p + 32] = False
    s.table[4] = -1
    seen[4][:] = False
    s.lens = np.array([300, -1, 200, blocks * 32 - T + 1, 10])
    q = s.queries(rng, G)
    got, status = s.attend(q)
    want, mag = ref.attention(q, s.k, s.v, lens, [T, 0, T, 0, T], 128 ** -0.5, seen)
    _close(got, want, mag, False)
    assert status.tolist() == [0, 2, 0, 2, 0] and not got[1].any() and not got[3].any() and not got[4].any()
    s.lens, s.new = np.array(lens), np.array([T, T + 1, T, -1, T])
    got, status = s.attend(q)
    _close(got, want, mag, False)
    assert status.tolist() == [0, 2, 0, 2, 0] and not got[1].any() and not got[3].any()


@pytest.mark.parametrize("f16", [False, True])
@pytest.mark.parametrize("T,G", [(1, 2), (6, 4), (70, 4)])
def test_what_a_token_sees_and_what_it_does_not(T, G, f16):
    """NaN and infinities in the keys and values of new tokens reach those from there on: a value's its dimension, a key's
    NaN the whole head; earlier tokens, other heads and other rows as without them."""
    rng = np.random.default_rng(11)
    lens, new = [100, 250], [T, T]
    s = Setup(rng, lens, new, 2, 64, 16, f16, T)
    q = s.queries(rng, G)
    plain, _ = s.attend(q)
    at = T // 2
    s.v[0][100 + at, 0, 5], s.v[0][100 + at, 0, 9], s.v[0][100 + at, 1, 33] = np.nan, np.inf, -np.inf
    s.k[1][250 + at, 1, 3] = np.nan
    s.put(0, np.arange(350)[:100 + T])
    s.put(1, np.arange(250 + T))
    got, status = s.attend(q)
    assert not status.any()
    want = plain.copy()
    want[0, at:, :G, 5], want[0, at:, :G, 9], want[0, at:, G:, 33], want[1, at:, G:] = np.nan, np.inf, -np.inf, np.nan
    assert np.array_equal(got, want, equal_nan=True)


@pytest.mark.parametrize("f16", [False, True])
@pytest.mark.parametrize("T", [1, 9])
def test_scores_of_all_sizes(T, f16):
    """Large scores, one key far above the rest, equal ones, a negative scale, a scale of 0."""
    rng = np.random.default_rng(7)
    lens, new = [1000, 77], [T, T]
    for scale, size in ((1.0, 3.0), (-0.3, 1.0), (0.0, 1.0), (40.0, 0.05)):
        s = Setup(rng, lens, new, 1, 128, 16, f16, T, q_size=size)
        q = s.queries(rng, 4)
        got, status = s.attend(q, scale=scale)
        want, mag = ref.attention(q, s.k, s.v, lens, new, scale)
        # a score's error: 2^-24 of sum |q k| scale for each of 128 additions at most, and it moves the weights by that much
        big = max(np.abs(scale) * (np.abs(q).max() * np.abs(k).sum(-1).max()) for k in s.k)
        e = 2.0 ** -11 if f16 else 2.0 ** -8
        assert (np.abs(got - want) <= e * np.abs(want) + (e + 2.0 ** -10 + 2 * 2.0 ** -17 * big) * mag).all()
        assert not status.any()


def test_values_far_apart_in_size():
    """Weights of many sizes: a few large ones on values of 0, the others on ordinary values."""
    rng = np.random.default_rng(13)
    for T in (1, 9):
        s = Setup(rng, [600], [T], 1, 64, 32, False, T)
        s.k[0][::7] = _round(s.k[0][::7] * 0 + 0.4, False)
        s.v[0][::7] = 0
        q = np.abs(s.queries(rng, 2)) * 0.5
        q = _round(q, False)
        s.put(0, np.arange(600 + T))
        got, _ = s.attend(q)
        want, mag = ref.attention(q, s.k, s.v, [600], [T], 0.125)
        _close(got, want, mag, False)


def test_a_cache_beyond_32_bits():
    """Pages whose elements lie beyond 2^31 and 2^32 of the cache's first."""
    import torch
    rng = np.random.default_rng(17)
    for T in (1, 20):
        s = Setup(rng, [500, 90], [T, T], 1, 128, 256, False, T, first_page=66000, pages=66010)  # 65,536 elements a page
        assert s.cache.numel() > 2**32
        q = s.queries(rng, 4)
        got, status = s.attend(q)
        want, mag = ref.attention(q, s.k, s.v, [500, 90], [T, T], 128 ** -0.5)
        _close(got, want, mag, False)
        slots = _i32(s.table[:, :1] * 256 + 3)
        out = torch.empty(2, 2, 1, 1, 128, dtype=torch.bfloat16, device="cuda")
        _fw().switchsd_kv16_read(s.cache, slots, out[0], out[1])
        assert np.array_equal(_numpy(out[0, :, 0]), np.stack([k[3] for k in s.k])) and np.array_equal(_numpy(out[1, :, 0]), np.stack([v[3] for v in s.v]))


@pytest.mark.parametrize("T,G", [(1, 4), (17, 4), (150, 8)])
def test_the_same_twice_and_in_a_graph(T, G):
    """Twice bit for bit; captured with a workspace of its own and replayed on other lengths, queries and cache contents."""
    import torch
    fw = _fw()
    rng = np.random.default_rng(T)
    lens, new = [2000, 300, 0], [T, T, T]
    s = Setup(rng, lens, new, 2, 128, 64, False, T)
    q = _tensor(s.queries(rng, G), False)
    table, tl, tn = _i32(s.table), _i32(lens), _i32(new)
    a, b = torch.empty_like(q), torch.empty_like(q)
    fw.switchsd_kv16_attention(q, s.cache, table, tl, tn, a)
    fw.switchsd_kv16_attention(q, s.cache, table, tl, tn, b)
    assert torch.equal(a, b)
    w = torch.empty(fw.switchsd_kv16_attention_workspace(128), dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(q)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        fw.switchsd_kv16_attention(q, s.cache, table, tl, tn, out, workspace=w)
        fw.switchsd_kv16_attention(q, s.cache, table, tl, tn, b, workspace=w)
    g.replay()
    assert torch.equal(a, out) and torch.equal(a, b)
    q.copy_(_tensor(s.queries(rng, G), False))
    tl.copy_(_i32([1500, 120, 0]))
    g.replay()
    want = torch.empty_like(q)
    fw.switchsd_kv16_attention(q, s.cache, table, tl, tn, want)
    assert torch.equal(out, want) and not torch.equal(want, a)


def test_a_call_on_another_stream():
    import torch
    fw = _fw()
    rng = np.random.default_rng(1)
    s = Setup(rng, [3000, 100], [9, 9], 2, 128, 64, False, 9)
    q = _tensor(s.queries(rng, 4), False)
    args = (q, s.cache, _i32(s.table), _i32(s.lens), _i32(s.new))
    want, got = torch.empty_like(q), torch.zeros_like(q)
    fw.switchsd_kv16_attention(*args, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    fw.switchsd_kv16_attention(*args, got, stream=side)
    for _ in range(50):
        torch.empty(fw.switchsd_kv16_attention_workspace(128), dtype=torch.uint8, device="cuda").fill_(0xff)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("f16", [False, True])
def test_a_cache_of_16_bits(f16):
    """KVCache(dtype=): a prompt's chunk, drafts of which some are taken back, and single tokens, by the map's pages."""
    import torch
    fw = _fw()
    rng = np.random.default_rng(23)
    B, T, H, G, D = 3, 70, 2, 4, 64
    cache = fw.KVCache(B, T, layers=2, heads=H, dim=D, pages=40, max_len=400, page=16, dtype=_dtype(f16))
    lens = np.zeros(B, np.int64)
    k, v = [[np.zeros((0, H, D))] * B for _ in range(2)]
    for new, keep in (([70, 33, 5], [70, 33, 5]), ([9, 0, 9], [3, 0, 9]), ([1, 1, 1], [1, 1, 1]), ([17, 17, 17], [17, 17, 17])):
        x = _round(rng.standard_normal((B, T, (G + 2) * H, D)), f16)
        y = _tensor(x, f16)
        cache.map(_i32(lens), _i32(new))
        out = torch.empty(B, T, G * H, D, dtype=_dtype(f16), device="cuda")
        for layer in (0, 1):
            cache.append(layer, y[:, :, G * H:G * H + H], y[:, :, G * H + H:])
            cache.attend(layer, y[:, :, :G * H], out)
            kk = [np.concatenate([k[b][:lens[b]], x[b, :new[b], G * H:G * H + H]]) for b in range(B)]
            vv = [np.concatenate([v[b][:lens[b]], x[b, :new[b], G * H + H:]]) for b in range(B)]
            want, mag = ref.attention(x[:, :, :G * H], kk, vv, lens, new, D ** -0.5)
            _close(_numpy(out), want, mag, f16)
        got = cache.read(1, cache.slots)
        assert got[0].dtype == _dtype(f16)
        for b in range(B):
            assert np.array_equal(_numpy(got[0][b, :new[b]]), x[b, :new[b], G * H:G * H + H])
            assert np.array_equal(_numpy(got[1][b, :new[b]]), x[b, :new[b], G * H + H:])
        k, v = kk, vv
        lens = lens + keep
        assert not cache.attend_status.any() and not cache.status.any()
