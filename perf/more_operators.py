"""The measured cases of the operators that a verification step at temperature > 0 needs, with the target's own numbers.

``perf/operators.py`` has the greedy step over the 4-bit cache.  A step at temperature > 0 on a cache in 16 bits runs

- ``append``    ``switchsd_kv16_append`` of the new tokens' keys and values into the paged 16-bit cache, and
                ``switchsd_kv16_read`` of what the cache then holds for them;
- ``attn``      ``switchsd_kv16_attention`` of the new tokens over it: one, a draft and its root, or a prompt's chunk;
- ``logprobs``  ``switchsd_logprobs``: log probabilities of given tokens (drafts, or a prompt's own), the entropy and the
                top alternatives of every position;
- ``resample``  ``switchsd_resample``: the token that the sampled verification appends, drawn for the one position that
                it will append at.

The cache of one layer is [pages, 2, heads, page, D], bf16 or f16: keys, then values.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
GOLDEN, MIX1, MIX2 = 0x9E3779B97F4A7C15, 0xBF58476D1CE4E5B9, 0x94D049BB133111EB  # splitmix64
INF = float("inf")


# ---------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------
def _append(name, **kw):
    return dict(dict(name=name, op="append", B=64, T=17, Hkv=8, G=4, D=128, page=16, dtype="bf16", ragged=True), **kw)


def _attn(name, **kw):
    return dict(dict(name=name, op="attn", B=64, L=32768, T=1, Hkv=8, G=4, D=128, page=16, dtype="bf16", ragged=True), **kw)


def _logprobs(name, **kw):
    return dict(dict(name=name, op="logprobs", B=64, T=17, V=128256, dtype="bf16", top=0, temperature=True, draft=True, mask=False), **kw)


def _resample(name, **kw):
    return dict(dict(name=name, op="resample", B=64, T=17, V=128256, dtype="bf16", q=False, temperature=True), **kw)


def listed():
    return [
        # the new tokens of one verification step
        _append("append_64x17"),
        # a chunk of prompts of odd lengths
        _append("append_16x2k", B=16, T=2048, page=64, dtype="f16"),
        # one chat sequence's single token: latency
        _attn("attn_1x2k", B=1, L=2048, ragged=False),
        # the benchmark's batch and context, one token a row
        _attn("attn_64x32k"),
        # verification of drafts of 16 on the 8K contexts
        _attn("verify_64x8k", L=8192, T=17, page=32),
        # chunks of two long prompts
        _attn("chunk_2x2k", B=2, L=30720, T=2048, page=64, ragged=False),
        # the first chunks of many prompts of odd lengths, heads of 64 dimensions
        _attn("chunk_16x500", B=16, L=1000, T=500, G=8, D=64, page=32, dtype="f16"),
        # one sequence's next token with its alternatives: latency
        _logprobs("logprobs_1x1", B=1, T=1, dtype="f32", top=20, draft=False),
        # the probabilities of a batch's drafts
        _logprobs("logprobs_64x17", mask=True),
        # scoring a prompt's chunks, five alternatives a token
        _logprobs("logprobs_4x2k", B=4, T=2048, top=5, temperature=False, draft=False),
        # the benchmark's batch after copied drafts of 16
        _resample("resample_64x17"),
        # drafts of 32 from a drafter with a distribution of its own
        _resample("resample_16x33", B=16, T=33, V=152064, dtype="f16", q=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attn", "verify", "chunk", "logprobs", "score", "resample"])
    dtype, page, D = rng.choice(["bf16", "f16"]), rng.choice([16, 32, 64, 128, 256]), rng.choice([64, 128, 128])
    if op == "append":
        T = _log(rng, 1, 2048)
        return dict(_append(None, B=_log(rng, 1, max(2, 16384 // T)), T=T, Hkv=rng.choice([1, 2, 5, 8]), G=rng.choice([1, 4]), D=D, page=page,
                            dtype=dtype, ragged=rng.choice([True, False])), name="")
    if op in ("attn", "verify", "chunk"):
        Hkv = rng.choice([1, 2, 4, 8])
        T = 1 if op == "attn" else _log(rng, 2, 65) if op == "verify" else _log(rng, 100, 2048)
        L = _log(rng, 1, 100000) if op == "attn" else _log(rng, 16, 32000) if op == "verify" else _log(rng, 1, 16384)
        G = rng.choice([1, 2, 3, 4, 6, 8]) if op == "attn" else rng.choice([1, 4, 5, 8])
        most = max(1, min(256, 1_000_000 // (L + T), 3_000_000_000 // (T * G * Hkv * (L + T))))
        return dict(_attn(None, B=_log(rng, 1, most + 1) if most > 1 else 1, L=L, T=T, Hkv=Hkv, G=G, D=D, page=page, dtype=dtype,
                          ragged=rng.choice([True, True, False])), name="")
    V, dtype = rng.choice([128256, 152064, _log(rng, 100, 262144)]), rng.choice(["bf16", "f16", "f32"])
    if op == "resample":
        T = _log(rng, 1, 65)
        most = max(1, min(256, 200_000_000 // (V * T)))
        return dict(_resample(None, B=_log(rng, 1, most), T=max(2, T), V=V, dtype=dtype, q=rng.choice([True, False]), temperature=rng.choice([True, False])), name="")
    T = _log(rng, 1, 33) if op == "logprobs" else _log(rng, 64, 2048)
    most = max(1, min(256, 400_000_000 // (V * T)))
    return dict(_logprobs(None, B=_log(rng, 1, most), T=T, V=V, dtype=dtype, top=rng.choice([0, 1, 5, 20, 32]), temperature=rng.choice([True, False]),
                          draft=op == "logprobs" and T > 1, mask=rng.choice([True, False])), name="")


# ---------------------------------------------------------------------------------------------------------------
# sizes that do not depend on the seed
# ---------------------------------------------------------------------------------------------------------------
def _lens(c):
    """Cached tokens of each row: L, or evenly from L / 4 to L (the seed permutes them)."""
    B, L = c["B"], c["L"]
    if not c["ragged"] or B == 1:
        return np.full(B, L, np.int64)
    return L - (np.arange(B, dtype=np.int64) * (3 * L // 4)) // (B - 1)


def _new(c):
    """New tokens (positions) of each row: T, or evenly from 1 to T, beside short and long contexts alike."""
    B, T = c["B"], c["T"]
    if not c.get("ragged", c.get("draft", True)) or B == 1:
        return np.full(B, T, np.int64)
    return 1 + (np.argsort(np.arange(B) * 0.6180339887 % 1) * (T - 1)) // (B - 1)


def work(case):
    c = case
    if c["op"] == "append":
        n = int(_new(c).sum()) * c["Hkv"] * c["D"] * 2 * 2  # bytes of the new tokens' keys and values
        return {"bytes": 3 * n + c["B"] * c["T"] * c["Hkv"] * c["D"] * 4, "flops": 0}  # in, into the cache, out of it, what is read back
    if c["op"] == "attn":
        lens, new = _lens(c), _new(c)
        tokens = int((lens + new).sum()) * c["Hkv"]
        seen = int((lens * new + new * (new + 1) // 2).sum())
        io = int(new.sum()) * 2 * c["Hkv"] * c["G"] * c["D"] * 2
        return {"bytes": tokens * c["D"] * 4 + io, "flops": 4 * c["D"] * c["Hkv"] * c["G"] * seen}
    e = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "logprobs":
        n = int(_new(c).sum())
        return {"bytes": n * (c["V"] * e + 12 + 8 * c["top"]), "flops": n * c["V"] * 5}
    return {"bytes": c["B"] * c["V"] * e * (2 if c["q"] else 1), "flops": c["B"] * c["V"] * 20}


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) & 0x7FFFFFFFFFFF)
    return g


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


def _f32(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda()


def _qkv(c, g):
    """q, k, v as views of a fused projection [B, T, (Hq + 2 Hkv) D]: keys with a few strong channels and an offset, scores
    that spread by about two, values about 0.5."""
    B, T, H, Hq, D = c["B"], c["T"], c["Hkv"], c["Hkv"] * c["G"], c["D"]
    x = torch.randn(B, T, Hq + 2 * H, D, generator=g, device="cuda")
    x[:, :, :Hq] *= 0.75 * math.sqrt(128 / D)
    _like_keys(x[:, :, Hq:Hq + H])
    x[:, :, Hq + H:] *= 0.5
    x = x.to(DTYPES[c["dtype"]])
    return x[:, :, :Hq], x[:, :, Hq:Hq + H], x[:, :, Hq + H:]


def _like_keys(k):
    k[..., 5::32] *= 4
    k[..., 9::64] += 2


def _tables(c, rng, lens, new, pages=None):
    """A block table [B, blocks] with pages in random order and the number of pages of the pool (a few more than needed)."""
    need = -(-(lens + new) // c["page"])
    pages = pages or int(need.sum()) + 3
    table = np.full((c["B"], int(need.max()) + 1), -1, np.int32)
    table[np.arange(table.shape[1])[None] < need[:, None]] = rng.permutation(pages)[:int(need.sum())]
    return table, pages


def _slots(table, lens, new, T, P):
    t = np.arange(T)[None]
    p = lens[:, None] + t
    s = np.take_along_axis(table, np.minimum(p // P, table.shape[1] - 1), 1).astype(np.int64) * P + p % P
    return np.where(t < new[:, None], s, -1)


def _some_logits(c, g, n):
    """Logits [B, n, V] of a sharpened distribution: a wide bulk and a few tokens far above it at each position."""
    B, V = c["B"], c["V"]
    x = torch.randn(B, n, V, generator=g, device="cuda") * 2
    few = torch.randint(0, V, (B, n, 8), generator=g, device="cuda")
    return x.scatter_add_(2, few, torch.rand(B, n, 8, generator=g, device="cuda") * 14), few


def prepare(case, seed):
    c = case
    rng, g = np.random.default_rng(seed), _gen(seed)
    s = {"c": c}
    B, T = c["B"], c["T"]
    if c["op"] == "append":
        new = rng.permutation(_new(c))
        lens = rng.integers(0, 4 * c["page"], B)
        table, pages = _tables(c, rng, lens, new, B * (4 + -(-T // c["page"])))
        _, s["k"], s["v"] = _qkv(c, g)
        dtype = DTYPES[c["dtype"]]
        s["slots"] = _i32(_slots(table, lens, new, T, c["page"]))
        s["cache"] = torch.randn(pages, 2, c["Hkv"], c["page"], c["D"], generator=g, device="cuda").to(dtype)
        s["out_k"] = torch.zeros(B, T, c["Hkv"], c["D"], dtype=dtype, device="cuda")
        s["out_v"] = torch.zeros_like(s["out_k"])
        return s
    if c["op"] == "attn":
        order = rng.permutation(B)
        lens, new = _lens(c)[order], _new(c)[order]
        table, pages = _tables(c, rng, lens, new)
        s["q"], _, _ = _qkv(c, g)
        dtype = DTYPES[c["dtype"]]
        s["cache"] = torch.empty(pages, 2, c["Hkv"], c["page"], c["D"], dtype=dtype, device="cuda")
        for half, like in ((0, _like_keys), (1, lambda v: v.mul_(0.5))):
            x = torch.randn(pages, c["Hkv"], c["page"], c["D"], generator=g, device="cuda")
            like(x)
            s["cache"][:, half] = x
        s.update(table=_i32(table), lens=_i32(lens), new=_i32(new), out=torch.zeros(B, T, c["Hkv"] * c["G"], c["D"], dtype=dtype, device="cuda"))
        if own:
            s["workspace"] = _workspace(c)
        return s
    dtype = DTYPES[c["dtype"]]
    x, few = _some_logits(c, g, T)
    if c.get("mask"):  # a grammar that leaves every other row a third of the vocabulary
        x[::2].masked_fill_(torch.rand(c["V"], generator=g, device="cuda") < 0.67, -INF)
    s["logits"] = x.to(dtype)
    del x
    s["temp"] = _f32(np.where(rng.random(B) < 0.1, 0.0, rng.uniform(0.5, 1.3, B))) if c["temperature"] else None
    if c["op"] == "logprobs":
        k = T - 1 if c["draft"] else T
        likely = torch.rand(B, T, generator=g, device="cuda") < 0.7
        tokens = torch.where(likely, few[..., 0], torch.randint(0, c["V"], (B, T), generator=g, device="cuda"))
        s["tokens"] = tokens[:, :k].to(torch.int32).contiguous()
        s["vlen"] = _i32(rng.permutation(_new(c)) - 1)  # a draft of vlen tokens has vlen + 1 positions
        f32 = dict(dtype=torch.float32, device="cuda")
        s.update(logprob=torch.zeros(B, k, **f32), prob=torch.zeros(B, k, **f32), entropy=torch.zeros(B, T, **f32), lse=torch.zeros(B, T, **f32))
        if c["top"]:
            s.update(top_ids=torch.zeros(B, T, c["top"], dtype=torch.int32, device="cuda"), top_logprobs=torch.zeros(B, T, c["top"], **f32))
        return s
    k = T - 1
    s["vlen"] = _i32(rng.permutation(_new(c)) - 1)
    s["draft"] = few[:, :k, 0].to(torch.int32).contiguous()
    s["seeds"] = torch.from_numpy(rng.integers(-2**63, 2**63 - 1, B, dtype=np.int64)).cuda()
    s["lens"] = _i32(rng.integers(1, 32768, B))
    s["u"] = torch.rand(B, k, generator=g, device="cuda")
    s["lse"], s["p"] = _lse_and_prob(s["logits"], s["temp"], s["draft"])
    if c["q"]:
        x = torch.randn(B, k, c["V"], generator=g, device="cuda").mul_(0.7).add_(s["logits"][:, :k])
        s["q_logits"] = x.to(dtype)
        s["q_lse"], s["q"] = _lse_and_prob(s["q_logits"], s["temp"], s["draft"])
        s["mode"] = _i32(rng.integers(0, 3, B))  # copied drafts among the drafter's
        s["q"][s["mode"] == 1] = 1.0
    s["out"] = torch.zeros(B, T, dtype=torch.int32, device="cuda")
    return s


def _workspace(c):
    from paper_2609_20186_gb300 import switchsd_kv16_attention_workspace
    return torch.empty(switchsd_kv16_attention_workspace(c["D"]), dtype=torch.uint8, device="cuda")


def _lse_and_prob(logits, temp, draft):
    """ln sum exp(l / temp) of each position, and the draft's probabilities."""
    x = logits.float()
    top = x.amax(2, keepdim=True)
    greedy = temp == 0 if temp is not None else torch.zeros(x.shape[0], dtype=torch.bool, device="cuda")
    t = (torch.where(greedy, torch.ones_like(temp), temp) if temp is not None else torch.ones(x.shape[0], device="cuda"))[:, None]
    first = x.argmax(2)[:, :draft.shape[1]]
    lse = torch.exp((x - top) / t[..., None]).sum(2).log() + top[..., 0] / t
    l = torch.gather(x[:, :draft.shape[1]], 2, draft.long()[..., None])[..., 0]
    return lse, torch.where(greedy[:, None], (first == draft).float(), torch.exp(l / t - lse[:, :draft.shape[1]]))


# ---------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------
def run(s):
    if own:
        return _own(s)
    return {"append": _plain_append, "attn": _plain_attn, "logprobs": _plain_logprobs, "resample": _plain_resample}[s["c"]["op"]](s)


def _own(s):
    import paper_2609_20186_gb300 as sd
    c = s["c"]
    if c["op"] == "append":
        sd.switchsd_kv16_append(s["k"], s["v"], s["slots"], s["cache"])
        sd.switchsd_kv16_read(s["cache"], s["slots"], s["out_k"], s["out_v"])
        return s["cache"], s["out_k"], s["out_v"]
    if c["op"] == "attn":
        sd.switchsd_kv16_attention(s["q"], s["cache"], s["table"], s["lens"], s["new"], s["out"], workspace=s["workspace"])
        return s["out"]
    if c["op"] == "logprobs":
        sd.switchsd_logprobs(s["logits"], tokens=s["tokens"], new_lens=s["vlen"], new_add=1, temperature=s["temp"], logprob=s["logprob"], prob=s["prob"],
                             entropy=s["entropy"], lse=s["lse"], top_ids=s.get("top_ids"), top_logprobs=s.get("top_logprobs"))
        return {k: s[k] for k in ("logprob", "prob", "entropy", "lse", "top_ids", "top_logprobs") if k in s}
    sd.switchsd_resample(s["logits"], s["draft"], s["vlen"], s["p"], s["u"], s["out"], seeds=s["seeds"], ctx_lens=s["lens"], temperature=s["temp"],
                         lse=s["lse"], q_draft=s.get("q"), q_logits=s.get("q_logits"), q_lse=s.get("q_lse"), mode=s.get("mode"))
    return s["out"]


def _plain_append(s):
    cache, slots, P = s["cache"], s["slots"].long(), s["c"]["page"]
    here = slots >= 0
    at = slots[here]
    cache[at // P, 0, :, at % P] = s["k"][here]
    cache[at // P, 1, :, at % P] = s["v"][here]
    at, zero = slots.clamp_min(0), torch.zeros((), dtype=cache.dtype, device="cuda")
    k, v = cache[at // P, 0, :, at % P], cache[at // P, 1, :, at % P]
    return cache, torch.where(here[..., None, None], k, zero), torch.where(here[..., None, None], v, zero)


def _plain_attn(s):
    c, q, table = s["c"], s["q"], s["table"].long()
    B, T, Hq, D = q.shape
    H, G, n = c["Hkv"], c["G"], table.shape[1] * c["page"]
    kv = s["cache"][table.clamp_min(0)]  # [B, blocks, 2, H, page, D]
    k, v = (kv[:, :, half].permute(0, 2, 1, 3, 4).reshape(B, H, n, D).float() for half in (0, 1))
    del kv
    q = q.float().reshape(B, T, H, G, D).permute(0, 2, 3, 1, 4).reshape(B, H, G * T, D)
    x = torch.matmul(q * D ** -0.5, k.transpose(2, 3)).reshape(B, H, G, T, n)
    t, j = torch.arange(T, device="cuda"), torch.arange(n, device="cuda")
    last = torch.where(t[None] < s["new"][:, None], s["lens"][:, None] + t[None], -1)  # of the positions that token t sees
    hidden = (j > last[..., None]) | (table < 0).repeat_interleave(c["page"], 1)[:, None]
    x.masked_fill_(hidden[:, None, None], -INF)
    top = x.amax(-1, keepdim=True)
    x.sub_(torch.where(top == -INF, torch.zeros_like(top), top)).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.reshape(B, H, G * T, n), v).reshape(B, H, G, T, D) / torch.where(total == 0, torch.ones_like(total), total)
    return o.permute(0, 3, 1, 2, 4).reshape(B, T, Hq, D).to(s["q"].dtype)


def _order(x):
    """Whole numbers in the order of the float32 numbers x, with -0 = 0 (NaN is not among them)."""
    i = (x + 0.0).view(torch.int32)
    return torch.where(i < 0, i ^ 0x7FFFFFFF, i)


def _plain_logprobs(s):
    c, x = s["c"], s["logits"].float()
    B, T, V = x.shape
    k = s["tokens"].shape[1]
    temp = s["temp"] if s["temp"] is not None else torch.ones(B, device="cuda")
    greedy = (temp == 0)[:, None].expand(B, T)
    t = torch.where(temp == 0, torch.ones_like(temp), temp)[:, None]
    here = torch.arange(T, device="cuda")[None] < s["vlen"][:, None] + 1
    top = x.amax(2)
    first = x.argmax(2) if s["temp"] is not None else None
    y = (x - top[..., None]) / t[..., None]
    w = torch.exp(y)
    total = w.sum(2)
    w.mul_(y.clamp_min_(-1e30))
    log = total.log()
    entropy = torch.where(greedy, torch.zeros_like(log), log - w.sum(2) / total)
    lse = torch.where(greedy, top, top / t + log)
    del w, y

    def logprob_of(ids):  # [B, n <= T, m]
        n = ids.shape[1]
        lp = (torch.gather(x[:, :n], 2, ids) - top[:, :n, None]) / t[..., None] - log[:, :n, None]
        if first is not None:
            one = torch.where(ids == first[:, :n, None], torch.zeros_like(lp), torch.full_like(lp, -INF))
            lp = torch.where(greedy[:, :n, None], one, lp)
        return torch.where(here[:, :n, None], lp, torch.full_like(lp, -INF))

    lp = logprob_of(s["tokens"].long()[..., None])[..., 0]
    out = {"logprob": lp, "prob": torch.exp(lp), "entropy": torch.where(here, entropy, torch.zeros_like(entropy)), "lse": torch.where(here, lse, torch.full_like(lse, -INF))}
    if c["top"]:
        key = (_order(x).long() << 32) | (0xFFFFFFFF - torch.arange(V, device="cuda"))  # the lowest index of equal ones first
        ids = 0xFFFFFFFF - (key.topk(c["top"], 2).values & 0xFFFFFFFF)
        gone = ~here[..., None] | (torch.gather(x, 2, ids) == -INF)
        out["top_ids"] = torch.where(gone, torch.full_like(ids, -1), ids).to(torch.int32)
        out["top_logprobs"] = torch.where(gone, torch.full(ids.shape, -INF, device="cuda"), logprob_of(ids))
    return out


def _mix(z):
    """splitmix64's output function on int64 numbers."""
    z = (z ^ ((z >> 30) & ((1 << 34) - 1))) * (MIX1 - 2**64)
    z = (z ^ ((z >> 27) & ((1 << 37) - 1))) * (MIX2 - 2**64)
    return z ^ ((z >> 31) & ((1 << 33) - 1))


def _plain_resample(s):
    c = s["c"]
    B, T, V = s["logits"].shape
    k, rows, dev = T - 1, torch.arange(B, device="cuda"), "cuda"
    i = torch.arange(k, device=dev)[None]
    q = s["q"] if c["q"] else torch.ones_like(s["p"])
    rejected = (s["u"] * q >= s["p"]) & (i < s["vlen"][:, None])
    a = torch.where(rejected, i, s["vlen"][:, None]).amin(1).long()
    # E = -ln(1 - x), x = (r + 1/2) / 2^32, in 64 bits: what decides is how far the two best are apart
    key = _mix(s["seeds"] + (s["lens"].long() + a + 1) * (GOLDEN - 2**64))
    r = _mix(key[:, None] + (torch.arange((V + 1) // 2, device=dev)[None] + 1) * (GOLDEN - 2**64))
    r = torch.stack((r & 0xFFFFFFFF, (r >> 32) & 0xFFFFFFFF), 2).reshape(B, -1)[:, :V]
    noise = torch.log(-torch.log1p(-(r.double() + 0.5) / 2**32))
    temp = s["temp"].double() if s["temp"] is not None else torch.ones(B, dtype=torch.float64, device=dev)
    greedy, t = temp == 0, torch.where(temp == 0, torch.ones_like(temp), temp)
    l = s["logits"][rows, a].double()
    y = l / t[:, None] - s["lse"][rows, a].double()[:, None]
    drafted = a < s["vlen"]
    last = a.clamp_max(k - 1)
    w = y.clone()
    copied = torch.ones_like(drafted)
    if c["q"]:
        yq = s["q_logits"][rows, last].double() / t[:, None] - s["q_lse"][rows, last].double()[:, None]
        copied = s["mode"] == 1
        w = torch.where((drafted & ~copied)[:, None], torch.log((y.exp() - yq.exp()).clamp_min(0)), w)
    name = torch.arange(V, device=dev)[None]
    w.masked_fill_((drafted & copied)[:, None] & (name == s["draft"][rows, last][:, None]), -INF)
    w = torch.where((w.amax(1) == -INF)[:, None], y, w)
    best = torch.where(greedy[:, None], l, w - noise)
    token = torch.where(best.amax(1) == -INF, torch.full_like(a, -1), best.argmax(1))
    return torch.where(torch.arange(T, device=dev)[None] == a[:, None], token[:, None], -1).to(torch.int32)


# ---------------------------------------------------------------------------------------------------------------
# the same from the definitions, in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    c = case
    if c["op"] == "append":
        return _exact_append(s)
    if c["op"] == "attn":
        return _exact_attn(s) if work(c)["flops"] < 8e12 else None
    if c["op"] == "logprobs":
        return _exact_logprobs(s)
    return None  # whole numbers only


def _exact_append(s):
    c = s["c"]
    B, T, H, D = s["k"].shape
    flat = s["cache"].double().permute(0, 3, 1, 2, 4).reshape(-1, 2, H, D)  # by slots
    kv = torch.stack((s["k"], s["v"]), 2).double().reshape(B * T, 2, H, D)
    slots = s["slots"].reshape(-1).long()
    got = torch.zeros_like(kv)
    for n in (slots >= 0).nonzero()[:, 0].split(4096):
        flat[slots[n]] = kv[n]
        got[n] = kv[n]
    cache = flat.reshape(-1, c["page"], 2, H, D).permute(0, 2, 3, 1, 4).contiguous()
    return cache, got[:, 0].reshape(B, T, H, D), got[:, 1].reshape(B, T, H, D)


def _exact_attn(s):
    c = s["c"]
    B, T, Hq, D = s["q"].shape
    out = torch.zeros(B, T, Hq, D, dtype=torch.float64, device="cuda")
    lens, new, table = s["lens"].tolist(), s["new"].tolist(), s["table"].long()
    for b in range(B):
        n, total = new[b], lens[b] + new[b]
        kv = s["cache"].index_select(0, table[b, :-(-total // c["page"])])
        for h in range(c["Hkv"]):
            k, v = (kv[:, half, h].reshape(-1, D)[:total].double() for half in (0, 1))
            for t0 in range(0, n, 512):
                t1 = min(n, t0 + 512)
                q = s["q"][b, t0:t1, h * c["G"]:(h + 1) * c["G"]].double()
                x = torch.einsum("tgd,jd->tgj", q, k) / math.sqrt(D)
                seen = torch.ones(t1 - t0, total, dtype=torch.bool, device="cuda").tril(lens[b] + t0)
                p = torch.softmax(x.masked_fill(~seen[:, None], -INF), -1)
                out[b, t0:t1, h * c["G"]:(h + 1) * c["G"]] = torch.einsum("tgj,jd->tgd", p, v)
    return out


def _exact_logprobs(s):
    c = s["c"]
    B, T, V = s["logits"].shape
    k = s["tokens"].shape[1]
    out = {"logprob": torch.full((B, k), -INF, dtype=torch.float64, device="cuda"), "entropy": torch.zeros(B, T, dtype=torch.float64, device="cuda"),
           "lse": torch.full((B, T), -INF, dtype=torch.float64, device="cuda"), "top_ids": None}
    if c["top"]:
        out["top_logprobs"] = torch.full((B, T, c["top"]), -INF, dtype=torch.float64, device="cuda")
    temps = s["temp"].double().tolist() if s["temp"] is not None else [1.0] * B
    for b, n in enumerate((s["vlen"] + 1).tolist()):
        for t0 in range(0, n, 256):
            t1 = min(n, t0 + 256)
            raw = s["logits"][b, t0:t1].double()
            if temps[b] == 0:
                lp = torch.full_like(raw, -INF).scatter_(1, raw.argmax(1, keepdim=True), 0.0)
                out["lse"][b, t0:t1] = raw.amax(1)
            else:
                lp = torch.log_softmax(raw / temps[b], 1)
                out["lse"][b, t0:t1] = torch.logsumexp(raw / temps[b], 1)
                out["entropy"][b, t0:t1] = -torch.special.xlogy(lp.exp(), lp.exp()).sum(1)
            m = min(t1, k)
            if m > t0:
                out["logprob"][b, t0:m] = lp[:m - t0].gather(1, s["tokens"][b, t0:m].long()[:, None])[:, 0]
            if c["top"]:  # (of equal ones any: their log probabilities are equal, and a greedy row's first one's is 0)
                best = lp.topk(c["top"], 1).values if temps[b] == 0 else raw.topk(c["top"], 1).indices
                out["top_logprobs"][b, t0:t1] = best if temps[b] == 0 else lp.gather(1, best)
    out["prob"] = out["logprob"].exp()
    return out
