"""The measured cases of the operators on the target's side of a verification step.

A serving loop around the controller runs, every step, on lengths and drafts that live on the GPU:

- ``map``     ``switchsd_kv_map``: block tables and slot maps of a paged cache from the rows' lengths; a pass is
              two steps of the loop (the lengths of one step, then of the next), so that pages move both ways;
- ``append``  ``switchsd_kv4_append`` of the new tokens' keys and values (views of a fused projection) into the
              4-bit cache, and ``switchsd_kv4_read`` of what the cache then holds for them;
- ``attn``    ``switchsd_kv4_attention`` of the new tokens (one, or a draft and its root) over the 4-bit cache;
- ``logits``  ``switchsd_logits``: penalties for repeated tokens, biases and grammar masks on the target's logits,
              and the greedy token of every position.

The cache of one layer is uint8 [pages, heads, page * (D + D / 64 * 4)]; a (page, head) holds
    key codes    [page][D / 8] words: word c * 2G + 2g + i (G = D / 64, g < G, c < 4, i < 2) has d = 64 g + 16 c + 8 i + 0..7
    value codes  [page / 8][D] words: the word of d has the block's eight tokens
    scales       [page][2 G] f16: the G of the key, then the G of the value
and element j = 2 p + e of a word is its nibble p + 4 e, standing for (nibble - 8) * scale of its group of 64 d.
A group's scale is max(max x / 7, max -x / 8), rounded up to 7 significant bits, in f16.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
NIBBLE_OF = (0, 4, 1, 5, 2, 6, 3, 7)     # element j of a word -> its nibble
ELEMENT_OF = (0, 2, 4, 6, 1, 3, 5, 7)    # nibble n of a word -> its element
SCALE_MAX = 8128.0


# ---------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------
def _map(name, **kw):
    return dict(dict(name=name, op="map", B=64, L=32768, T=17, page=16, turnover=0.0, room=1.1), **kw)


def _append(name, **kw):
    return dict(dict(name=name, op="append", B=64, T=17, Hkv=8, G=4, D=128, page=16, dtype="bf16", ragged=True), **kw)


def _attn(name, **kw):
    return dict(dict(name=name, op="attn", B=64, L=32768, T=1, Hkv=8, G=4, D=128, page=16, dtype="bf16", ragged=True), **kw)


def _logits(name, **kw):
    return dict(dict(name=name, op="logits", B=64, T=17, V=128256, L=32768, dtype="bf16", nbias=0, mask=False, write=False,
                     prompt=False), **kw)


def listed():
    return [
        # one decoding step of the benchmark's batch: a page now and then, latency only
        _map("map_64x32k"),
        # many short chats, a third of which end or begin between the two steps: most pages of the pool move
        _map("map_1024x8k", B=1024, L=8192, T=33, turnover=0.34),
        # the new tokens of one verification step
        _append("append_64x17"),
        # a chunk of prompts of odd lengths
        _append("append_16x2k", B=16, T=2048, page=32, dtype="f16"),
        # one chat sequence's single token: latency
        _attn("attn_1x2k", B=1, L=2048, ragged=False),
        # the benchmark's batch and context, one token a row
        _attn("attn_64x32k"),
        # a few long documents, eight query heads a key head, one token a row
        _attn("attn_4x128k", B=4, L=131071, G=8, page=64, dtype="f16"),
        # verification of drafts of 16 on the 8K contexts
        _attn("verify_64x8k", L=8192, T=17, page=32),
        # verification of drafts of 32, five query heads a key head (d = 5120): the tensor cores' case
        _attn("verify_16x32k", B=16, T=33, G=5, page=64),
        # one sequence's next token, plain sampling penalties: latency
        _logits("logits_1x2k", B=1, T=1, L=2048, dtype="f32", write=True),
        # greedy verification of a batch: penalties and a grammar's masks, only the tokens go on
        _logits("logits_64x17", mask=True, nbias=64),
        # long documents and drafts: the processed logits go on to a sampler
        _logits("logits_16x33", B=16, T=33, V=152064, L=131072, dtype="bf16", write=True, prompt=True, nbias=300),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["map", "append", "attn", "attn", "verify", "logits"])
    if op == "map":
        return dict(_map(None, B=_log(rng, 1, 1024), L=_log(rng, 64, 32768), T=_log(rng, 1, 65), page=rng.choice([16, 32, 64, 128]),
                         turnover=rng.choice([0.0, 0.1, 0.5]), room=rng.choice([1.2, 1.0, 0.9])), name="")
    if op == "append":
        T = _log(rng, 1, 2048)
        return dict(_append(None, B=_log(rng, 1, max(2, 32768 // T // 2)), T=T, Hkv=rng.choice([1, 2, 5, 8]), G=rng.choice([1, 4]), D=rng.choice([64, 128]),
                            page=rng.choice([16, 32, 64, 128]), dtype=rng.choice(["bf16", "f16"]), ragged=rng.choice([True, False])), name="")
    if op in ("attn", "verify"):
        L, Hkv = _log(rng, 32, 100000), rng.choice([1, 2, 4, 8])
        T = 1 if op == "attn" else _log(rng, 2, 33)
        G = rng.choice([1, 2, 3, 4, 6, 8]) if op == "attn" else rng.choice([1, 4, 5])
        most = max(1, min(256, 1_000_000 // L if op == "attn" else 400_000 // L))
        return dict(_attn(None, B=_log(rng, 1, most + 1), L=L, T=T, Hkv=Hkv, G=G, D=rng.choice([64, 128, 128]), page=rng.choice([16, 32, 64, 128]),
                          dtype=rng.choice(["bf16", "f16"]), ragged=rng.choice([True, True, False])), name="")
    V, T = rng.choice([128256, 152064, _log(rng, 1000, 160000)]), _log(rng, 1, 33)
    dtype = rng.choice(["bf16", "f16", "f32"])
    most = max(1, min(256, 60_000_000 // (V * T)))
    return dict(_logits(None, B=_log(rng, 1, most), T=T, V=V, L=_log(rng, 16, 65536), dtype=dtype, nbias=rng.choice([0, 1, 500]), mask=rng.choice([True, False]),
                        write=rng.choice([True, False]), prompt=rng.choice([True, False])), name="")


# ---------------------------------------------------------------------------------------------------------------
# sizes that do not depend on the seed
# ---------------------------------------------------------------------------------------------------------------
def _lens(c):
    """Cached tokens of each row: L, or evenly from L / 4 to L (the seed permutes them)."""
    B, L = c["B"], c["L"]
    if not c.get("ragged", True) or B == 1:
        return np.full(B, L, np.int64)
    return L - (np.arange(B, dtype=np.int64) * (3 * L // 4)) // (B - 1)


def _new(c):
    """New tokens of each row: T, or evenly from 1 to T."""
    B, T = c["B"], c["T"]
    if not c.get("ragged", True) or B == 1:
        return np.full(B, T, np.int64)
    return 1 + (np.arange(B, dtype=np.int64) * (T - 1)) // (B - 1)


def _steps(c, rng):
    """Lengths and new tokens of the two steps of a map case."""
    B, L, T = c["B"], c["L"], c["T"]
    a = rng.permutation(_lens(dict(c, ragged=True)))
    new = rng.permutation(_new(dict(c, ragged=True)))
    b = a + rng.integers(1, T + 1, B)
    off = rng.random(B)
    ends, begins = off < c["turnover"] / 2, (off >= c["turnover"] / 2) & (off < c["turnover"])
    b[ends] = 0
    a[begins] = 0
    return (a, np.where(begins, 0, new)), (b, np.where(ends, 0, new))


def work(case):
    c = case
    if c["op"] == "map":
        # both steps: lengths, new tokens, held in and out, slots; the pages that change hands, list and table
        moved = int(c["turnover"] * c["B"] * c["L"] * 0.6 / c["page"])
        return {"bytes": 2 * (c["B"] * (16 + 4 * c["T"])) + 2 * moved * 16, "flops": 2 * c["B"] * c["T"] * 4}
    if c["op"] == "append":
        n = int(_new(c).sum()) * c["Hkv"]
        full = c["B"] * c["T"] * c["Hkv"] * c["D"] * 2 * 2  # what is read back, zeros included
        return {"bytes": n * (2 * c["D"] * 2 + c["D"] + c["D"] // 64 * 4) + full + n * (c["D"] + c["D"] // 64 * 4), "flops": n * c["D"] * 2 * 4}
    if c["op"] == "attn":
        lens, new = _lens(c), _new(c)
        tokens = int((lens + new).sum()) * c["Hkv"]
        seen = int((lens * new + new * (new + 1) // 2).sum())
        io = 2 * c["B"] * c["T"] * c["Hkv"] * c["G"] * c["D"] * 2
        return {"bytes": tokens * (c["D"] + c["D"] // 64 * 4) + io, "flops": 4 * c["D"] * c["Hkv"] * c["G"] * seen}
    lens, new = _lens(dict(c, ragged=True)), _new(dict(c, ragged=True))
    n = int(new.sum()) * c["V"]
    e = 4 if c["dtype"] == "f32" else 2
    return {"bytes": n * e * (2 if c["write"] else 1) + (n // 8 if c["mask"] else 0) + int(lens.sum()) * 4, "flops": n * 6}


# ---------------------------------------------------------------------------------------------------------------
# the 4-bit format in elementary torch
# ---------------------------------------------------------------------------------------------------------------
def _quantise(x):
    """x [..., D] float32 -> codes int [..., D] (0..15) and scales f16 [..., D / 64]."""
    g = x.reshape(*x.shape[:-1], -1, 64)
    pos, neg = g.amax(-1).clamp_min(0), (-g).amax(-1).clamp_min(0)
    s = torch.maximum(pos / torch.full_like(pos, 7.0), neg * 0.125).clamp_max(SCALE_MAX)
    s = ((s.view(torch.int32) + 0x1FFFF) & ~0x1FFFF).view(torch.float32).half()
    sf = s.float().unsqueeze(-1)
    q = torch.round(g / torch.where(sf > 0, sf, torch.ones_like(sf))).clamp(-8, 7)
    return (q + 8).to(torch.uint8).reshape(x.shape), s


def _dequantise(q, s):
    g = q.reshape(*q.shape[:-1], -1, 64).float() - 8
    return (g * s.float().unsqueeze(-1)).reshape(q.shape)


def _key_words(D, dev):
    """word of the layout -> word of d in order."""
    G = D // 64
    w = torch.arange(D // 8, device=dev)
    c, r = w // (2 * G), w % (2 * G)
    return 8 * (r // 2) + 2 * c + r % 2


def _pack_words(q):
    """codes [..., 8] of a word's elements -> bytes [..., 4]."""
    n = q[..., list(ELEMENT_OF)]
    return n[..., 0::2] | (n[..., 1::2] << 4)


def _unpack_words(b):
    """bytes [..., 4] -> codes [..., 8]."""
    n = torch.stack((b & 15, b >> 4), -1).reshape(*b.shape[:-1], 8)
    return n[..., list(NIBBLE_OF)]


def _pack(kq, ks, vq, vs):
    """codes [N, P, D] and scales [N, P, D / 64] of N (page, head)s -> bytes [N, page bytes]."""
    N, P, D = kq.shape
    kb = _pack_words(kq.reshape(N, P, D // 8, 8)[:, :, _key_words(D, kq.device)]).reshape(N, -1)
    vb = _pack_words(vq.reshape(N, P // 8, 8, D).transpose(2, 3)).reshape(N, -1)
    sb = torch.cat((ks, vs), -1).contiguous().view(torch.uint8).reshape(N, -1)
    return torch.cat((kb, vb, sb), 1)


def _unpack(data, P, D):
    """bytes [..., page bytes] -> values of keys and values, float32 [..., P, D]."""
    lead, n = data.shape[:-1], P * D // 2
    kb, vb, sb = data[..., :n], data[..., n:2 * n], data[..., 2 * n:]
    kw = _unpack_words(kb.reshape(*lead, P, D // 8, 4))
    kq = torch.empty_like(kw)
    kq[..., _key_words(D, data.device), :] = kw
    vq = _unpack_words(vb.reshape(*lead, P // 8, D, 4)).transpose(-1, -2)
    s = sb.contiguous().view(torch.float16).reshape(*lead, P, D // 32)
    return (_dequantise(kq.reshape(*lead, P, D), s[..., :D // 64]),
            _dequantise(vq.reshape(*lead, P, D), s[..., D // 64:]))


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) & 0x7FFFFFFFFFFF)
    return g


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


def _keys_values(g, n, P, D):
    """Keys with a few strong channels and an offset, values about 0.5: [n, P, D] each."""
    k = torch.randn(n, P, D, generator=g, device="cuda")
    k[..., 5::32] *= 4
    k[..., 9::64] += 2
    v = torch.randn(n, P, D, generator=g, device="cuda") * 0.5
    return k, v


def _qkv(c, g):
    """q, k, v as views of a fused projection [B, T, (Hq + 2 Hkv) D]."""
    B, T, H, Hq, D = c["B"], c["T"], c["Hkv"], c["Hkv"] * c["G"], c["D"]
    x = torch.randn(B, T, Hq + 2 * H, D, generator=g, device="cuda")
    x[:, :, :Hq] *= 1.5 / 8 * math.sqrt(128 / D)  # scores that spread by about two
    x[:, :, :Hq] *= 4
    x = x.to(DTYPES[c["dtype"]])
    return x[:, :, :Hq], x[:, :, Hq:Hq + H], x[:, :, Hq + H:]


def _tables(c, rng, lens, new):
    """A block table [B, blocks] with pages in random order and the number of pages of the pool."""
    P = c["page"]
    need = -(-(lens + new) // P)
    pages = int(need.sum()) + 3
    ids = rng.permutation(pages)
    table = np.full((c["B"], int(need.max()) + 1), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += int(n)
    return table, pages


def _slots(table, lens, new, T, P):
    t = np.arange(T)[None]
    p = lens[:, None] + t
    s = np.take_along_axis(table, np.minimum(p // P, table.shape[1] - 1), 1).astype(np.int64) * P + p % P
    return np.where(t < new[:, None], s, -1)


def prepare(case, seed):
    c = case
    rng, g = np.random.default_rng(seed), _gen(seed)
    s = {"c": c}
    if c["op"] == "map":
        (la, na), (lb, nb) = _steps(c, rng)
        P = c["page"]
        blocks = -(-(c["L"] + 2 * c["T"]) // P) + 1
        most = _lens(dict(c, ragged=True)) + c["T"]  # the pool's size goes by the case, not by the seed
        pages = max(4, int((-(-most // P)).sum() * c["room"]))
        i32 = dict(dtype=torch.int32, device="cuda")
        s.update(la=_i32(la), na=_i32(na), lb=_i32(lb), nb=_i32(nb), table=torch.full((c["B"], blocks), -1, **i32), held=torch.zeros(c["B"], **i32),
                 free=_i32(rng.permutation(pages)), count=torch.full((1,), pages, **i32))
        for k in ("slots_a", "slots_b"):
            s[k] = torch.zeros(c["B"], c["T"], **i32)
        for k in ("status_a", "status_b"):
            s[k] = torch.zeros(c["B"], **i32)
        return s
    if c["op"] == "append":
        new = rng.permutation(_new(c))
        lens = rng.integers(0, 4 * c["page"], c["B"])
        table, pages = _tables(c, rng, lens, new)
        _, s["k"], s["v"] = _qkv(c, g)
        s["slots"] = _i32(_slots(table, lens, new, c["T"], c["page"]))
        s["cache"] = torch.zeros(pages, c["Hkv"], c["page"] * (c["D"] + c["D"] // 16), dtype=torch.uint8, device="cuda")
        for k in ("out_k", "out_v"):
            s[k] = torch.empty(c["B"], c["T"], c["Hkv"], c["D"], dtype=torch.float16, device="cuda")
        return s
    if c["op"] == "attn":
        order = rng.permutation(c["B"])
        lens, new = _lens(c)[order], rng.permutation(_new(c))
        if c["ragged"]:  # the sums of work() take the two in the same order
            new = _new(c)[order]
        table, pages = _tables(c, rng, lens, new)
        P, D, H = c["page"], c["D"], c["Hkv"]
        cache = torch.empty(pages * H, P * (D + D // 16), dtype=torch.uint8, device="cuda")
        step = max(1, (1 << 27) // (P * D))
        for at in range(0, pages * H, step):
            n = min(step, pages * H - at)
            k, v = _keys_values(g, n, P, D)
            cache[at:at + n] = _pack(*_quantise(k), *_quantise(v))
        s["q"], _, _ = _qkv(c, g)
        s.update(cache=cache.view(pages, H, -1), table=_i32(table), lens=_i32(lens), new=_i32(new), scale=1 / math.sqrt(D))
        s["out"] = torch.empty(c["B"], c["T"], H * c["G"], D, dtype=DTYPES[c["dtype"]], device="cuda")
        return s
    B, T, V = c["B"], c["T"], c["V"]
    order = rng.permutation(B)
    lens, new = _lens(dict(c, ragged=True))[order], _new(dict(c, ragged=True))[order]
    ld = -(-V // 8) * 8 if c["nbias"] else V  # a projection padded to eight columns, or not
    logits = torch.empty(B, T, ld, dtype=DTYPES[c["dtype"]], device="cuda")
    for b in range(0, B, 8):
        logits[b:b + 8] = torch.randn(min(8, B - b), T, ld, generator=g, device="cuda") * 3
    cap = -(-(int(lens.max()) + T) // 4) * 4
    u = torch.rand(B, cap + T, generator=g, device="cuda", dtype=torch.float64)
    ids = (torch.exp(u * math.log(V)) - 1).to(torch.int32).clamp_(0, V - 1)  # about Zipf: frequent low ids, many rare ones
    s.update(logits=logits[..., :V], ctx=ids[:, :cap].contiguous(), lens=_i32(lens), draft=ids[:, cap:cap + max(1, T - 1)].contiguous(), new=_i32(new))
    r = rng.random((3, B))
    s.update(rep=torch.from_numpy((1 + 0.3 * r[0]).astype(np.float32)).cuda(), freq=torch.from_numpy((0.5 * r[1]).astype(np.float32)).cuda(),
             pres=torch.from_numpy((0.5 * r[2]).astype(np.float32)).cuda())
    s["prompt"] = _i32(lens // 2) if c["prompt"] else None
    s["bias_ids"] = s["bias"] = s["mask"] = s["out"] = None
    if c["nbias"]:
        n = min(c["nbias"], V)
        s["bias_ids"] = _i32(np.stack([rng.permutation(V)[:n] for _ in range(B)]))
        s["bias"] = torch.randn(B, n, generator=g, device="cuda") * 4
    if c["mask"]:
        w = -(-V // 32)
        m = torch.randint(-2**31, 2**31, (B, T, w), generator=g, device="cuda", dtype=torch.int32)
        m &= torch.randint(-2**31, 2**31, (B, T, w), generator=g, device="cuda", dtype=torch.int32)
        m[::7, T // 2] = 0  # a position that the grammar leaves nothing
        s["mask"] = m
    if c["write"]:
        s["out"] = torch.zeros(B, T, V, dtype=DTYPES[c["dtype"]], device="cuda")
    s["argmax"] = torch.empty(B, T, dtype=torch.int32, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------
def _own(s):
    import paper_2609_20186_gb300 as fw

    c = s["c"]
    if c["op"] == "map":
        fw.switchsd_kv_map(s["la"], s["na"], s["table"], s["held"], s["free"], s["count"], s["slots_a"], page=c["page"], status=s["status_a"])
        fw.switchsd_kv_map(s["lb"], s["nb"], s["table"], s["held"], s["free"], s["count"], s["slots_b"], page=c["page"], status=s["status_b"])
        return {k: s[k] for k in ("table", "held", "free", "count", "slots_a", "slots_b", "status_a", "status_b")}
    if c["op"] == "append":
        fw.switchsd_kv4_append(s["k"], s["v"], s["slots"], s["cache"], page=c["page"])
        fw.switchsd_kv4_read(s["cache"], s["slots"], s["out_k"], s["out_v"], page=c["page"])
        return {"k": s["out_k"], "v": s["out_v"]}
    if c["op"] == "attn":
        fw.switchsd_kv4_attention(s["q"], s["cache"], s["table"], s["lens"], s["new"], s["out"], page=c["page"], scale=s["scale"])
        return s["out"]
    fw.switchsd_logits(s["logits"], ctx_tokens=s["ctx"], ctx_lens=s["lens"], draft=s["draft"], new=s["new"], rep=s["rep"], freq=s["freq"], pres=s["pres"],
                       prompt_lens=s["prompt"], bias_ids=s["bias_ids"], bias=s["bias"], mask=s["mask"], out=s["out"], argmax=s["argmax"])
    return {"argmax": s["argmax"], "logits": s["out"]} if c["write"] else s["argmax"]


def _map_plain(lens, new, table, held, free, count, T, P):
    """One step, in place; the slots and the rows' status (1: no room)."""
    B, blocks = table.shape
    j = torch.arange(blocks, device=table.device)[None]
    need = (lens + new + P - 1) // P
    give = (j >= need[:, None]) & (j < held[:, None])
    back = table[give]
    n = int(count) + back.numel()
    free[int(count):n] = back
    table[give] = -1
    want = torch.where(need > held, need - held, torch.zeros_like(need))
    fits = (need <= blocks) & (torch.cumsum(torch.where(need <= blocks, want, torch.zeros_like(want)), 0) <= n)
    fails = (want > 0) & ~fits
    take = (j >= held[:, None]) & (j < need[:, None]) & ~fails[:, None]
    m = int(take.sum())
    table[take] = free[n - m:n].flip(0)
    free[n - m:n] = -1
    held.copy_(torch.where(fails, held, need))
    count.fill_(n - m)
    t = torch.arange(T, device=table.device, dtype=torch.int32)[None]
    p = lens[:, None] + t
    slot = table.gather(1, (p // P).clamp_max(blocks - 1).long()) * P + p % P
    return torch.where((t < new[:, None]) & ~fails[:, None], slot, torch.full_like(slot, -1)), fails.to(torch.int32)


def _attn_plain(s):
    c = s["c"]
    B, T, H, G, D, P = c["B"], c["T"], c["Hkv"], c["G"], c["D"], c["page"]
    k, v = _unpack(s["cache"][s["table"].clamp_min(0).long()], P, D)  # [B, blocks, H, P, D]
    n = k.shape[1] * P
    k = k.transpose(1, 2).reshape(B, H, n, D)
    v = v.transpose(1, 2).reshape(B, H, n, D)
    q = s["q"].float().reshape(B, T, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, T * G, D) * s["scale"]
    x = torch.matmul(q, k.transpose(-1, -2)).view(B, H, T, G, n)
    t = torch.arange(T, device="cuda")[None, :, None]
    j = torch.arange(n, device="cuda")[None, None]
    lens, new = s["lens"][:, None, None], s["new"][:, None, None]
    see = ((j <= lens + t) & (t < new))[:, None, :, None]
    x = torch.where(see, x, torch.full((), -math.inf, device="cuda"))
    m = x.amax(-1, keepdim=True).clamp_min(-1e30)
    e = torch.exp(x - m)
    o = torch.matmul(e.view(B, H, T * G, n), v).view(B, H, T, G, D)
    l = e.sum(-1, keepdim=True)
    o = torch.where(l > 0, o / torch.where(l > 0, l, torch.ones_like(l)), torch.zeros_like(o))
    return o.permute(0, 2, 1, 3, 4).reshape(B, T, H * G, D).to(s["q"].dtype)


def _counts(s):
    """Seen and output counts of every position, before its token: int32 [B, T, V] each."""
    c = s["c"]
    B, T, V = c["B"], c["T"], c["V"]
    ctx, lens = s["ctx"].long(), s["lens"]
    at = torch.arange(ctx.shape[1], device="cuda")[None]
    one = (at < lens[:, None]).to(torch.int32)
    first = s["prompt"][:, None] if s["prompt"] is not None else torch.zeros_like(lens)[:, None]
    seen = torch.zeros(B, V, dtype=torch.int32, device="cuda").scatter_add_(1, ctx, one)
    said = torch.zeros(B, V, dtype=torch.int32, device="cuda").scatter_add_(1, ctx, one * (at >= first))
    step = torch.zeros(B, T, V, dtype=torch.int32, device="cuda")
    if T > 1:
        step[:, 1:].scatter_(2, s["draft"][:, :T - 1, None].long(), 1)
        step = torch.cumsum(step, 1, dtype=torch.int32)
    return seen[:, None] + step, said[:, None] + step


def _logits_plain(s):
    c = s["c"]
    B, T, V = c["B"], c["T"], c["V"]
    x = s["logits"].float()
    seen, said = _counts(s)
    rep, freq, pres = (s[k][:, None, None] for k in ("rep", "freq", "pres"))
    x = torch.where(seen > 0, torch.where(x > 0, x / rep, x * rep), x)
    del seen
    x = torch.where(said > 0, x - freq * said.float() - pres, x)
    del said
    if s["bias"] is not None:
        x = x + torch.zeros(B, V, device="cuda").scatter_(1, s["bias_ids"].long(), s["bias"])[:, None]
    if s["mask"] is not None:
        bit = torch.arange(32, device="cuda", dtype=torch.int32)
        allowed = ((s["mask"][..., None] >> bit) & 1).bool().reshape(B, T, -1)[..., :V]
        x = torch.where(allowed, x, torch.full((), -math.inf, device="cuda"))
    inside = torch.arange(T, device="cuda")[None] < s["new"][:, None]
    top = x.amax(-1, keepdim=True)
    j = torch.arange(V, device="cuda", dtype=torch.int32)
    best = torch.where(x == top, j, torch.full((), V, dtype=torch.int32, device="cuda")).amin(-1)
    best = torch.where(inside & (top[..., 0] > -math.inf), best, torch.full((), -1, dtype=torch.int32, device="cuda"))
    if not c["write"]:
        return best
    return {"argmax": best, "logits": torch.where(inside[..., None], x, torch.zeros((), device="cuda")).to(s["logits"].dtype)}


def run(state):
    s = state
    if own:
        return _own(s)
    c = s["c"]
    if c["op"] == "map":
        s["slots_a"], s["status_a"] = _map_plain(s["la"], s["na"], s["table"], s["held"], s["free"], s["count"], c["T"], c["page"])
        s["slots_b"], s["status_b"] = _map_plain(s["lb"], s["nb"], s["table"], s["held"], s["free"], s["count"], c["T"], c["page"])
        return {k: s[k] for k in ("table", "held", "free", "count", "slots_a", "slots_b", "status_a", "status_b")}
    if c["op"] == "append":
        # into the cache and back: the codes and scales as they stand in it
        inside = (s["slots"] >= 0)[..., None, None]
        k, v = (_dequantise(*_quantise(s[n].float())) for n in ("k", "v"))
        return {"k": torch.where(inside, k, torch.zeros_like(k)).half(), "v": torch.where(inside, v, torch.zeros_like(v)).half()}
    if c["op"] == "attn":
        return _attn_plain(s)
    return _logits_plain(s)


# ---------------------------------------------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def _exact_values(x, inside):
    """What the 4-bit cache stands for, of x [B, T, H, D]: a loop over the rows, in 64 bits."""
    out = np.zeros(x.shape)
    for b in range(x.shape[0]):
        g = x[b].double().reshape(x.shape[1], x.shape[2], -1, 64)
        s = torch.maximum(g.amax(-1).clamp_min(0) / 7, (-g).amax(-1).clamp_min(0) / 8).clamp_max(SCALE_MAX)
        f, e = torch.frexp(s)                                   # s = f 2^e, f in [1/2, 1): 7 bits are 128 f
        s = torch.ldexp(torch.ceil(f * 128) / 128, e.double())
        s = (s * 2.0 ** 24).round() / 2.0 ** 24                 # f16's smallest step; above it 7 bits are exact
        s = s.unsqueeze(-1)
        q = torch.round(g / torch.where(s > 0, s, torch.ones_like(s))).clamp(-8, 7)
        out[b] = (q * s).reshape(x.shape[1:]).cpu().numpy()
    return out * inside[..., None, None]


def _exact_attn(s):
    c = s["c"]
    T, H, G, D, P = c["T"], c["Hkv"], c["G"], c["D"], c["page"]
    out = np.zeros((c["B"], T, H * G, D))
    lens, new, table = (s[k].cpu().numpy() for k in ("lens", "new", "table"))
    for b in range(c["B"]):
        L, n = int(lens[b]), int(new[b])
        pages = torch.from_numpy(table[b, :-(-(L + n) // P)].astype(np.int64)).cuda()
        for h in range(H):
            k, v = (a.reshape(-1, D)[:L + n].double() for a in _unpack(s["cache"][pages, h], P, D))
            q = s["q"][b, :n, h * G:(h + 1) * G].double().reshape(n * G, D) * s["scale"]
            x = (q @ k.T).view(n, G, L + n)
            last = L + torch.arange(n, device="cuda")[:, None, None]
            x = x.masked_fill(torch.arange(L + n, device="cuda") > last, -math.inf)
            p = torch.exp(x - x.amax(-1, keepdim=True))
            o = (p.view(n * G, -1) @ v).view(n, G, D) / p.sum(-1, keepdim=True)
            out[b, :n, h * G:(h + 1) * G] = o.cpu().numpy()
    return out


def _exact_logits(s):
    c = s["c"]
    out = np.zeros((c["B"], c["T"], c["V"]))
    ctx, lens, new, draft = (s[k].cpu().numpy() for k in ("ctx", "lens", "new", "draft"))
    rep, freq, pres = (s[k].cpu().double().numpy() for k in ("rep", "freq", "pres"))
    for b in range(c["B"]):
        first = int(s["prompt"][b]) if s["prompt"] is not None else 0
        seen = np.bincount(ctx[b, :lens[b]], minlength=c["V"])
        said = np.bincount(ctx[b, first:lens[b]], minlength=c["V"])
        for t in range(int(new[b])):
            x = s["logits"][b, t].double().cpu().numpy()
            x = np.where(seen > 0, np.where(x > 0, x / rep[b], x * rep[b]), x) - freq[b] * said - pres[b] * (said > 0)
            if s["bias"] is not None:
                x[s["bias_ids"][b].cpu().numpy()] += s["bias"][b].double().cpu().numpy()
            if s["mask"] is not None:
                bits = np.unpackbits(s["mask"][b, t].cpu().numpy().view(np.uint8), bitorder="little")[:c["V"]]
                x = np.where(bits > 0, x, -np.inf)
            out[b, t] = x
            if t + 1 < c["T"] and t < draft.shape[1]:
                seen[draft[b, t]] += 1
                said[draft[b, t]] += 1
    return {"argmax": None, "logits": out}


def exact(case, seed):
    c = case
    if c["op"] == "map" or (c["op"] == "logits" and not c["write"]):
        return None  # whole numbers
    s = prepare(c, seed)
    if c["op"] == "append":
        inside = (s["slots"] >= 0).cpu().numpy()
        return {"k": _exact_values(s["k"], inside), "v": _exact_values(s["v"], inside)}
    if c["op"] == "attn":
        return _exact_attn(s)
    return _exact_logits(s)
