"""Plain implementations, in 64 bits, of the operators of include/switchsd_target.h (numpy, loops, no shared code)."""
import numpy as np


def bf16_round(x):
    """float64 -> the nearest bf16 (ties to even), as float64."""
    b = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    return ((b + 0x7fff + ((b >> 16) & 1)) & 0xffff0000).astype(np.uint32).view(np.float32).astype(np.float64)


# --- block tables and slot maps -----------------------------------------------------------------------------------
class MapState:
    def __init__(self, B, blocks, free):
        self.rows = [[] for _ in range(B)]
        self.free, self.blocks, self.pages = list(free), blocks, len(free)

    def step(self, lens, new, T, page):
        """Returns slots [B, T] and status [B]."""
        B = len(self.rows)
        status, need = [0] * B, [None] * B
        for b in range(B):
            if lens[b] < 0 or not 0 <= new[b] <= T:
                status[b] = 2
                continue
            n = -(-(lens[b] + new[b]) // page)
            if n > self.blocks:
                status[b] = 1
                continue
            need[b] = n
        for b in range(B):
            if need[b] is not None and need[b] < len(self.rows[b]):
                self.free += self.rows[b][need[b]:]
                del self.rows[b][need[b]:]
        room, asked = len(self.free), 0
        for b in range(B):
            want = 0 if need[b] is None else max(0, need[b] - len(self.rows[b]))
            if want == 0:
                continue
            asked += want
            if asked > room:
                status[b], need[b] = 1, None
                continue
            for _ in range(want):
                self.rows[b].append(self.free.pop())
        slots = -np.ones((B, T), np.int32)
        for b in range(B):
            if need[b] is None:
                continue
            for t in range(new[b]):
                p = lens[b] + t
                slots[b, t] = self.rows[b][p // page] * page + p % page
        return slots, np.array(status, np.int32)

    def arrays(self):
        table = -np.ones((len(self.rows), self.blocks), np.int32)
        for b, r in enumerate(self.rows):
            table[b, :len(r)] = r
        free = -np.ones(self.pages, np.int32)
        free[:len(self.free)] = self.free
        return table, np.array([len(r) for r in self.rows], np.int32), free, len(self.free)


# --- the 4-bit format ---------------------------------------------------------------------------------------------
def quantise(x):
    """x [..., D] float64 -> (codes int [..., D], scales float64 [..., D / 64])."""
    x = np.asarray(x, np.float64)
    g = x.reshape(*x.shape[:-1], x.shape[-1] // 64, 64)
    s = np.maximum(np.maximum(g.max(-1), 0) / 7, np.maximum((-g).max(-1), 0) / 8)
    with np.errstate(invalid="ignore"):
        s = np.minimum(s, 8128.0)
        m, e = np.frexp(s)
        s = np.ldexp(np.ceil(m * 128) / 128, e)
        s = np.where(s < 2.0 ** -14, np.round(s * 2.0 ** 24) / 2.0 ** 24, s)
        sx = s[..., None]
        q = np.where(sx > 0, np.clip(np.rint(g / np.where(sx > 0, sx, 1)), -8, 7), 0)
    return (np.nan_to_num(q).astype(np.int64) + 8).reshape(x.shape), s


def dequantise(codes, s):
    g = codes.reshape(*codes.shape[:-1], codes.shape[-1] // 64, 64).astype(np.float64) - 8
    return (g * s[..., None]).reshape(codes.shape)


def decode_slot(cache, page, D, slot, h):
    """Key and value codes and scales of one slot, from the cache's bytes as the header describes them."""
    G = D // 64
    raw = cache[slot // page, h]
    i = slot % page
    kw = raw[:page * D // 2].view(np.uint32).reshape(page, D // 8)[i]
    vw = raw[page * D // 2:page * D].view(np.uint32).reshape(page // 8, D)[i // 8]
    sc = raw[page * D:].view(np.float16).reshape(page, 2 * G)[i].astype(np.float64)
    nib = [(j >> 1) + 4 * (j & 1) for j in range(8)]
    k, v = np.zeros(D, np.int64), np.zeros(D, np.int64)
    for c in range(4):
        for g in range(G):
            for u in range(2):
                w = int(kw[c * 2 * G + 2 * g + u])
                for j in range(8):
                    k[64 * g + 16 * c + 8 * u + j] = (w >> (4 * nib[j])) & 15
    for d in range(D):
        v[d] = (int(vw[d]) >> (4 * nib[i % 8])) & 15
    return k, v, sc[:G], sc[G:]


# --- attention ----------------------------------------------------------------------------------------------------
def attention(q, k, v, lens, new, scale, seen=None):
    """q [B, T, Hq, D]; k, v lists of [n_b, Hkv, D] (the row's tokens in order of position); seen: lists of bool [n_b].
    Returns out and sum_j p_j |v_j| [B, T, Hq, D]."""
    B, T, Hq, D = q.shape
    out, mag = np.zeros(q.shape), np.zeros(q.shape)
    for b in range(B):
        Hkv = k[b].shape[1] if len(k[b]) else 1
        for t in range(new[b]):
            n = lens[b] + t + 1
            for h in range(Hq):
                kk, vv = k[b][:n, h // (Hq // Hkv)], v[b][:n, h // (Hq // Hkv)]
                if seen is not None:
                    kk, vv = kk[seen[b][:n]], vv[seen[b][:n]]
                if len(kk) == 0:
                    continue
                x = scale * (kk @ q[b, t, h])
                p = np.exp(x - x.max())
                p /= p.sum()
                out[b, t, h] = p @ vv
                mag[b, t, h] = p @ np.abs(vv)
    return out, mag


# --- logits -------------------------------------------------------------------------------------------------------
def logits(x, ctx, lens, draft, new, rep, freq, pres, prompt, bias_ids, bias, mask, dtype=np.float64):
    """x [B, T, V]; returns the processed logits in `dtype` (float32: every operation rounded, as the kernel's) and the
    greedy tokens."""
    B, T, V = x.shape
    out, best = np.zeros((B, T, V), dtype), -np.ones((B, T), np.int32)
    for b in range(B):
        c = ctx[b, :lens[b]]
        ok = (c >= 0) & (c < V)
        seen = np.bincount(c[ok], minlength=V)
        at = np.arange(len(c)) >= (prompt[b] if prompt is not None else 0)
        said = np.bincount(c[ok & at], minlength=V)
        for t in range(new[b]):
            y = x[b, t].astype(dtype)
            r, f, p = (dtype(a[b]) for a in (rep, freq, pres))
            y = np.where(seen > 0, np.where(y > 0, y / r, y * r), y)
            y = np.where(said > 0, (y - f * said.astype(dtype)) - p, y)
            if bias_ids is not None:
                last = {}
                for i, v in enumerate(bias_ids[b]):
                    if 0 <= v < V:
                        last[int(v)] = i
                for v, i in last.items():
                    y[v] = y[v] + dtype(bias[b, i])
            if mask is not None:
                y = np.where(np.unpackbits(mask[b, t].view(np.uint8), bitorder="little")[:V] > 0, y, dtype(-np.inf))
            out[b, t] = y
            z = np.where(np.isnan(y), -np.inf, y)
            if z.max() > -np.inf:
                best[b, t] = int(np.argmax(z))
            if draft is not None and t + 1 < new[b] and 0 <= draft[b, t] < V:
                seen[draft[b, t]] += 1
                said[draft[b, t]] += 1
    return out, best
