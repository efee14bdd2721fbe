"""The controller and the target's side of a verification step together, on a small target with random weights.

    python -m paper_2609_20186_gb300.target_demo [--rows 8] [--steps 64] [--no-drafts] [--temperature 0.8] [--cache16]

Every step, with nothing read back by the host: pages and slots for the step's tokens (the context's last one and the
draft; a row that the pool has no pages for sits the step out), their keys and values into the 4-bit cache and their
attention over it, penalties and biases on the logits and the greedy token of every position, then the controller's
verification, append and next draft.  With a temperature the drafts' probabilities and the token that is appended come from
the same logits, and the verification is the sampled one.  The cache may be held in 16 bits.  The target here is attention layers without positions and a head that prefers, by far, the token that follows in a fixed cycle of tokens,
so that its text repeats and copied drafts are accepted; its products are torch's.
"""
from __future__ import annotations

import argparse

import numpy as np
import torch

from . import binding as bd
from .kvcache import KVCache
from .session import Session


class SmallTarget:
    """Attention layers and a head.  Token v is followed by the next of its cycle of `cycle` tokens."""

    def __init__(self, *, vocab: int = 512, dim: int = 256, heads: int = 4, kv_heads: int = 2, layers: int = 2, cycle: int = 24,
                 seed: int = 0, device="cuda"):
        self.vocab, self.dim, self.heads, self.kv_heads, self.layers, self.head_dim = vocab, dim, heads, kv_heads, layers, dim // heads
        g = torch.Generator().manual_seed(seed)

        def weight(rows, cols, scale):
            return (torch.randn(rows, cols, generator=g) * scale).to(device, torch.bfloat16)
        self.embed = weight(vocab, dim, 1.0)
        self.qkv = [weight(dim, (heads + 2 * kv_heads) * self.head_dim, dim ** -0.5) for _ in range(layers)]
        self.out = [weight(dim, dim, 0.1 * dim ** -0.5) for _ in range(layers)]
        v = torch.arange(vocab, device=device)
        last = (v % cycle == cycle - 1) | (v == vocab - 1)
        self.follows = torch.where(last, v - v % cycle, v + 1)
        self.head = torch.zeros_like(self.embed)
        self.head[self.follows] = self.embed

    def hidden(self, tokens: torch.Tensor, cache: KVCache) -> torch.Tensor:
        """The states of tokens [B, T] at the positions that the cache mapped last, their keys and values appended."""
        B, T = tokens.shape
        H, K = self.heads, self.kv_heads
        x = self.embed[tokens.long()]
        mixed = torch.empty(B, T, H, self.head_dim, dtype=x.dtype, device=x.device)
        for layer in range(self.layers):
            qkv = (x @ self.qkv[layer]).view(B, T, H + 2 * K, self.head_dim)
            cache.append(layer, qkv[:, :, H:H + K], qkv[:, :, H + K:])
            cache.attend(layer, qkv[:, :, :H], mixed)
            x = x + mixed.view(B, T, self.dim) @ self.out[layer]
        return x


class Decoder:
    """A batch of sequences between a SmallTarget, a KVCache and a Session."""

    def __init__(self, target: SmallTarget, prompts: np.ndarray, lens: np.ndarray, *, k: int = 8, room: int = 256, page: int = 16,
                 drafts: bool = True, pages: int | None = None, temperature: float | None = None, seed: int = 0,
                 dtype: torch.dtype | None = None):
        """`pages` pages for all rows: enough for every row's whole context when None.  temperature None: the greedy
        verification; else the sampled one, with draws from `seed`.  dtype: the cache's (None: 4 bits)."""
        B = prompts.shape[0]
        self.target, self.k, self.drafts = target, k, drafts
        cap = -(-(prompts.shape[1] + room) // 4) * 4
        ctx = np.zeros((B, cap), np.int32)
        ctx[:, :prompts.shape[1]] = prompts
        probe = np.zeros(target.dim, np.uint16)  # a probe of zeros: with the threshold below, every repetition is copied
        self.sess = Session(ctx, lens, probe, k=k, n_min=2, n_max=4, logit_tau=-1.0, d=target.dim, hidden_rows=k + 1)
        dev = self.sess.ctx.device
        # lengths as the context's: its last token is the first of the step
        self.cache = KVCache(B, k + 1, layers=target.layers, heads=target.kv_heads, dim=target.head_dim, pages=pages or B * -(-cap // page),
                             max_len=cap, page=page, lens_add=-1, new_add=1, device=dev, dtype=dtype)
        f32 = dict(dtype=torch.float32, device=dev)
        self.rep, self.freq, self.pres = torch.full((B,), 1.02, **f32), torch.full((B,), 0.01, **f32), torch.full((B,), 0.1, **f32)
        self.prompt_lens = self.sess.lens.clone()
        self.banned = torch.full((B, 1), target.vocab - 1, dtype=torch.int32, device=dev)  # a token that never comes
        self.bias = torch.full((B, 1), float("-inf"), **f32)
        self.temperature = None
        if temperature is not None:
            self.temperature = torch.full((B,), temperature, **f32)
            self.seeds = torch.arange(B, dtype=torch.int64, device=dev) + (seed << 32)
            self.draws = torch.Generator(device=dev)
            self.draws.manual_seed(seed)
        self._prefill(prompts.shape[1])

    def _prefill(self, longest: int) -> None:
        """All of a context but its last token, k + 1 tokens at a time."""
        T = self.k + 1
        for start in range(0, longest - 1, T):
            cached = torch.clamp(self.sess.lens - 1, max=start)
            self.cache.map(cached + 1, torch.clamp(self.sess.lens - 1 - cached, max=T) - 1)
            if self.cache.status.any():
                raise RuntimeError("the cache has too few pages for the prompts")
            # (places past a row's new tokens get tokens too, which no slot and no result has)
            at = torch.clamp(cached[:, None] + torch.arange(T, device=cached.device), max=self.sess.ctx.shape[1] - 1)
            self.target.hidden(self.sess.ctx.gather(1, at.long()), self.cache)

    def step(self) -> None:
        """One verification step: the target on the last token and the draft, then the controller."""
        s = self.sess
        self.cache.map(s.lens, s.vlen)
        s.vlen.copy_(self.cache.new)  # rows without pages: no logits, nothing appended, and another try in the next step
        tokens = torch.cat([s.ctx.gather(1, (s.lens - 1).long()[:, None]), s.vdraft], 1)
        x = self.target.hidden(tokens, self.cache)
        logits = x @ self.target.head.T
        bd.switchsd_logits(logits, ctx_tokens=s.ctx, ctx_lens=s.lens, draft=s.vdraft, new_lens=s.vlen, new_add=1,
                           rep=self.rep, freq=self.freq, pres=self.pres, prompt_lens=self.prompt_lens, bias_ids=self.banned,
                           bias=self.bias, **(dict(argmax=s.target) if self.temperature is None else dict(out=logits)))
        if self.temperature is None:
            s.verify_step(x)
        else:  # (every draft is a copied one: the drafter's probabilities stay 1)
            s.vu.uniform_(generator=self.draws)
            bd.switchsd_logprobs(logits, tokens=s.vdraft, new_lens=s.vlen, new_add=1, temperature=self.temperature, prob=s.vp)
            bd.switchsd_resample(logits, s.vdraft, s.vlen, s.vp, s.vu, s.target, seeds=self.seeds, ctx_lens=s.lens,
                                 temperature=self.temperature)
            s.verify_sampled_step(x)
        if self.drafts:
            s.vdraft.copy_(s.draft)
            # (a row that sat the step out tries the next one with its one token)
            s.vlen.copy_(torch.where((s.mode == bd.MODE_COPY) & (s.accept >= 0), s.len, 0))
        else:
            s.vlen.zero_()


def prompts_of(rows: int, target: SmallTarget, longest: int = 40, seed: int = 0) -> tuple[np.ndarray, np.ndarray]:
    """Random prompts of 1 to `longest` tokens (without the banned one)."""
    rng = np.random.default_rng(seed)
    return rng.integers(0, target.vocab - 8, (rows, longest)).astype(np.int32), rng.integers(1, longest + 1, rows).astype(np.int32)


def main(argv=None) -> None:
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--rows", type=int, default=8)
    p.add_argument("--steps", type=int, default=64)
    p.add_argument("--no-drafts", action="store_true")
    p.add_argument("--temperature", type=float, default=None)
    p.add_argument("--cache16", action="store_true")
    a = p.parse_args(argv)
    target = SmallTarget()
    prompts, lens = prompts_of(a.rows, target)
    d = Decoder(target, prompts, lens, room=a.steps * 9, drafts=not a.no_drafts, temperature=a.temperature,
                dtype=torch.bfloat16 if a.cache16 else None)
    for _ in range(a.steps):
        d.step()
    new = d.sess.lens.cpu().numpy() - lens
    held, free = int(d.cache.held.sum()), int(d.cache.free_count)
    print(f"{a.steps} steps of {a.rows} rows: {new.sum()} tokens, {new.mean() / a.steps:.2f} a row and step; "
          f"{held} pages held, {free} free of {d.cache.pages}")


if __name__ == "__main__":
    main()
