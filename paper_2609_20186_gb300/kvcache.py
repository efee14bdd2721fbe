"""A paged 4-bit key/value cache of a batch of sequences on one CUDA device.

A ``KVCache`` owns the pages of every layer, the pool's free list and the rows' block tables, and runs the target's side
of a verification step on device-resident lengths:

    cache.map(lens, new)            pages and slots for the step's new tokens (switchsd_kv_map)
    cache.append(layer, k, v)       their keys and values (switchsd_kv4_append)
    cache.attend(layer, q, out)     their attention over the cache (switchsd_kv4_attention)

With a ``Session`` whose draft is in ``sess.vdraft`` / ``sess.vlen``, ``lens`` is ``sess.lens`` with ``lens_add = -1``
(the context's last token is the first one of the step) and ``new`` is ``sess.vlen`` with ``new_add = 1``.  The next
step's ``map`` gives back the pages of rejected tokens; a row with length 0 and no new tokens gives back all of its pages.

A row that the pool has no pages for has to sit the step out, or it would go on without its tokens' keys and values:
``map`` puts the step's new tokens into ``cache.new``, -1 - new_add for such a row.  ``attend`` goes by it; give it to the
logits (``new_lens=cache.new``) and to the verification (``sess.vlen.copy_(cache.new)``), and the row stays as it is.
Nothing here computes any part of the operators.

With a stream of its own (``stream=``) a cache's calls run there, whatever the current stream is: what fills their inputs
has to be ahead of them on that stream, and the inputs live until the calls are done.
"""
from __future__ import annotations

import torch

from . import binding as bd


class KVCache:
    def __init__(self, B: int, T: int, *, layers: int, heads: int, dim: int, pages: int, max_len: int, page: int = 64,
                 lens_add: int = 0, new_add: int = 0, device="cuda", stream: torch.cuda.Stream | None = None):
        """B rows of at most max_len tokens, T new tokens a step, `pages` pages of `page` tokens shared by the rows;
        lens_add and new_add are added to the lengths that the calls take.  `stream` (the current one of each call when
        None) is the stream of the calls; it waits for what fills the buffers here."""
        size = bd.switchsd_kv4_bytes(page, dim)
        if size == 0:
            raise ValueError(f"no 4-bit cache has pages of {page} tokens and heads of {dim} dimensions")
        self.B, self.T, self.layers, self.heads, self.dim, self.page, self.pages = B, T, layers, heads, dim, page, pages
        self.lens_add, self.new_add, self.stream = lens_add, new_add, stream
        i32 = dict(dtype=torch.int32, device=device)
        self.data = torch.zeros(layers, pages, heads, size, dtype=torch.uint8, device=device)
        self.table = torch.full((B, -(-max_len // page)), -1, **i32)
        self.held = torch.zeros(B, **i32)
        self.free_list = torch.arange(pages - 1, -1, -1, **i32)  # page 0 on top
        self.free_count = torch.full((1,), pages, **i32)
        self.slots = torch.full((B, T), -1, **i32)
        self.status = torch.zeros(B, **i32)
        self.new = torch.zeros(B, **i32)
        self.attend_status = torch.zeros(layers, B, **i32)
        self._layers = list(zip(self.data, self.attend_status))  # (a view made anew costs a call a microsecond)
        self.workspace = torch.empty(bd.switchsd_kv4_attention_workspace_of(dim), dtype=torch.uint8, device=device)
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream(self.data.device))
            for t in (self.data, self.table, self.held, self.free_list, self.free_count, self.slots, self.status, self.new, self.attend_status,
                      self.workspace):
                t.record_stream(stream)  # freed behind the calls
        self._lens = None

    def map(self, lens: torch.Tensor, new: torch.Tensor) -> None:
        """Pages for lens[b] + lens_add cached and new[b] + new_add new tokens of each row; fills slots, status and
        cache.new.  The calls that follow use the same `lens`, and cache.new."""
        self._lens = lens
        bd.switchsd_kv_map(lens, new, self.table, self.held, self.free_list, self.free_count, self.slots, page=self.page,
                           lens_add=self.lens_add, new_add=self.new_add, status=self.status, granted=self.new, stream=self.stream)

    def append(self, layer: int, k: torch.Tensor, v: torch.Tensor) -> None:
        """The new tokens' keys and values [B, T, heads, dim] into `layer`."""
        bd.switchsd_kv4_append(k, v, self.slots, self._layers[layer][0], page=self.page, stream=self.stream)

    def attend(self, layer: int, q: torch.Tensor, out: torch.Tensor, scale: float | None = None) -> torch.Tensor:
        """Attention of the new tokens' queries [B, T, query heads, dim] over `layer`, into `out`.  The rows' statuses go
        to attend_status[layer]: other than 0 where the row was left out or, ROW_TIMEOUT in all rows, where `out` does not
        count."""
        if self._lens is None:
            raise RuntimeError("map() comes before attend()")
        data, status = self._layers[layer]
        bd.switchsd_kv4_attention(q, data, self.table, self._lens, self.new, out, page=self.page, scale=scale,
                                  lens_add=self.lens_add, new_add=self.new_add, workspace=self.workspace, status=status,
                                  stream=self.stream)
        return out

    def read(self, layer: int, slots: torch.Tensor) -> tuple[torch.Tensor, torch.Tensor]:
        """What `layer` holds for slots int32 [B, n]: keys and values, f16 [B, n, heads, dim].  They belong to the current
        stream, which a cache's own stream waits for here, and which has to wait for that one before it uses them."""
        shape = (*slots.shape, self.heads, self.dim)
        k = torch.empty(shape, dtype=torch.float16, device=slots.device)
        v = torch.empty_like(k)
        if self.stream is not None:
            self.stream.wait_stream(torch.cuda.current_stream(slots.device))
            for t in (k, v):
                t.record_stream(self.stream)
        bd.switchsd_kv4_read(self._layers[layer][0], slots, k, v, page=self.page, stream=self.stream)
        return k, v
