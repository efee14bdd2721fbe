"""Memory that the binding takes from torch for a call belongs to the call's stream."""
import contextlib
import inspect

import torch

from paper_2609_20186_gb300 import binding as bd
from paper_2609_20186_gb300 import build


def test_scratch_is_taken_under_the_calls_stream(monkeypatch):
    build.build()
    under, seen = [], []
    real = torch.empty

    @contextlib.contextmanager
    def stream(s):
        under.append(s)
        yield
        under.pop()

    def empty(*a, **k):
        seen.append(under[-1] if under else None)
        return real(*a, **k)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch, "empty", empty)
    side = object()
    assert bd._scratch(16, "cpu", side).numel() == 16 and bd._scratch(16, "cpu", None).numel() == 16
    p = bd.switchsd_params()
    p.B, p.d, p.probe_kind, p.probe_hidden = 4, 256, bd.PROBE_MLP, 64
    assert seen == [side, None]
    with contextlib.suppress(ValueError):  # (this one is not a CUDA tensor)
        bd._attach_workspace(p, None, "cpu", side)
    assert seen == [side, None, side]


def test_the_binding_takes_memory_in_no_other_place():
    text = inspect.getsource(bd)
    inside = inspect.getsource(bd._scratch)
    for what in ("torch.empty", "torch.zeros", "torch.full", "empty_like", "new_empty"):
        assert text.count(what) == inside.count(what), what
