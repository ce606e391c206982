"""The workspace of a stage's variant comes from the stage stream's memory: what another stream frees may still be in use
there.  Without a device: the stage's torch layer over stand-ins of the C ABI and of torch's streams."""
import contextlib
import types

import torch

from paper_2606_30634_amd import binding as B
from paper_2606_30634_amd import stage as stage_mod


class _Stream:
    def __init__(self, name):
        self.name, self.waited = name, []

    def wait_stream(self, other):
        self.waited.append(other)


def _stage(monkeypatch):
    mine, callers = _Stream("stage"), _Stream("caller")
    st = types.SimpleNamespace(stream=mine, device=torch.device("cpu"), handle=1, arena=torch.empty(1, dtype=torch.uint8),
                               shape=stage_mod.make_shape(1, 64, 2, 1, 32, 64, 0, False, False, False, 16, 1),
                               _hold_old_variant=lambda: None)
    at = [callers]

    @contextlib.contextmanager
    def stream(s):
        at.append(s)
        yield
        at.pop()

    made, empty = [], torch.empty

    def record(*a, **kw):
        made.append(at[-1])
        return empty(*a, **kw)

    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: at[-1])
    monkeypatch.setattr(torch, "empty", record)
    monkeypatch.setattr(B, "stage_variant_bytes", lambda s, v: 1000)
    monkeypatch.setattr(B, "stage_set_variant", lambda *a: None)
    return st, mine, callers, made


def test_the_variants_workspace_is_the_stage_streams(monkeypatch):
    st, mine, callers, made = _stage(monkeypatch)
    stage_mod.Stage.set_variant(st, softcap=2.0, documents=True)
    assert made == [mine] and mine.waited == []


def test_slopes_are_read_behind_the_callers_stream(monkeypatch):
    st, mine, callers, made = _stage(monkeypatch)
    stage_mod.Stage.set_variant(st, slopes=torch.ones(2))
    assert made == [mine] and mine.waited == [callers]
