"""Where the checked calls of the row operators run, with the GPU's side replaced."""
import contextlib
from types import SimpleNamespace

import pytest
import torch

from paper_2309_15812_amd import _lib, ops


@pytest.mark.parametrize("current", [0, 1])
def test_calls_run_with_their_tensors_device_as_the_current_one(monkeypatch, current):
    state, ran = {"device": current}, []

    @contextlib.contextmanager
    def device(d):
        was, state["device"] = state["device"], d
        yield
        state["device"] = was

    def entry(*args):
        ran.append((state["device"], args))
        return 0

    monkeypatch.setattr(torch.cuda, "current_device", lambda: state["device"])
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(_lib, "lib", lambda: SimpleNamespace(o1d_pack=entry))
    monkeypatch.setattr(ops, "_stream", lambda t: 7)
    ops._run("o1d_pack", SimpleNamespace(get_device=lambda: 1), 1, 2, 3)
    assert ran == [(1, (1, 2, 3, 7))] and state["device"] == current
