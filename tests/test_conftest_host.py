"""Tests that name invented device addresses stay off machines with a GPU."""
import pathlib

import pytest
import torch

import conftest


class Item:
    def __init__(self, name):
        self.path, self.marks = pathlib.Path("tests") / name, []

    def add_marker(self, mark):
        self.marks.append(mark.name)


@pytest.mark.parametrize("gpus", [0, 1, 8])
def test_invented_addresses_are_for_machines_without_a_gpu(monkeypatch, gpus):
    monkeypatch.setattr(torch.cuda, "device_count", lambda: gpus)
    items = [Item(n) for n in ("test_abi_host.py", "test_rows_host.py", "test_rows_gpu.py", "test_pw_host.py")]
    conftest.pytest_collection_modifyitems(None, items)
    assert [i.marks for i in items] == [["skip"] * (gpus > 0)] * 2 + [[]] * 2
