"""Tests that give entry points made-up addresses stay off machines whose GPU these would reach."""
import pathlib
import re

import pytest
import torch

import conftest

HERE = pathlib.Path(__file__).parent
MADE_UP = re.compile(r"c_void_p\(\d|\bvp\(\d|FakeTensorMode\(")


class Item:
    def __init__(self, path, gpu):
        self.path, self.gpu, self.markers = path, gpu, []

    def get_closest_marker(self, name):
        return name == "gpu" and self.gpu

    def add_marker(self, marker):
        self.markers.append(marker.name)


@pytest.mark.parametrize("gpus", [0, 1, 8])
def test_made_up_addresses_need_a_machine_without_a_gpu(monkeypatch, gpus):
    monkeypatch.setattr(torch.cuda, "device_count", lambda: gpus)
    items = [Item(p, gpu) for p in sorted(HERE.glob("test_*.py")) for gpu in (False, True)]
    conftest.pytest_collection_modifyitems(items=items)
    made_up = [i for i in items if not i.gpu and MADE_UP.search(i.path.read_text())]
    assert len(made_up) >= 5
    for i in made_up:
        assert i.markers == (["skip"] if gpus else []), i.path
    assert not any(i.markers for i in items if i.gpu)
