"""The serving example: histories taken in as prompts and grown item by item give what one prompt over everything gives."""
import importlib.util
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
@pytest.mark.parametrize("users,history,steps", [(5, 70, 3), (1, 300, 2), (40, 33, 40)])
def test_serving_example(users, history, steps):
    spec = importlib.util.spec_from_file_location("serve_paged", os.path.join(ROOT, "examples", "serve_paged.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    # both sides are within the bf16 bound (2e-2 of values up to about 3) of the exact result
    assert module.main(users, history, steps) <= 0.12
