"""The example of a served layer: every step of a small server against each request's own keys and values."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


def _example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serving_steps.py")
    spec = importlib.util.spec_from_file_location("serving_steps", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("slots,chunk,seed", [(6, 48, 1), (3, 7, 2), (9, 200, 3)])
def test_server_steps(slots, chunk, seed):
    worst, steps = _example().check(slots, chunk, seed)
    assert steps > 12 and worst <= 1.0
