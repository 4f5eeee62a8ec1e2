"""The example runs every operator next to the steps it serves, and learns."""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_head_is_trained_and_served(cuda_device):
    spec = importlib.util.spec_from_file_location("example", os.path.join(ROOT, "examples", "train_and_serve_head.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    first, last, share = m.train_and_serve(steps=60, say=lambda *a: None)
    # an untrained model is near log V; the chain's own entropy is about 1
    # nat, and a model that knows every successor generates only those
    assert abs(first - math.log(1024)) < 1.0
    assert last < 0.5 * first and share > 0.9
