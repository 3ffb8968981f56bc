"""The example's parameters, on the CPU: experts start from the scale of the layer that they replace."""
import importlib.util
import math
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("training_iteration", os.path.join(ROOT, "examples", "training_iteration.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("experts", [1, 4])
def test_scales(example, experts):
    """Normal with the variance 1 / terms of the sum: a mean square of N of them is within six of its standard
    deviations, sqrt(2 / N), of that."""
    width = 32
    dense, some = example.model(10, width, "cpu", 1), example.model(10, width, "cpu", 1, experts)
    for p, leads in ((dense, {"up": width, "down": 4 * width}),
                     (some, {"up": width, "down": 4 * width, "router": width})):
        for name, terms in leads.items():
            w = p[name].detach().double()
            assert abs(float(w.square().mean()) * terms - 1) <= 6 * math.sqrt(2 / w.numel()), name
