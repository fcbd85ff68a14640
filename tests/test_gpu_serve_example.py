"""The serving example: prompts, decode steps through a captured graph, and
their distance from the layer in fp32.

The bound: each of the two quantized operands of a product carries a rounding
of half a step of amax / 127 at most, 0.29 steps rms; with amax near five deviations
that is 1.1% of an operand, keys and values a third and fourth rounding and a page's
largest token a larger step.  Six such roundings in quadrature stay below 5%.
"""
import importlib.util
import os

import pytest

from conftest import ROOT

pytestmark = pytest.mark.gpu

pytest.importorskip("paper_2608_23144_amd")


@pytest.mark.parametrize("prompts,steps", [("700,65,1", 8), ("1", 0), ("64,128", 1)])
def test_serve_layer_example(prompts, steps):
    spec = importlib.util.spec_from_file_location("serve_layer", os.path.join(ROOT, "examples", "serve_layer.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    assert mod.main(["--seeds", "2", "--prompts", prompts, "--steps", str(steps)]) < 0.05
