"""The example that generates with drafted tokens: planning, e4m3 linear layers, the cache, attention and verification
together, on a cache whose pages come back and are taken again.

The bound on its logits: an e4m3 code is off by 2^-4 of its value at most, 2^-4 / sqrt(3) = 3.6% rms at most; the three
products that follow one another have two such operands each, 8.8% in quadrature.  The int8 cache adds 1.1% a rounding to
queries' products and values, 3% for all of them.  Together below 10%.
"""
import importlib.util
import os

import pytest

from conftest import ROOT

pytestmark = pytest.mark.gpu

pytest.importorskip("paper_2608_23144_amd")


@pytest.mark.parametrize("prompts,turns,drafts", [("300,65,1", 12, 4), ("1", 3, 1), ("64,128,127,129,5,70", 6, 7), ("40,3", 4, 0)])
def test_serve_drafts_example(prompts, turns, drafts):
    spec = importlib.util.spec_from_file_location("serve_drafts", os.path.join(ROOT, "examples", "serve_drafts.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    r = mod.main(["--seeds", "2", "--prompts", prompts, "--turns", str(turns), "--drafts", str(drafts)])
    assert r["worst"] < 0.10
    held, free, pages = r["pages"]
    assert held + free == pages
    assert 0 <= r["accepted"] <= r["offered"]
