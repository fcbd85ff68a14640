"""The example with drafted tokens: no turn waits for the host, and a prompt that comes later may be the longest."""
import importlib.util
import os

import pytest
import torch

from conftest import ROOT

pytestmark = pytest.mark.gpu

pytest.importorskip("paper_2608_23144_amd")


def _example():
    spec = importlib.util.spec_from_file_location("serve_drafts", os.path.join(ROOT, "examples", "serve_drafts.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_turns_do_not_wait_for_the_host():
    """Drafting and a turn under torch's own check, which raises where something waits."""
    mod = _example()
    calls = []

    def watched(f):
        def g(*args):
            torch.cuda.set_sync_debug_mode("error")
            try:
                return f(*args)
            finally:
                torch.cuda.set_sync_debug_mode("default")
                calls.append(f.__name__)
        return g

    mod.Model.turn, mod.Model.draft = watched(mod.Model.turn), watched(mod.Model.draft)
    mod.main(["--seeds", "2", "--prompts", "20,3", "--turns", "3", "--drafts", "2"])
    assert calls.count("draft") == 3 and calls.count("turn") == 5  # (and two turns of prompts)


def test_the_later_prompt_is_the_longest():
    """The prompt that takes the first slot is seven tokens longer than the last one: 135 here, which the tables have to hold.
    The bound is that of test_gpu_drafts_example.py."""
    r = _example().main(["--seeds", "2", "--prompts", "64,128", "--turns", "2", "--drafts", "1"])
    assert r["worst"] < 0.10
