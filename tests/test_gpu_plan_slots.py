"""Plans of more slots than one round of the scan takes (4096), and lengths written over the kept ones; all whole numbers,
all equal to the plan on Python lists."""
import numpy as np
import pytest
import torch

import drafts_ref as R
from test_gpu_drafts import Server, _ints, awsrc

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_seq,page,width,n_pages", [(4096, 16, 8, 12000), (4097, 32, 6, 9000), (8192, 16, 7, 30000), (9001, 64, 5, 15000),
                                                      (12289, 128, 3, 30000)])
def test_plan_of_many_slots(n_seq, page, width, n_pages):
    """Sums carried from round to round, lengths written in place before the next round reads its own; pools that run dry
    in the middle, slots that are turned away on both sides of a round's end."""
    rng = np.random.default_rng(n_seq)
    server = Server(rng, n_seq, page, width, n_pages)
    turned = 0
    for i in range(5):
        keep = np.maximum(0, server.kv - rng.integers(0, 9, n_seq)) * (rng.random(n_seq) > 0.15)
        new = np.where(rng.random(n_seq) < 0.7, rng.integers(0, 10, n_seq), rng.integers(0, page * width // 2, n_seq))
        rows = int(new.sum() * (0.8 if i % 2 else 1.0)) + 3
        want = server.step(keep, new, rows)
        turned += int(((np.diff(want["cu"]) == 0) & (new > 0)).sum())
        assert sorted(server.held() + server.free) == list(range(n_pages))
    assert turned


def test_plan_of_the_most_slots():
    """2^20 slots with a token or two each."""
    rng = np.random.default_rng(1)
    n = 1 << 20
    server = Server(rng, n, 16, 2, n + 1000)
    server.step(np.zeros(n, int), rng.integers(0, 3, n), 1100000)
    server.step(np.maximum(0, server.kv - rng.integers(0, 2, n)), rng.integers(0, 2, n), 600000)


@pytest.mark.parametrize("n_seq,rows", [(3, 20), (300, 1500), (2048, 9000), (5000, 20000)])
@pytest.mark.parametrize("same", [False, True])
def test_plan_into_keep(n_seq, rows, same):
    """kv_len_out given as keep, which may also be kv_len itself: everything stays."""
    rng = np.random.default_rng(n_seq)
    page, width, n_pages = 16, 9, n_seq * 8
    server = Server(rng, n_seq, page, width, n_pages)
    server.step(np.zeros(n_seq, int), rng.integers(0, 60, n_seq), n_seq * 60)
    kv = server.kv.copy()
    keep = kv if same else np.maximum(0, kv - rng.integers(0, 20, n_seq))
    new = rng.integers(0, 2 * rows // n_seq, n_seq)
    d_keep = server.d_kv if same else _ints(keep)
    got = awsrc.awsrc_kv_plan(server.pool, server.d_kv, d_keep, _ints(new), server.d_table, page, rows, kv_len_out=d_keep)
    want = R.plan(page, n_pages, server.free, kv.tolist(), keep.tolist(), new.tolist(), server.table, rows)
    for t, name in zip(got, ("cu", "seq", "pos", "slot")):
        assert np.array_equal(t.cpu().numpy(), want[name]), name
    assert np.array_equal(d_keep.cpu().numpy(), want["kv"])
    if not same:
        assert np.array_equal(server.d_kv.cpu().numpy(), kv)
    assert np.array_equal(server.d_table.cpu().numpy(), want["table"])
    assert server.pool[1].item() == len(want["free"])
    assert np.array_equal(server.pool[0].cpu().numpy()[:len(want["free"])], want["free"])
