"""Layers of few rows from two host threads at once, each with another need of LDS."""
import threading

import pytest
import torch

from test_gpu_f8 import DEV, _gen, _randn, awsrc

pytestmark = pytest.mark.gpu


def test_two_threads_at_once():
    """2 x 20480 takes the most LDS of all layers that quantize themselves, the others less."""
    shapes = [(2, 4000, 20480), (3, 4000, 6800), (16, 4000, 2500), (3, 4000, 13600)]
    work = []
    for M, N, K in shapes:
        g = _gen("threads", M, N, K)
        w, ws = awsrc.awsrc_quantize_blocks_f8(_randn(g, N, K).to(DEV), 128)
        x = _randn(g, M, K).bfloat16().to(DEV)
        assert awsrc.linear_f8_workspace_bytes(M, N, K) == 0
        work.append((x, w, ws, awsrc.awsrc_linear_f8(x, w, ws)))
    torch.cuda.synchronize()
    failed = []

    def calls(i):
        try:
            torch.cuda.set_device(0)
            stream = torch.cuda.Stream()
            for j in range(300):
                x, w, ws, want = work[(i + 2 * j) % 4 if j % 3 else i]
                got = awsrc.awsrc_linear_f8(x, w, ws, stream=stream)
                if j % 50 == 0:
                    stream.synchronize()
                    assert torch.equal(got, want)
            stream.synchronize()
        except BaseException as e:  # noqa: BLE001
            failed.append((i, e))

    threads = [threading.Thread(target=calls, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed
