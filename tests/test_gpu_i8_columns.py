"""The int8 product of one row against more columns than a launch has threads for."""
import pytest
import torch

pytestmark = pytest.mark.gpu

awsrc = pytest.importorskip("paper_2608_23144_amd")

DEV = "cuda"


def test_more_columns_than_a_launch_has_threads_for():
    """2^30 + 100 columns, in tiles of 64 columns and 128 threads: past 2^31 threads.  Sums of whole numbers, exact in bf16's 8 bits."""
    g = torch.Generator(DEV)
    g.manual_seed(1)
    N, K = 2 ** 30 + 100, 16
    w = torch.randint(0, 5, (N, K), generator=g, device=DEV, dtype=torch.int8).sub_(2)
    ws = torch.exp2(torch.randint(0, 2, (N,), generator=g, device=DEV).float())
    a = torch.randint(-3, 4, (1, K), generator=g, device=DEV, dtype=torch.int8)
    out = awsrc.awsrc_matmul_i8(a, torch.ones(1, device=DEV), w, ws)
    for n in (0, 2 ** 26 - 64, 2 ** 29 + 1, 2 ** 30 - 2 ** 26, 2 ** 30 - 64, 2 ** 30 + 99):
        m = min(N, n + 2 ** 24)
        assert torch.equal(out[0, n:m], ((w[n:m].float() * a.float()).sum(1) * ws[n:m]).bfloat16())
