"""e4m3 codes, values and products whose last elements lie past 2^32: each end against the same call on a small part."""
import pytest
import torch

from test_gpu_f8 import DEV, F8, awsrc

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("block_rows", [1, 128])
def test_codes_and_values_past_2_32(block_rows):
    rows, cols = 128 * 520 + 5, 65536 + 77
    assert rows * cols > 2 ** 32
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV).normal_()
    codes, scale = awsrc.awsrc_quantize_blocks_f8(x, block_rows)
    back = awsrc.awsrc_dequantize_blocks_f8(codes, scale, block_rows)
    for r0 in (0, 128 * 255, 128 * 518):  # from whole blocks on
        part = slice(r0, r0 + 261)
        c, s = awsrc.awsrc_quantize_blocks_f8(x[part].contiguous(), block_rows)
        assert torch.equal(codes[part].contiguous().view(torch.uint8)[:256], c.contiguous().view(torch.uint8)[:256])
        n = len(x[part])
        want = scale[:, r0:r0 + n] if block_rows == 1 else scale[r0 // 128:r0 // 128 + 2]
        assert torch.equal(want, s if block_rows == 1 else s[:2])
        v = awsrc.awsrc_dequantize_blocks_f8(c, s, block_rows)
        assert torch.equal(back[part][:256], v[:256])
    assert torch.equal(back[-5:], awsrc.awsrc_dequantize_blocks_f8(*awsrc.awsrc_quantize_blocks_f8(x[-5:].contiguous(), block_rows), block_rows))


def test_results_past_2_32():
    """Whole numbers, exact in any order."""
    M, N, K = 66001, 65537, 40
    assert M * N > 2 ** 32
    g = torch.Generator(DEV)
    g.manual_seed(3)
    x = torch.randint(-3, 4, (M, K), generator=g, device=DEV).float()
    x[:, 0] = 7.0  # the largest: every scale is 7 / 448, 2^-6
    w = torch.randint(-3, 4, (N, 48), generator=g, device=DEV).float().to(F8)[:, :K]
    sb = torch.exp2(torch.randint(0, 2, (-(-N // 128), 1), generator=g, device=DEV).float())
    out = awsrc.awsrc_linear_f8(x, w, sb, out_dtype=torch.bfloat16)
    scales = sb[torch.arange(N, device=DEV) // 128, 0]
    for m in (0, 32770, 65500, M - 130):
        want = (x[m:m + 130] @ w.float().T) * scales
        assert torch.equal(out[m:m + 130], want.bfloat16())
