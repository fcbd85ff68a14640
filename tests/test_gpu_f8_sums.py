"""Products of e4m3 matrices keep their sums in fp32 whatever the type of the result: exact where fp32 is, rounded once,
and on random codes within a few roundings of fp32 beside the result's own."""
import pytest
import torch

from test_gpu_f8 import DEV, EPS, F8, FLOOR, SHAPES, TYPES, _blocks, _codes, _gen, _scales, awsrc

pytestmark = pytest.mark.gpu

# weights that are read once, past the caches (up to 64 rows, 2^26 codes and more), with remainders in all three sizes, and
# long sums through the large tiles
ONCE = [(64, 24600, 2750), (33, 16640, 4100), (16, 13824, 4861), (16, 4096, 16400), (11, 4091, 16411), (2, 9001, 8203), (1, 12300, 5501),
        (27, 8203, 8200), (64, 8203, 8200)]
LONG = [(1100, 8200, 3001), (515, 5121, 5117), (140, 11001, 2055), (321, 11003, 1029)]


def _dense(t, s, block_rows):
    """code * scale in 64 bits."""
    s = s.double().T if block_rows == 1 else s.double().repeat_interleave(128, 0)[:t.shape[0]]
    return t.float().double() * s.repeat_interleave(128, 1)[:, :t.shape[1]]


def _numbers(g, rows, K):
    """Whole numbers of -3 to 3, NaN past the columns."""
    v = torch.randint(-3, 4, (rows, -(-K // 16) * 16), generator=g).float().to(F8)
    v.view(torch.uint8)[:, K:] = 0x7F
    return v.to(DEV)[:, :K]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", SHAPES + ONCE + LONG)
def test_sums_that_fp32_holds_are_exact(M, N, K, dtype):
    """Products of -9 to 9 beside a few of 2^16 and -2^16, scales of 1 or 2: every sum of some of them is a whole number
    below 2^24, which fp32 holds, whatever the order.  Then one rounding to the result's type."""
    g = _gen("loud", M, N, K)
    a, b = _numbers(g, M, K), _numbers(g, N, K)
    loud = torch.randperm(K - 1, generator=g)[:4].tolist() if K > 1 else []
    for k in loud:  # (neighbours, some of one eight and some of two)
        a[:, k], a[:, k + 1] = 256.0, -256.0
        b[:, k:k + 2] = 256.0
    sa, sb = (torch.exp2(torch.randint(0, 2, s, generator=g).float()).to(DEV) for s in _blocks(M, N, K))
    assert 4 * (8 * 2 ** 16 + 9 * K) < 2 ** 24
    want = _dense(a, sa, 1) @ _dense(b, sb, 128).T
    assert (want.float().double() == want).all()
    assert torch.equal(awsrc.awsrc_matmul_f8(a, sa, b, sb, out_dtype=dtype), want.float().to(dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(1, 2560, 2048), (13, 2048, 4100), (24, 3000, 1000), (24, 9001, 1000), (64, 2048, 2100), (64, 24600, 300),
                                   (300, 3000, 1337), (1100, 9001, 1111)] + ONCE[:4])
def test_sums_of_random_codes(M, N, K, dtype):
    """The error of a sum of random codes of both signs, on average.

    A sum of 128 products takes at most 127 additions in fp32, each off by at most a step, 2^-23 of a partial sum, whose rms is
    at most the whole sum's.  Their errors have no sign in common: sqrt(127) 2^-23 of the sum's rms together, and half a step for
    each of the blocks' scales and sums, sqrt(2 blocks) 2^-24.  Three times that is the bound on the error's rms, E.

    A result of 16 bits hides it behind its own rounding.  But it differs from the exact sum's rounding only where a border
    between two results lies between the two sums, which for sums that lie anywhere in a step is the case for a share of
    |error| / step of them, E / step on average; the count of such results may pass its expected value by six of its
    deviations."""
    g = _gen("rms", M, N, K)
    a, b = _codes(g, M, K), _codes(g, N, K)
    sa, sb = (_scales(g, *s) for s in _blocks(M, N, K))
    x, w = _dense(a, sa, 1), _dense(b, sb, 128)
    want = x @ w.T
    got = awsrc.awsrc_matmul_f8(a, sa, b, sb, out_dtype=dtype).double()
    rms, blocks = want.square().mean().sqrt().item(), -(-K // 128)
    most = 3 * (127 ** 0.5 * 2.0 ** -23 + (2 * blocks) ** 0.5 * 2.0 ** -24) * rms
    if dtype == torch.float32:
        assert (got - want).square().mean().sqrt().item() <= most + 2.0 ** -24 * rms
        return
    fine = want.abs() < 0.99 * torch.finfo(dtype).max
    once = want.to(dtype).double()
    step = (2 * EPS[dtype] * torch.exp2(torch.floor(torch.log2(want.abs().clamp_min(2.0 ** -140))))).clamp_min(2 * FLOOR[dtype])
    share = (most / step[fine]).clamp_max(1)
    expect = share.sum().item()
    assert (got != once)[fine].sum().item() <= expect + 6 * (expect ** 0.5 + 1)


def test_more_columns_than_a_launch_has_threads_for():
    """One row against 2^30 + 100 columns, in tiles of 64 columns and 128 threads: past 2^31 threads."""
    g = torch.Generator(DEV)
    g.manual_seed(1)
    N, K = 2 ** 30 + 100, 16
    w = torch.randint(0, 3, (N, K), generator=g, device=DEV, dtype=torch.uint8).mul_(24).view(F8)  # 0, 2^-4 or 0.5
    sb = torch.exp2(torch.randint(0, 2, (-(-N // 128), 1), generator=g, device=DEV).float())
    x = torch.randint(-3, 4, (1, K), generator=g, device=DEV).float()
    a, sa = x.to(F8), torch.ones(1, 1, device=DEV)
    out = awsrc.awsrc_matmul_f8(a, sa, w, sb)
    for n in (0, 2 ** 26 - 64, 2 ** 29 + 1, 2 ** 30 - 2 ** 26, 2 ** 30 - 64, 2 ** 30 + 99):
        m = min(N, n + 2 ** 24)
        columns = torch.arange(n, m, device=DEV) // 128
        want = (w[n:m].float() * x).sum(1) * sb[columns, 0]  # (multiples of 2^-4 below 2^6: exact)
        assert torch.equal(out[0, n:m], want.bfloat16())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(1, 4091, 16411), (2, 4096, 16384), (1, 2101, 32767), (1, 9001, 8203), (1, 4097, 16400), (1, 70001, 1001),
                                   (16, 13825, 4861), (64, 24600, 2750)])
def test_linear_on_weights_past_the_caches(M, N, K, dtype):
    """Layers whose weights are read once, quantized in the product's launch and in one of its own.  The sum of each block's 128
    products is off by 127 steps of fp32 at most, the scales' product, each block's fma, up to 16 parts, the bias and the result's
    rounding by half a step each."""
    g = _gen("once", M, N, K)
    x = (torch.randn(M, K, generator=g) * torch.exp(torch.randn(K, generator=g))).to(dtype).to(DEV)
    w, sb = _codes(g, N, K), _scales(g, *_blocks(M, N, K)[1])
    bias = torch.randn(N, generator=g).to(DEV)
    codes, sa = awsrc.awsrc_quantize_blocks_f8(x)
    a, b = _dense(codes, sa, 1), _dense(w, sb, 128)
    want, mag = a @ b.T + bias.double(), a.abs() @ b.abs().T + bias.double().abs()
    tol = mag * (127 * 2.0 ** -23 + (-(-K // 128) + 18) * 2.0 ** -24) + EPS[dtype] * want.abs() * (1 + 2.0 ** -10) + FLOOR[dtype]
    got = awsrc.awsrc_linear_f8(x, w, sb, bias=bias).double()
    sure = want.abs() + tol < torch.finfo(dtype).max
    assert ((got - want).abs() <= tol)[sure].all()
    assert sure.double().mean() > 0.9
