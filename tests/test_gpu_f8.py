"""e4m3 codes, their values and their products on the GPU: codes and scales to
the bit against the fp32 recipe, products exact where the arithmetic is, and
otherwise within the bound of their roundings."""
import numpy as np
import pytest
import torch

import drafts_ref as R

pytestmark = pytest.mark.gpu

awsrc = pytest.importorskip("paper_2608_23144_amd")

DEV = "cuda"
F8 = torch.float8_e4m3fn
TYPES = [torch.float32, torch.bfloat16, torch.float16]
EPS = {t: torch.finfo(t).eps / 2 for t in TYPES}  # half a step, relative
FLOOR = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}  # half a step of subnormals


def _gen(*key):
    g = torch.Generator()
    g.manual_seed(sum((i + 1) * ord(c) for i, c in enumerate(repr(key))))
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g)


def _bytes(t):
    return t.view(torch.uint8).cpu().numpy()


def _same(a, b):
    a, b = np.asarray(a), np.asarray(b)
    assert a.shape == b.shape and a.dtype == b.dtype
    if a.dtype.kind == "f":
        assert np.array_equal(np.isnan(a), np.isnan(b))
        a, b = np.nan_to_num(a, nan=0.0), np.nan_to_num(b, nan=0.0)
    assert np.array_equal(a, b), f"{np.sum(a != b)} of {a.size} differ"


# ------------------------------------------------------------------ codes
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (3, 16), (5, 129), (2, 255), (129, 500), (128, 128), (300, 700), (31, 4097),
                                       (33, 513), (2100, 300)])
def test_quantize_bits(rows, cols, block_rows, dtype):
    g = _gen("rows", rows, cols)
    x = (_randn(g, rows, cols) * torch.exp(2 * _randn(g, rows, 1)) * torch.exp(_randn(g, 1, cols))).to(dtype)
    c, s = awsrc.awsrc_quantize_blocks_f8(x.to(DEV), block_rows)
    want_c, want_s = R.quantize_blocks(x.float().numpy(), block_rows)
    _same(s.cpu().numpy(), want_s)
    _same(_bytes(c), want_c)
    assert c.dtype == F8 and c.stride(0) % 16 == 0


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_every_rounding(block_rows):
    """Values on and beside the borders between codes, of both signs, down to the smallest."""
    v = R.decode(np.arange(127))
    mid = (v[1:] + v[:-1]) / 2
    x = np.concatenate([v, mid, np.nextafter(mid.astype(np.float32), np.float32(0)), np.nextafter(mid.astype(np.float32), np.float32(500))])
    x = np.concatenate([x, -x])
    x = np.concatenate([x, np.zeros(-len(x) % 127)]).reshape(-1, 127).astype(np.float32)
    x = np.concatenate([x, np.full((len(x), 1), 448, np.float32)], 1)  # scale 1
    c, s = awsrc.awsrc_quantize_blocks_f8(torch.from_numpy(x).to(DEV), block_rows)
    assert (s == 1).all()
    _same(_bytes(c), R.encode(x))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("cols", [33, 300])
def test_quantize_special_values(cols, block_rows, dtype):
    g = _gen("special", cols)
    x = _randn(g, 9 * 128, cols)
    at = np.s_[::128] if block_rows == 128 else np.s_[:9]
    y = x[at]
    if block_rows == 128:
        for i in range(9):  # blocks that hold nothing louder than what is put there
            if i in (0, 1, 6):
                x[i * 128:(i + 1) * 128] = 0
    y[0] = -0.0
    y[1] = -2.0 ** -110  # below the smallest stored magnitude (0 in fp16 already)
    y[2, cols - 1] = float("inf")
    y[3, 0] = float("nan")
    y[4, cols // 2] = -float("inf")
    y[5] = -y[5].abs()
    y[6] = 0
    y[6, cols - 1] = 1e-3
    y[7] = 3.0
    y[8, :] = torch.finfo(dtype).max if dtype != torch.float32 else 3e38
    x[at] = y
    x = x.to(dtype)
    c, s = awsrc.awsrc_quantize_blocks_f8(x.to(DEV), block_rows)
    want_c, want_s = R.quantize_blocks(x.float().numpy(), block_rows)
    _same(s.cpu().numpy(), want_s)
    _same(_bytes(c), want_c)
    assert torch.isnan(s).any() and (s == 0).any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("offset,stride,at,after", [(0, 151, 0, 0), (1, 152, 3, 5), (3, 149, 16, 12), (8, 160, 1, 40)])
def test_quantize_and_back_inside_wider_buffers(offset, stride, at, after, block_rows, dtype):
    """Rows at any alignment, codes and values into column slices: nothing around them is written."""
    rows, cols = 131, 149
    g = _gen("views", offset, stride)
    buf = _randn(g, rows * stride + offset).to(dtype).to(DEV)
    x = buf[offset:].as_strided((rows, cols), (stride, 1))
    full = torch.full((rows + 2, at + cols + after), 77, dtype=torch.uint8, device=DEV)
    codes = full.view(F8)[1:rows + 1, at:at + cols]
    shape = (2, rows) if block_rows == 1 else (2, 2)
    s = torch.empty(shape, device=DEV)
    awsrc.awsrc_quantize_blocks_f8(x, block_rows, out=(codes, s))
    want_c, want_s = R.quantize_blocks(x.float().cpu().numpy(), block_rows)
    want = np.full(full.shape, 77, np.uint8)
    want[1:rows + 1, at:at + cols] = want_c
    _same(full.cpu().numpy(), want)
    _same(s.cpu().numpy(), want_s)
    back = torch.full((rows + 2, at + cols + after), 7.0, dtype=dtype, device=DEV)
    awsrc.awsrc_dequantize_blocks_f8(codes, s, block_rows, out=back[1:rows + 1, at:at + cols])
    v = torch.full(back.shape, 7.0, dtype=dtype)
    v[1:rows + 1, at:at + cols] = torch.from_numpy(R.values(want_c, want_s, block_rows).astype(np.float32)).to(dtype)
    assert torch.equal(back.cpu(), v)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("block_rows", [1, 128])
def test_every_code_back(block_rows, dtype):
    """All 256 codes in every place of a lane, with scales from tiny to large: one rounding of code * scale."""
    codes = torch.arange(256, dtype=torch.int32).repeat(5)[:1275].to(torch.uint8).repeat(3, 1).to(DEV).view(F8)
    g = _gen("back")
    s = torch.exp(20 * _randn(g, *((10, 3) if block_rows == 1 else (1, 10)))).to(DEV)
    got = awsrc.awsrc_dequantize_blocks_f8(codes, s, block_rows, dtype=dtype)
    want = torch.from_numpy(R.values(_bytes(codes), s.cpu().numpy(), block_rows)).float().to(dtype)
    _same(got.float().cpu().numpy(), want.float().numpy())


# ------------------------------------------------------------------ products
def _codes(g, rows, cols, fill=0x7F):
    """Random finite codes in rows on 16 bytes; past the columns NaN codes, which must not matter."""
    ld = -(-cols // 16) * 16
    buf = torch.randint(0, 127, (rows, ld), generator=g, dtype=torch.int32)
    buf = (buf | torch.randint(0, 2, (rows, ld), generator=g, dtype=torch.int32) << 7).to(torch.uint8)
    if fill is not None:
        buf[:, cols:] = fill
    return buf.view(F8).to(DEV)[:, :cols]


def _scales(g, *shape):
    return (torch.exp(_randn(g, *shape)) * 1e-2).to(DEV)


def _blocks(M, N, K):
    return (-(-K // 128), M), (-(-N // 128), -(-K // 128))


def _dense(t, s, block_rows):
    return torch.from_numpy(R.values(_bytes(t.contiguous()), s.cpu().numpy(), block_rows)).to(DEV)


def _check(out, a, sa, b, sb, bias, dtype):
    x, w = _dense(a, sa, 1), _dense(b, sb, 128)
    want, mag = x @ w.T, x.abs() @ w.abs().T
    if bias is not None:
        want, mag = want + bias.double(), mag + bias.double().abs()
    # A block's 128 products are exact (8 bits) and summed by the matrix core in fp32, in an order that is its own: each of
    # 127 additions is off by a step at most.  For 16-bit results it takes eight products at a time, at the exponent of the
    # largest: seven of them lose less than 2^-13 of it each, and it is at most the eight's sum of magnitudes.  Then half a
    # step each: the scales' product, an fma a block, up to 16 parts joined, the bias, the result's own rounding.
    blocks = -(-a.shape[1] // 128)
    cut = 0 if dtype == torch.float32 else 7 * 2.0 ** -13
    tol = mag * (cut + 127 * 2.0 ** -23 + (blocks + 18) * 2.0 ** -24) + EPS[dtype] * want.abs() * (1 + 2.0 ** -10) + FLOOR[dtype]
    got, big = out.double(), torch.finfo(dtype).max
    sure = want.abs() + tol < big
    err = torch.where(sure, got - want, torch.zeros_like(want)).abs()
    assert (err <= tol).all(), f"{float((err / tol).max())} times the bound"
    over = want.abs() - tol > big * 1.01
    assert torch.equal(got[over], want[over].sign() * float("inf"))


SHAPES = [(1, 1, 1), (1, 16, 16), (1, 2560, 2048), (2, 17, 33), (3, 100, 1000), (13, 96, 4100), (16, 64, 64), (17, 130, 127),
          (31, 48, 272), (33, 256, 128), (64, 300, 513), (65, 65, 65), (100, 257, 1040), (128, 128, 128), (129, 127, 2000),
          (255, 513, 96), (256, 256, 256), (300, 1003, 1337), (511, 260, 144), (1, 33, 131071), (70, 40, 20000),
          (5, 8200, 300), (30, 200, 9000), (50, 130, 5003), (64, 9001, 513), (40, 24700, 144), (129, 16640, 260), (90, 100, 12289),
          (9, 12400, 129), (20, 8300, 200), (32, 100, 17000), (700, 3000, 640), (2000, 4100, 200), (1500, 9001, 333), (1025, 12300, 384),
          (130, 2050, 6000), (16, 4096, 4097), (7, 4097, 4096), (16, 100, 4095), (40, 8203, 8200), (5, 8203, 8200), (130, 8200, 300), (513, 4097, 260), (24, 5120, 4000), (64, 2048, 11008), (300, 12000, 250), (16, 12289, 2049), (48, 24600, 2100)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_matmul(M, N, K, dtype):
    g = _gen("mm", M, N, K)
    a, b = _codes(g, M, K), _codes(g, N, K, fill=0xFF)
    sa, sb = (_scales(g, *s) for s in _blocks(M, N, K))
    bias = _randn(g, N).to(DEV) if (M + N) % 2 else None
    out = awsrc.awsrc_matmul_f8(a, sa, b, sb, bias=bias, out_dtype=dtype)
    assert out.dtype == dtype
    _check(out, a, sa, b, sb, bias, dtype)


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_matmul_of_whole_numbers_is_exact(M, N, K):
    """Small whole numbers and scales that are powers of two: every sum is exact in fp32, whatever its order."""
    g = _gen("whole", M, N, K)

    def numbers(rows):
        v = torch.randint(-3, 4, (rows, -(-K // 16) * 16), generator=g).float().to(F8)
        v.view(torch.uint8)[:, K:] = 0x7F
        return v.to(DEV)[:, :K]

    a, b = numbers(M), numbers(N)
    sa, sb = (torch.exp2(torch.randint(0, 2, s, generator=g).float()).to(DEV) for s in _blocks(M, N, K))
    out = awsrc.awsrc_matmul_f8(a, sa, b, sb, out_dtype=torch.float32)
    want = _dense(a, sa, 1) @ _dense(b, sb, 128).T  # below 9 * 4 * 131071 < 2^24
    assert torch.equal(out.double(), want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(3, 37, 80), (20, 129, 65), (140, 270, 130), (260, 515, 400)])
def test_matmul_strided_and_guarded(M, N, K, dtype):
    """Operands and results inside wider buffers; nothing around the result is written."""
    g = _gen("guard", M, N, K)
    A, B = _codes(g, M + 2, K + 64, fill=None), _codes(g, N + 2, K + 96, fill=None)
    a, b = A[1:M + 1, 16:16 + K], B[1:N + 1, 32:32 + K]
    sa, sb = (_scales(g, *s) for s in _blocks(M, N, K))
    for pad, off in ((3, 0), (8, 0), (5, 1), (0, 0)):
        buf = torch.full(((M + 2) * (N + pad) + off,), 7.0, dtype=dtype, device=DEV)
        out = buf[off:].view(M + 2, N + pad)[1:M + 1, :N]
        awsrc.awsrc_matmul_f8(a, sa, b, sb, out=out)
        _check(out, a, sa, b, sb, None, dtype)
        mask = torch.ones_like(buf, dtype=torch.bool)
        mask[off:].view(M + 2, N + pad)[1:M + 1, :N] = False
        assert (buf[mask] == 7.0).all()


@pytest.mark.parametrize("M,N,K", [(7, 70, 80), (33, 160, 300), (70, 24640, 96), (300, 272, 1440)])
def test_matmul_scales_off_16_bytes(M, N, K):
    """Scales and bias from any element of a longer vector."""
    g = _gen("scales", M, N, K)
    a, b = _codes(g, M, K), _codes(g, N, K)
    shapes = _blocks(M, N, K)
    big = [_scales(g, s[0] * s[1] + 3) for s in shapes]
    bias = _randn(g, N + 3).to(DEV)
    for i, j, k in ((0, 1, 0), (3, 0, 2), (1, 2, 3)):
        sa, sb = (t[o:o + s[0] * s[1]].view(s) for t, o, s in zip(big, (i, j), shapes))
        out = awsrc.awsrc_matmul_f8(a, sa, b, sb, bias=bias[k:k + N])
        _check(out, a, sa, b, sb, bias[k:k + N], torch.bfloat16)


@pytest.mark.parametrize("M,N,K", [(5, 300, 400), (70, 300, 400), (300, 600, 700)])
def test_matmul_nan_stays_where_it_belongs(M, N, K):
    g = _gen("nan", M)
    a, b = _codes(g, M, K), _codes(g, N, K)
    sa, sb = (torch.ones(s, device=DEV) for s in _blocks(M, N, K))
    sa[2, 3] = float("nan")  # one block of row 3
    sb[1, 0] = float("nan")  # one block of columns 128 to 255
    b.view(torch.uint8)[7, 200] = 0x7F
    a.view(torch.uint8)[1, K - 1] = 0xFF
    bad = torch.isnan(awsrc.awsrc_matmul_f8(a, sa, b, sb, out_dtype=torch.float32)).cpu()
    want = torch.zeros(M, N, dtype=torch.bool)
    want[3], want[1], want[:, 128:256], want[:, 7] = True, True, True, True
    assert torch.equal(bad, want)


@pytest.mark.parametrize("M,N,K", [(2, 600, 130), (40, 600, 130), (300, 600, 130)])
def test_matmul_rows_past_2_31_bytes(M, N, K):
    """Weight rows 4 MB apart: the last ones start beyond 2^31 bytes."""
    g = _gen("far", M)
    ld = 1 << 22
    wide = torch.empty(N * ld, dtype=torch.uint8, device=DEV).view(F8).view(N, ld)
    b = wide[:, :K]
    b.copy_(_codes(g, N, K))
    a = _codes(g, M, K)
    sa, sb = (_scales(g, *s) for s in _blocks(M, N, K))
    _check(awsrc.awsrc_matmul_f8(a, sa, b, sb), a, sa, b, sb, None, torch.bfloat16)


LINEAR = [(1, 70, 96), (1, 2560, 2048), (4, 65, 1000), (13, 200, 4100), (40, 90, 33), (200, 130, 257), (1, 40, 1), (1, 9000, 11008),
          (2, 16, 16384), (2, 9001, 100), (3, 50, 10922), (5, 300, 515), (8, 1030, 4096), (16, 33, 2048), (16, 130, 2047),
          (16, 130, 2049), (9, 17, 65), (3, 9000, 70), (300, 1003, 1337), (1, 1000, 32768), (1, 3000, 32767), (1, 100, 32769),
          (1, 30000, 500), (16, 4096, 1024), (16, 4112, 1025), (2, 100, 8192), (2, 100, 8193), (1, 8203, 8200), (4, 5000, 5120), (4, 5000, 5121),
          (16, 4096, 2560), (16, 4097, 2560), (16, 130, 2561), (5, 33, 8192), (2, 300, 20480)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", LINEAR)
def test_linear(M, N, K, dtype):
    """The product of the recipe's codes, from rows at any place."""
    g = _gen("lin", M, N, K)
    x = (_randn(g, M, K) * torch.exp(_randn(g, K))).to(dtype).to(DEV)
    if M > 2:
        x[1] = 0
    w, ws = awsrc.awsrc_quantize_blocks_f8(_randn(g, N, K).to(DEV), 128)
    bias = _randn(g, N).to(DEV)
    c, s = awsrc.awsrc_quantize_blocks_f8(x)
    got = awsrc.awsrc_linear_f8(x, w, ws, bias=bias)
    assert got.dtype == dtype
    _check(got, c, s, w, ws, bias, dtype)
    wide = torch.zeros(M, K + 5, dtype=dtype, device=DEV)  # rows that lie apart, at odd places
    wide[:, 3:3 + K] = x
    assert torch.equal(awsrc.awsrc_linear_f8(wide[:, 3:3 + K], w, ws, bias=bias), got)
    _check(awsrc.awsrc_linear_f8(x, w, ws, out_dtype=torch.float32), c, s, w, ws, None, torch.float32)


@pytest.mark.parametrize("M", [5, 20, 100])
def test_linear_block_that_is_not_finite(M):
    """A value that is not finite takes its row with it and no other."""
    g = _gen("inf")
    x = _randn(g, M, 300).to(DEV)
    x[2, 7] = float("inf")
    x[4, 299] = float("nan")
    w, ws = awsrc.awsrc_quantize_blocks_f8(_randn(g, 40, 300).to(DEV), 128)
    bad = torch.isnan(awsrc.awsrc_linear_f8(x, w, ws)).cpu()
    want = torch.zeros(M, 40, dtype=torch.bool)
    want[[2, 4]] = True
    assert torch.equal(bad, want)


@pytest.mark.parametrize("M,N,K", [(1, 2560, 2048), (13, 2048, 11008), (40, 300, 5000), (64, 9000, 600), (300, 700, 1337)])
def test_linear_repeats_itself(M, N, K):
    """The same bits on every call, whatever the workspace held, on another stream and from a graph; nothing is written past
    the workspace."""
    g = _gen("again", M, N, K)
    x = _randn(g, M, K).bfloat16().to(DEV)
    w, ws = awsrc.awsrc_quantize_blocks_f8(_randn(g, N, K).to(DEV), 128)
    first = awsrc.awsrc_linear_f8(x, w, ws)
    need = awsrc.linear_f8_workspace_bytes(M, N, K)
    scratch = torch.empty(need + 64, dtype=torch.uint8, device=DEV)
    for value in (0, 255, 127):
        scratch.fill_(value)
        assert torch.equal(awsrc.awsrc_linear_f8(x, w, ws, workspace=scratch[:need] if need else None), first)
        assert (scratch[need:] == value).all()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = awsrc.awsrc_linear_f8(x, w, ws, stream=side)
    side.synchronize()
    assert torch.equal(other, first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = awsrc.awsrc_linear_f8(x, w, ws)
    for i in range(4):
        x.copy_(_randn(g, M, K).bfloat16())
        graph.replay()
        eager = awsrc.awsrc_linear_f8(x, w, ws)
        torch.cuda.synchronize()
        assert torch.equal(held, eager)


def test_empty_products():
    w, ws = awsrc.awsrc_quantize_blocks_f8(torch.randn(5, 40, device=DEV), 128)
    assert awsrc.awsrc_linear_f8(torch.empty(0, 40, device=DEV), w, ws).shape == (0, 5)
    empty = torch.empty(0, 48, dtype=torch.uint8, device=DEV).view(F8)[:, :40]
    assert awsrc.awsrc_linear_f8(torch.randn(3, 40, device=DEV), empty, torch.empty(0, 1, device=DEV)).shape == (3, 0)
    c, s = awsrc.awsrc_quantize_blocks_f8(torch.empty(0, 40, device=DEV))
    assert c.shape == (0, 40) and s.shape == (1, 0) and awsrc.awsrc_dequantize_blocks_f8(c, s).shape == (0, 40)
