"""The e4m3 calls, the step plan and the draft verification refuse bad arguments
before anything touches a device, answer their workspace queries without one,
and take empty batches; the references they are held to, against torch's own types."""
import ctypes

import numpy as np
import pytest
import torch

import drafts_ref as R

awsrc = pytest.importorskip("paper_2608_23144_amd")

L = awsrc.LIB
OK, EINVAL, ENOSPC = awsrc.AWSRC_OK, awsrc.AWSRC_EINVAL, awsrc.AWSRC_ENOSPC
F32, BF16, F16 = 0, 1, 2
P = 4096  # an address that no refused call follows
F8 = torch.float8_e4m3fn


def _call(f, base, **bad):
    args = dict(base)
    for k in bad:
        assert k in args
    args.update(bad)
    st = f(*args.values())
    if st != OK:
        assert L.awsrc_last_error()
    return st


def _ws(n=0):
    return ctypes.byref(ctypes.c_size_t(n))


# ------------------------------------------------------------------ the references
def test_reference_codes_are_torchs():
    every = torch.arange(256, dtype=torch.uint8).view(F8).double().numpy()
    assert np.array_equal(np.isnan(R.decode(np.arange(256))), np.isnan(every))
    assert np.array_equal(np.nan_to_num(R.decode(np.arange(256))), np.nan_to_num(every))
    g = np.random.default_rng(0)
    x = np.clip(g.standard_normal(100000) * np.exp(3 * g.standard_normal(100000)), -448, 448).astype(np.float32)
    assert np.array_equal(R.encode(x), torch.from_numpy(x).to(F8).view(torch.uint8).numpy())


def test_reference_plan_by_hand():
    """Two slots, pages of 16: the first gives back two pages and the second takes three, the two and the stack's top."""
    table = np.array([[4, 5, 6, -1], [7, -1, -1, -1]], np.int32)
    r = R.plan(16, 9, [0, 1, 2, 3], [40, 16], [9, 16], [0, 40], table, 42)
    assert r["cu"].tolist() == [0, 0, 40] and r["kv"].tolist() == [9, 56]
    assert r["table"].tolist() == [[4, 5, 6, -1], [7, 5, 6, 3]] and r["free"] == [0, 1, 2]
    assert r["pos"][:2].tolist() == [16, 17] and r["slot"][0] == 5 * 16 and r["slot"][39] == 3 * 16 + 7 and r["slot"][40] == -1


def test_reference_verify_by_hand():
    p = np.array([[0.5, 0.5, 0], [0.1, 0.2, 0.7]], np.float32)
    q = np.array([[0.75, 0.25, 0], [1, 0, 0]], np.float32)
    cu = np.array([0, 2])
    assert R.verify(p, q, [9, 0], np.array([0.6, 0.25], np.float32), cu)[0].tolist() == [0, 1]  # 0.45 < 0.5; 0.1 <= 0.25 < 0.3
    out, n = R.verify(p, q, [9, 0], np.array([0.9, 0.0], np.float32), cu)  # refused: only token 1 has weight left
    assert out.tolist() == [1, -1] and n.tolist() == [1]


# ------------------------------------------------------------------ refusals
QUANT = dict(X=P, x_dtype=F32, rows=4, cols=33, ldx=40, block_rows=1, codes=P, ldc=48, scale=P, stream=None)


@pytest.mark.parametrize("bad", [dict(x_dtype=3), dict(x_dtype=-1), dict(rows=-1), dict(cols=0), dict(ldx=32), dict(ldc=32),
                                 dict(X=None), dict(codes=None), dict(scale=None), dict(X=P + 2), dict(scale=P + 2),
                                 dict(rows=1 << 31), dict(ldx=1 << 31), dict(ldc=1 << 31), dict(block_rows=0), dict(block_rows=2),
                                 dict(block_rows=64), dict(block_rows=-1)])
def test_quantize_refuses(bad):
    assert _call(L.awsrc_quantize_blocks_f8, QUANT, **bad) == EINVAL


BACK = dict(codes=P, ldc=48, scale=P, rows=4, cols=33, block_rows=128, out=P, out_dtype=BF16, ldo=33, stream=None)


@pytest.mark.parametrize("bad", [dict(out_dtype=3), dict(rows=-1), dict(cols=0), dict(ldc=32), dict(ldo=32), dict(codes=None),
                                 dict(scale=None), dict(out=None), dict(out=P + 1), dict(scale=P + 2), dict(block_rows=127),
                                 dict(ldo=1 << 31)])
def test_dequantize_refuses(bad):
    assert _call(L.awsrc_dequantize_blocks_f8, BACK, **bad) == EINVAL


def test_no_rows():
    assert _call(L.awsrc_quantize_blocks_f8, QUANT, rows=0, X=None, codes=None, scale=None) == OK
    assert _call(L.awsrc_dequantize_blocks_f8, BACK, rows=0, codes=None, scale=None, out=None) == OK


MATMUL = dict(A=P, lda=48, a_scale=P, B=P, ldb=48, b_scale=P, bias=None, M=3, N=5, K=33, out=P, out_dtype=BF16, ldo=5, ws=P,
              n=None, stream=None)
LINEAR = dict(X=P, x_dtype=BF16, ldx=33, B=P, ldb=48, b_scale=P, bias=None, M=3, N=5, K=33, out=P, out_dtype=BF16, ldo=5, ws=P,
              n=None, stream=None)


@pytest.mark.parametrize("bad", [dict(out_dtype=7), dict(M=-1), dict(N=-1), dict(K=0), dict(K=(1 << 22) + 1, lda=1 << 23, ldb=1 << 23),
                                 dict(lda=40), dict(ldb=40), dict(lda=32), dict(ldb=32), dict(ldo=4), dict(A=P + 8),
                                 dict(B=P + 8), dict(out=P + 1), dict(A=None), dict(B=None), dict(a_scale=None),
                                 dict(b_scale=None), dict(out=None), dict(bias=P + 2), dict(b_scale=P + 1), dict(a_scale=P + 1),
                                 dict(lda=(1 << 22) + 16), dict(M=1 << 31), dict(N=1 << 31, ldo=1 << 31)])
def test_matmul_refuses(bad):
    assert _call(L.awsrc_matmul_f8, {**MATMUL, "n": _ws(1 << 40)}, **bad) == EINVAL


@pytest.mark.parametrize("bad", [dict(out_dtype=7), dict(x_dtype=5), dict(M=-1), dict(K=0), dict(ldx=32), dict(ldb=40), dict(ldo=4),
                                 dict(X=P + 1), dict(B=P + 8), dict(X=None), dict(B=None), dict(b_scale=None), dict(out=None),
                                 dict(bias=P + 2)])
def test_linear_refuses(bad):
    assert _call(L.awsrc_linear_f8, {**LINEAR, "n": _ws(1 << 40)}, **bad) == EINVAL


def test_products_need_ws_bytes():
    assert _call(L.awsrc_matmul_f8, MATMUL) == EINVAL
    assert _call(L.awsrc_linear_f8, LINEAR) == EINVAL


def test_product_workspaces():
    n = ctypes.c_size_t(0)
    for M, N, K in ((17, 5, 33), (200, 500, 1000), (3, 9000, 33), (16, 64, 40000), (64, 2048, 11008), (1, 100, 60000)):
        shape = dict(M=M, N=N, K=K, ldx=K, ldb=-(-K // 16) * 16, ldo=N)
        query = dict(X=None, B=None, b_scale=None, out=None, ws=None)
        assert _call(L.awsrc_linear_f8, {**LINEAR, "n": ctypes.byref(n)}, **query, **shape) == OK
        assert awsrc.linear_f8_workspace_bytes(M, N, K) == n.value
        if n.value:
            assert _call(L.awsrc_linear_f8, {**LINEAR, "n": _ws(n.value - 1)}, **shape) == ENOSPC
            assert _call(L.awsrc_linear_f8, {**LINEAR, "n": _ws(n.value)}, ws=None, **shape) == ENOSPC
            assert _call(L.awsrc_linear_f8, {**LINEAR, "n": _ws(n.value)}, ws=P + 8, **shape) == EINVAL
        ld = -(-K // 16) * 16
        query = dict(A=None, a_scale=None, B=None, b_scale=None, out=None, ws=None)
        assert _call(L.awsrc_matmul_f8, {**MATMUL, "n": ctypes.byref(n)}, M=M, N=N, K=K, lda=ld, ldb=ld, ldo=N, **query) == OK
        assert awsrc.matmul_f8_workspace_bytes(M, N, K) == n.value
        if n.value:
            assert _call(L.awsrc_matmul_f8, {**MATMUL, "n": _ws(n.value - 1)}, M=M, N=N, K=K, lda=ld, ldb=ld, ldo=N) == ENOSPC
    for empty in (dict(M=0), dict(N=0, ldo=0)):
        assert _call(L.awsrc_matmul_f8, {**MATMUL, "n": _ws(0)}, **empty) == OK
        assert _call(L.awsrc_linear_f8, {**LINEAR, "n": _ws(0)}, **empty) == OK


def _pool(**bad):
    c = dict(free_pages=P, n_free=P, n_pages=10, page_tokens=64, reserved=0)
    c.update(bad)
    return ctypes.byref(awsrc.awsrc_page_pool(*c.values()))


PLAN = dict(pool=None, n_seq=3, kv_len=P, keep=P, new_len=P, table=P, table_ld=4, max_rows=9, kv_out=P, n_free_out=P, cu=P,
            seq=P, pos=P, slot=P, ws=P, n=None, stream=None)


@pytest.mark.parametrize("bad", [dict(n_pages=0), dict(n_pages=1 << 31), dict(page_tokens=8), dict(page_tokens=48), dict(page_tokens=0),
                                 dict(reserved=1), dict(free_pages=None), dict(n_free=None), dict(free_pages=P + 2), dict(n_free=P + 1)])
def test_plan_refuses_pools(bad):
    assert _call(L.awsrc_kv_plan, {**PLAN, "n": _ws(1 << 30)}, pool=_pool(**bad)) == EINVAL


@pytest.mark.parametrize("bad", [dict(pool=None), dict(n_seq=-1), dict(n_seq=(1 << 20) + 1), dict(table_ld=0), dict(table_ld=1 << 25),
                                 dict(n_seq=1 << 20, table_ld=1 << 11), dict(max_rows=-1), dict(max_rows=1 << 31), dict(kv_len=None),
                                 dict(keep=None), dict(new_len=None), dict(table=None), dict(kv_out=None), dict(n_free_out=None),
                                 dict(cu=None), dict(kv_len=P + 2), dict(keep=P + 1), dict(new_len=P + 2), dict(table=P + 2),
                                 dict(kv_out=P + 2), dict(n_free_out=P + 2), dict(cu=P + 2), dict(seq=P + 2), dict(pos=P + 1),
                                 dict(slot=P + 4), dict(n=None)])
def test_plan_refuses(bad):
    assert _call(L.awsrc_kv_plan, {**PLAN, "pool": _pool(), "n": _ws(1 << 40), **bad}) == EINVAL


def test_plan_workspace_and_nothing():
    n = ctypes.c_size_t(0)
    none = dict(kv_len=None, keep=None, new_len=None, table=None, kv_out=None, n_free_out=None, cu=None, seq=None, pos=None, slot=None, ws=None)
    for n_seq, rows in ((1, 100000), (5, 9), (300, 9), (2048, 8192), (2048, 8193), (3000, 0)):
        shape = dict(n_seq=n_seq, max_rows=rows)
        assert _call(L.awsrc_kv_plan, {**PLAN, "pool": _pool(), "n": ctypes.byref(n)}, **shape, **none) == OK
        assert n.value == awsrc.kv_plan_workspace_bytes(n_seq, rows)
        if n.value:
            assert _call(L.awsrc_kv_plan, {**PLAN, "pool": _pool(), "n": _ws(n.value - 1)}, **shape) == ENOSPC
            assert _call(L.awsrc_kv_plan, {**PLAN, "pool": _pool(), "n": _ws(n.value)}, ws=None, **shape) == ENOSPC
            assert _call(L.awsrc_kv_plan, {**PLAN, "pool": _pool(), "n": _ws(n.value)}, ws=P + 4, **shape) == EINVAL
    assert n.value > 0
    for missing in (dict(cu=None), dict(n_free_out=None)):  # without slots too
        assert _call(L.awsrc_kv_plan, {**PLAN, "pool": _pool(), "n": _ws(0)}, n_seq=0, **missing) == EINVAL
    assert _call(L.awsrc_kv_plan, {**PLAN, "pool": _pool(), "n": _ws(0)}, n_seq=0, max_rows=9000) == ENOSPC


VERIFY = dict(p=P, ldp=100, q=P, ldq=100, dtype=BF16, vocab=100, n_seq=3, n_rows=7, cu=P, tokens=P, u=P, kv_len=P, tokens_out=P, n_out=P,
              keep=P, ws=P, n=None, stream=None)


@pytest.mark.parametrize("bad", [dict(dtype=3), dict(dtype=-1), dict(vocab=0), dict(vocab=1 << 31), dict(n_seq=-1), dict(n_rows=-1),
                                 dict(n_rows=1 << 31), dict(ldp=99), dict(ldq=99), dict(p=None), dict(tokens=None), dict(u=None),
                                 dict(cu=None), dict(tokens_out=None), dict(n_out=None), dict(keep=None), dict(kv_len=None),
                                 dict(p=P + 1), dict(q=P + 1), dict(cu=P + 2), dict(tokens=P + 1), dict(u=P + 2), dict(kv_len=P + 2),
                                 dict(keep=P + 2), dict(tokens_out=P + 1), dict(n_out=P + 2), dict(n=None), dict(n_seq=(1 << 24) + 1)])
def test_verify_refuses(bad):
    assert _call(L.awsrc_verify_drafts, {**VERIFY, "n": _ws(1 << 40), **bad}) == EINVAL


def test_verify_workspace_and_nothing():
    n = ctypes.c_size_t(0)
    none = dict(p=None, q=None, cu=None, tokens=None, u=None, kv_len=None, tokens_out=None, n_out=None, keep=None, ws=None)
    for n_seq, vocab in ((1, 1), (3, 100), (3, 65537), (257, 65537), (3, 131073), (64, 262144)):
        shape = dict(n_seq=n_seq, vocab=vocab, ldp=vocab, ldq=vocab)
        assert _call(L.awsrc_verify_drafts, {**VERIFY, "n": ctypes.byref(n)}, **shape, **none) == OK
        assert n.value == awsrc.verify_drafts_workspace_bytes(n_seq, vocab)
        if n.value:
            assert _call(L.awsrc_verify_drafts, {**VERIFY, "n": _ws(n.value - 1)}, **shape) == ENOSPC
            assert _call(L.awsrc_verify_drafts, {**VERIFY, "n": _ws(n.value)}, ws=P + 8, **shape) == EINVAL
    assert n.value > 0
    assert _call(L.awsrc_verify_drafts, {**VERIFY, "n": _ws(0)}, n_seq=0) == OK


# ------------------------------------------------------------------ the binding
def test_binding_refuses():
    f8 = torch.zeros(4, 32, dtype=torch.uint8).view(F8)
    with pytest.raises(ValueError):  # not on a device
        awsrc.awsrc_quantize_blocks_f8(torch.zeros(3, 5))
    with pytest.raises(TypeError):
        awsrc.awsrc_matmul_f8(torch.zeros(4, 32, dtype=torch.int8), torch.zeros(1, 4), f8, torch.zeros(1, 1))
    with pytest.raises(TypeError):
        awsrc.awsrc_linear_f8(torch.zeros(4, 32), torch.zeros(4, 32, dtype=torch.int8), torch.zeros(1, 1))
    with pytest.raises(TypeError):
        awsrc.awsrc_dequantize_blocks_f8(torch.zeros(4, 32, dtype=torch.uint8), torch.zeros(1, 4))
    with pytest.raises(ValueError):
        awsrc.awsrc_linear_f8(torch.zeros(4, 31), f8, torch.zeros(1, 1))
    one = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        awsrc.awsrc_kv_plan((one, one), one, one, one, torch.zeros(1, 2, dtype=torch.int32), 16, 4)
    with pytest.raises(ValueError):
        awsrc.awsrc_verify_drafts(torch.zeros(1, 4), one, torch.zeros(1), torch.zeros(2, dtype=torch.int32))
