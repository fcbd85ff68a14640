"""Steps with drafted tokens on the GPU: the plan of pages and rows against
Python lists, the verification against its definition in 64 bits; all whole
numbers, all equal."""
import numpy as np
import pytest
import torch

import drafts_ref as R

pytestmark = pytest.mark.gpu

awsrc = pytest.importorskip("paper_2608_23144_amd")

DEV = "cuda"
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def _ints(v):
    return torch.tensor(np.asarray(v, np.int32), device=DEV)


# ------------------------------------------------------------------ plans
class Server:
    """Pools and tables on the device beside the lists of the reference."""

    def __init__(self, rng, n_seq, page, width, n_pages):
        self.rng, self.page, self.n_pages = rng, page, n_pages
        order = rng.permutation(n_pages).tolist()
        self.free = order
        self.pool = (_ints(order), _ints([n_pages]))
        self.kv = np.zeros(n_seq, np.int32)
        self.table = np.full((n_seq, width), -1, np.int32)
        self.d_table, self.d_kv = _ints(self.table), _ints(self.kv)

    def step(self, keep, new, rows, **given):
        got = awsrc.awsrc_kv_plan(self.pool, self.d_kv, _ints(keep), _ints(new), self.d_table, self.page, rows, **given)
        want = R.plan(self.page, self.n_pages, self.free, self.kv.tolist(), list(map(int, keep)), list(map(int, new)), self.table, rows)
        for t, name in zip(got, ("cu", "seq", "pos", "slot")):
            assert np.array_equal(t.cpu().numpy(), want[name]), name
        self.kv, self.free = want["kv"], want["free"]
        assert np.array_equal(self.d_kv.cpu().numpy(), self.kv)
        assert np.array_equal(self.d_table.cpu().numpy(), self.table)
        assert self.pool[1].item() == len(self.free)
        assert np.array_equal(self.pool[0].cpu().numpy()[:len(self.free)], self.free)
        return want

    def held(self):
        return [self.table[s, i] for s, n in enumerate(self.kv) for i in range(-(-n // self.page))]


@pytest.mark.parametrize("n_seq,page,width,n_pages", [(1, 16, 5, 4), (3, 16, 9, 40), (17, 32, 12, 60), (64, 64, 40, 900), (65, 128, 20, 300),
                                                      (1024, 16, 30, 9000), (1025, 16, 30, 5000), (3000, 16, 8, 9000)])
def test_plan_over_many_steps(n_seq, page, width, n_pages):
    """Prompts, drafts of which some are refused, sequences that end and start, more asked for than there is: every
    step as on lists, and at every step each page is held once or free."""
    rng = np.random.default_rng(n_seq * 1000 + page)
    server = Server(rng, n_seq, page, width, n_pages)
    served = refused = 0
    for i in range(8):
        kv = server.kv
        keep = np.maximum(0, kv - rng.integers(0, 9, n_seq)) * (rng.random(n_seq) > 0.15)
        new = np.where(rng.random(n_seq) < 0.7, rng.integers(0, 10, n_seq), rng.integers(0, page * width // 2, n_seq))
        rows = int(new.sum()) + int(rng.integers(-3, 4)) if i % 3 else int(new.sum() * 0.8)
        want = server.step(keep, new, max(0, rows))
        got = np.diff(want["cu"])
        served, refused = served + int((got > 0).sum()), refused + int(((got == 0) & (new > 0)).sum())
        assert sorted(server.held() + server.free) == list(range(n_pages))
    assert served and (refused or n_seq == 3)


@pytest.mark.parametrize("n_seq,rows", [(100, 1024), (100, 1025), (256, 1000), (256, 8192), (256, 8193), (257, 300), (1000, 8000), (1024, 5000),
                                        (1025, 1500), (2047, 8192), (2048, 8192), (2048, 8193), (2049, 4000)])
def test_plan_of_decode_steps(n_seq, rows):
    """Every sequence at work with about as many rows as there is room for: both sides of the bounds between launches."""
    rng = np.random.default_rng(n_seq + rows)
    server = Server(rng, n_seq, 32, 12, n_seq * 6)
    most = 2 * rows // n_seq + 1
    for i in range(5):
        keep = np.maximum(0, server.kv - rng.integers(0, 5, n_seq)) * (rng.random(n_seq) > 0.1)
        server.step(keep, rng.integers(0, most, n_seq), rows)
        assert sorted(server.held() + server.free) == list(range(n_seq * 6))


def test_plan_longer_than_the_pool_and_the_table():
    """A slot that is not served gives up what it does not keep; slots after it that need no page are served."""
    rng = np.random.default_rng(5)
    s = Server(rng, 4, 16, 6, 12)
    s.step([0, 0, 0, 0], [40, 16, 17, 5], 100)  # 3 + 1 + 2 + 1 pages
    want = s.step([40, 16, 17, 5], [100, 1, 1, 1], 200)  # the first is longer than its table's row
    assert np.diff(want["cu"]).tolist() == [0, 0, 1, 1]  # (the pages that it asks for count for those after it)
    want = s.step([1, 16, 18, 6], [90, 60, 1, 0], 200)  # the first two ask for 3 + 4 pages, 5 are free
    assert np.diff(want["cu"]).tolist() == [90, 0, 1, 0]
    want = s.step([0, 0, 0, 0], [0, 0, 0, 0], 3)
    assert want["cu"].tolist() == [0] * 5 and len(s.free) == 12 and (want["slot"] == -1).all()


def test_plan_there_and_back_leaves_everything_as_it_was():
    rng = np.random.default_rng(7)
    s = Server(rng, 40, 16, 30, 700)
    s.step(np.zeros(40, int), rng.integers(0, 300, 40), 20000)
    free, kv = list(s.free), s.kv.copy()
    held = s.held()
    s.step(kv, rng.integers(0, 100, 40), 9000)
    s.step(kv, np.zeros(40, int), 0)
    assert s.free == free and np.array_equal(s.kv, kv) and s.held() == held


def test_plan_into_other_buffers_repeats_itself():
    """kv_len_out and n_free_out given: the inputs stay, and the same call gives the same again, whatever the workspace held."""
    rng = np.random.default_rng(9)
    n, page, width, n_pages = 300, 32, 20, 3000
    kv = rng.integers(0, 400, n)
    keep = np.maximum(0, kv - rng.integers(0, 60, n))
    new = rng.integers(0, 200, n)
    order = rng.permutation(n_pages)
    held = -(-kv // page)
    table = np.full((n, width), -1)
    at = 0
    for s in range(n):
        table[s, :held[s]] = order[at:at + held[s]]
        at += held[s]
    free = np.full(n_pages, -5)
    free[:n_pages - at] = order[at:]
    d = {k: _ints(v) for k, v in (("kv", kv), ("keep", keep), ("new", new), ("table", table), ("free", free), ("n", [n_pages - at]))}
    rows = int(new.sum()) + 5
    want = R.plan(page, n_pages, free[:n_pages - at].tolist(), kv.tolist(), keep.tolist(), new.tolist(), table.astype(np.int32), rows)
    need = awsrc.kv_plan_workspace_bytes(n, rows)
    scratch = torch.empty(need + 64, dtype=torch.uint8, device=DEV)
    for value in (0, 255, 90):
        scratch.fill_(value)
        kv_out, n_out = torch.empty_like(d["kv"]), torch.empty_like(d["n"])
        got = awsrc.awsrc_kv_plan((d["free"], d["n"]), d["kv"], d["keep"], d["new"], d["table"], page, rows, kv_len_out=kv_out,
                                  n_free_out=n_out, workspace=scratch[:need])
        assert (scratch[need:] == value).all()
        for t, name in zip(got, ("cu", "seq", "pos", "slot")):
            assert np.array_equal(t.cpu().numpy(), want[name]), name
        assert np.array_equal(kv_out.cpu().numpy(), want["kv"]) and n_out.item() == len(want["free"])
        assert np.array_equal(d["table"].cpu().numpy(), want["table"])
        assert np.array_equal(d["free"].cpu().numpy()[:len(want["free"])], want["free"])
        assert np.array_equal(d["kv"].cpu().numpy(), kv) and d["n"].item() == n_pages - at


def test_plan_of_lengths_that_cannot_be():
    """Negative and huge lengths, pages that are not there, a pool that counts too many: nothing outside is touched, and
    what is written is what the definition says."""
    page, width, n_pages = 16, 4, 10
    big = 2 ** 31 - 1
    kv, keep, new = [-5, 1000, big, 10, 3, 16], [-1, 64, big, 20, -7, 16], [-3, 0, 1, big, 2, 1]
    table = np.array([[900, -900, big, 3]] * 6, np.int32)
    for count in (-4, 0, 3, 10, 11, big):
        guard = torch.full((n_pages + 64,), 55, dtype=torch.int32, device=DEV)
        free = guard[32:32 + n_pages]
        free.copy_(torch.arange(n_pages))
        t_guard = torch.full((8, width), 66, dtype=torch.int32, device=DEV)
        d_table = t_guard[1:7]
        d_table.copy_(torch.from_numpy(table))
        d_kv, n_free = _ints(kv), _ints([count])
        cu, seq, pos, slot = awsrc.awsrc_kv_plan((free, n_free), d_kv, _ints(keep), _ints(new), d_table, page, 30)
        have = list(range(min(max(count, 0), n_pages)))
        want = R.plan(page, n_pages, have, kv, keep, new, table.copy(), 30)
        assert np.array_equal(cu.cpu().numpy(), want["cu"])
        assert np.array_equal(pos.cpu().numpy(), want["pos"]) and np.array_equal(seq.cpu().numpy(), want["seq"])
        assert np.array_equal(slot.cpu().numpy(), want["slot"])
        assert np.array_equal(d_table.cpu().numpy(), want["table"])
        assert n_free.item() == min(len(want["free"]), n_pages)
        assert (guard[:32] == 55).all() and (guard[32 + n_pages:] == 55).all() and (t_guard[[0, 7]] == 66).all()


def test_plan_captured_and_replayed():
    """A decode step's plan in a graph, in place: lengths change from replay to replay."""
    rng = np.random.default_rng(11)
    n, page = 50, 16
    s = Server(rng, n, page, 40, 1500)
    s.step(np.zeros(n, int), rng.integers(1, 200, n), 20000)
    keep, new = _ints(np.zeros(n)), _ints(np.zeros(n))
    out = tuple(torch.empty(k, dtype=t, device=DEV) for k, t in ((n + 1, torch.int32), (300, torch.int32), (300, torch.int32), (300, torch.int64)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        awsrc.awsrc_kv_plan(s.pool, s.d_kv, keep, new, s.d_table, page, 300, out=out)
    for i in range(5):
        k, m = s.kv - rng.integers(0, 5, n), rng.integers(0, 6, n)
        k = np.maximum(k, 0) * (rng.random(n) > 0.1)
        keep.copy_(_ints(k))
        new.copy_(_ints(m))
        graph.replay()
        want = R.plan(page, s.n_pages, s.free, s.kv.tolist(), k.tolist(), m.tolist(), s.table, 300)
        for t, name in zip(out, ("cu", "seq", "pos", "slot")):
            assert np.array_equal(t.cpu().numpy(), want[name]), name
        s.kv, s.free = want["kv"], want["free"]
        assert s.pool[1].item() == len(s.free) and np.array_equal(s.d_table.cpu().numpy(), s.table)


def test_plan_of_nothing():
    pool = awsrc.make_page_pool(4, DEV)
    none = _ints([])
    for rows in (0, 1, 7, 5003, 9001):
        left = _ints([-1])
        filled = (_ints([9]), _ints([9] * rows), _ints([9] * rows), _ints([9] * rows).long())
        cu, *of_rows = awsrc.awsrc_kv_plan(pool, none, none, none, torch.empty(0, 3, dtype=torch.int32, device=DEV), 16, rows,
                                           n_free_out=left, out=filled)
        assert cu.tolist() == [0] and left.item() == 4 and all((t == -1).all() for t in of_rows)
    assert pool[1].item() == 4 and pool[0].tolist() == [3, 2, 1, 0]
    cu, seq, pos, slot = awsrc.awsrc_kv_plan(pool, _ints([0]), _ints([0]), _ints([0]), _ints([[0, 0, 0]]), 16, 0)
    assert cu.tolist() == [0, 0] and seq.numel() == 0


# ------------------------------------------------------------------ drafts
def _case(rng, counts, V, dtype, with_q, agree=0.7):
    n = sum(counts)
    logits = 2.5 * rng.standard_normal((n, V))
    p = np.exp(logits - logits.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    guess = np.exp(logits + 0.6 * rng.standard_normal((n, V)))
    guess /= guess.sum(1, keepdims=True)
    tokens = rng.integers(0, V, n)
    for r in range(n - 1):
        if rng.random() < agree:
            tokens[r + 1] = int(np.argmax(p[r]))
    as_t = lambda x: torch.from_numpy(x).to(dtype)
    return as_t(p), (as_t(guess) if with_q else None), tokens.astype(np.int32), rng.random(n).astype(np.float32)


def _verify(p, q, tokens, u, cu, **given):
    d = None if q is None else q.to(DEV)
    return awsrc.awsrc_verify_drafts(p.to(DEV), _ints(tokens), torch.from_numpy(u).to(DEV), _ints(cu), q=d, **given)


def _check(p, q, tokens, u, cu):
    kv = np.arange(len(cu) - 1) * 3 + 50
    out, n, keep = _verify(p, q, tokens, u, cu, kv_len=_ints(kv))
    want, count = R.verify(p.float().numpy(), None if q is None else q.float().numpy(), tokens, u, cu)
    assert np.array_equal(n.cpu().numpy(), count)
    end = cu[-1]
    assert np.array_equal(out.cpu().numpy()[:end], want[:end])
    assert np.array_equal(keep.cpu().numpy(), kv - np.diff(cu) + count)
    here, same = _ints(tokens), _ints(kv)  # over the tokens, and over the lengths
    awsrc.awsrc_verify_drafts(p.to(DEV), here, torch.from_numpy(u).to(DEV), _ints(cu), q=None if q is None else q.to(DEV),
                              kv_len=same, keep=same, out=(here, torch.empty_like(n)))
    assert torch.equal(here[:end], out[:end]) and torch.equal(same, keep)
    return want, count


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("with_q", [True, False])
@pytest.mark.parametrize("V", [1, 2, 7, 255, 2047, 2049, 8191, 8193, 33001, 65536, 65537, 70001, 131072, 131073, 270001])
def test_verify(V, with_q, dtype):
    rng = np.random.default_rng(V + with_q)
    counts = [1, 5, 0, 2, 9, 1, 3, 0]
    for i in range(3):
        case = _case(rng, counts, V, dtype, with_q)
        _check(*case, np.concatenate([[0], np.cumsum(counts)]))


@pytest.mark.parametrize("with_q", [True, False])
@pytest.mark.parametrize("V,more", [(50, 300), (65600, 5)])
def test_verify_many_sequences_and_long_drafts(V, more, with_q):
    """More drafts than a wavefront has lanes, sequences beyond a workgroup's threads."""
    rng = np.random.default_rng(3)
    counts = [200, 65, 66, 1] + [int(c) for c in rng.integers(0, 5, more)]
    p, q, tokens, u = _case(rng, counts, V, torch.float32, with_q, agree=1.0)
    u[:330] *= 0.01  # long runs of accepted drafts
    _, count = _check(p, q, tokens, u, np.concatenate([[0], np.cumsum(counts)]))
    assert count[0] > 64


def test_verify_borders_of_the_random_numbers():
    """u of 0, just below 1, on a border between tokens, 1 and NaN; exact ties are refused."""
    p = torch.tensor([[0.25, 0.0, 0.5, 0.25, 0.0]] * 2)
    q = torch.tensor([[0.5, 0.0, 0.25, 0.25, 0.0]] * 2)
    for u0, x, u1 in ((0.5, 0, 0.0), (0.4999999, 0, 0.0), (0.0, 1, 0.3), (0.9999999, 2, 0.0), (0.5, 1, 0.9999999), (0.0, 0, 0.25),
                      (0.0, 0, 0.75), (0.0, 0, 0.7499999), (0.0, 0, 1.0), (0.0, 0, float("nan")), (float("nan"), 2, 0.1), (0.0, 4, -1.0)):
        _check(p, q, np.array([3, x], np.int32), np.array([u0, u1], np.float32), np.array([0, 2]))
    out, n, _ = _verify(p, q, np.array([3, 0], np.int32), np.array([0.5, 0.0], np.float32), np.array([0, 2]))
    assert out.tolist() == [2, -1] and n.tolist() == [1]  # 0.5 * 0.5 < 0.25 does not hold; only token 2 has weight


@pytest.mark.parametrize("with_q", [True, False])
@pytest.mark.parametrize("V", [700, 3000, 66001])
def test_verify_values_that_cannot_be(V, with_q):
    """NaN and infinite probabilities, negative ones, drafts outside the vocabulary, rows of zeros."""
    rng = np.random.default_rng(1)
    counts = [4] * 12
    p, q, tokens, u = _case(rng, counts, V, torch.float32, with_q, agree=0.5)
    bad = [float("nan"), float("inf"), -float("inf"), -0.5]
    for r in range(len(tokens)):
        p[r, rng.integers(0, V, 40)] = bad[r % 4]
        if q is not None:
            q[r, rng.integers(0, V, 40)] = bad[(r + 1) % 4]
    tokens[[1, 5, 9, 14]] = [V, -1, 2 ** 31 - 1, -2 ** 31]
    p[20:24] = 0
    if q is not None:
        q[24:28] = p[24:28].nan_to_num(0, 0, 0) * 2  # nothing of p lies above q
        tokens[25] = 2 ** 30
    p[28:32] = float("nan")
    want, _ = _check(p, q, tokens, u, np.concatenate([[0], np.cumsum(counts)]))
    assert (want[20] == -1) and (want[28] == -1) and want[24] >= 0


def test_verify_rows_of_wider_buffers():
    """Rows at odd places, rows behind the last sequence, starts that point outside: nothing else is written."""
    rng = np.random.default_rng(8)
    counts, V = [3, 1, 4], 501
    p, q, tokens, u = _case(rng, counts + [5], V, torch.bfloat16, True)
    n = len(tokens)
    wide_p, wide_q = torch.full((n, V + 9), float("nan"), dtype=torch.bfloat16), torch.full((n, V + 4), float("nan"), dtype=torch.bfloat16)
    wide_p[:, 3:3 + V], wide_q[:, 1:1 + V] = p, q
    cu = np.array([0, 3, 4, 8])
    out = (torch.full((n,), 99, dtype=torch.int32, device=DEV), torch.full((3,), 99, dtype=torch.int32, device=DEV))
    awsrc.awsrc_verify_drafts(wide_p.to(DEV)[:, 3:3 + V], _ints(tokens), torch.from_numpy(u).to(DEV), _ints(cu),
                              q=wide_q.to(DEV)[:, 1:1 + V], out=out)
    want, count = R.verify(p.float().numpy(), q.float().numpy(), tokens, u, cu)
    assert np.array_equal(out[0].cpu().numpy()[:8], want[:8]) and (out[0][8:] == 99).all()
    assert np.array_equal(out[1].cpu().numpy(), count)
    for strange in ([-7, 3, 1, 10 ** 6], [5, 2, 13, 4], [14, 15, 16, 17]):
        got, k, _ = awsrc.awsrc_verify_drafts(p.to(DEV), _ints(tokens), torch.from_numpy(u).to(DEV), _ints(strange), q=q.to(DEV))
        rows = np.diff(np.clip(strange, 0, n))
        assert ((k.cpu().numpy() <= np.maximum(rows, 0)) & (k.cpu().numpy() >= (rows > 0))).all()


def test_verify_follows_the_targets_distribution():
    """One draft drawn from q, verified: what comes out is distributed as p (6 deviations of a binomial, 300,000 draws)."""
    n, V = 300000, 6
    g = torch.Generator(device=DEV)
    g.manual_seed(4)
    p = torch.tensor([0.4, 0.05, 0.25, 0.0, 0.2, 0.1], device=DEV)
    q = torch.tensor([0.1, 0.3, 0.2, 0.15, 0.25, 0.0], device=DEV)
    tokens = torch.zeros(2 * n, dtype=torch.int32, device=DEV)
    tokens[1::2] = torch.multinomial(q, n, replacement=True, generator=g).int()
    out, count, _ = awsrc.awsrc_verify_drafts(p.expand(2 * n, V).contiguous(), tokens, torch.rand(2 * n, generator=g, device=DEV),
                                              torch.arange(0, 2 * n + 1, 2, device=DEV).int(), q=q.expand(2 * n, V).contiguous())
    first = torch.bincount(out[::2].long(), minlength=V).double() / n
    assert ((first - p.double()).abs() <= 6 * (p.double() * (1 - p.double()) / n).sqrt()).all()
    assert abs((count == 2).double().mean().item() - float(torch.minimum(p, q).sum())) < 6 * 0.5 / n ** 0.5
    second = torch.bincount(out[1::2][count == 2].long(), minlength=V).double() / int((count == 2).sum())
    assert ((second - p.double()).abs() <= 6 * (p.double() * (1 - p.double()) / int((count == 2).sum())).sqrt()).all()


@pytest.mark.parametrize("V", [9001, 140003])
def test_verify_repeats_itself_and_can_be_captured(V):
    rng = np.random.default_rng(2)
    counts = [5, 1, 3, 4]
    cu = _ints(np.concatenate([[0], np.cumsum(counts)]))
    p, q, tokens, u = _case(rng, counts, V, torch.float16, True)
    p, q, tokens, u = p.to(DEV), q.to(DEV), _ints(tokens), torch.from_numpy(u).to(DEV)
    need = awsrc.verify_drafts_workspace_bytes(4, V)
    scratch = torch.empty(need + 64, dtype=torch.uint8, device=DEV)
    first = awsrc.awsrc_verify_drafts(p, tokens, u, cu, q=q)
    for value in (0, 255):
        scratch.fill_(value)
        again = awsrc.awsrc_verify_drafts(p, tokens, u, cu, q=q, workspace=scratch[:need] if need else None)
        assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1]) and (scratch[need:] == value).all()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = awsrc.awsrc_verify_drafts(p, tokens, u, cu, q=q, stream=side)
    side.synchronize()
    assert torch.equal(other[0], first[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = awsrc.awsrc_verify_drafts(p, tokens, u, cu, q=q)
    for i in range(4):
        a = _case(rng, counts, V, torch.float16, True)
        for into, x in zip((p, q, tokens, u), (a[0], a[1], torch.from_numpy(a[2]), torch.from_numpy(a[3]))):
            into.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        want, count = R.verify(a[0].float().numpy(), a[1].float().numpy(), a[2], a[3], np.concatenate([[0], np.cumsum(counts)]))
        assert np.array_equal(held[0].cpu().numpy(), want) and np.array_equal(held[1].cpu().numpy(), count)


def test_verify_rows_past_2_32_elements():
    """Probabilities whose last rows start beyond 2^32 elements."""
    V, n = 1 << 26, 70
    p = torch.zeros(n, V, dtype=torch.float16, device=DEV)
    tokens = torch.zeros(n, dtype=torch.int32, device=DEV)
    p[-2, 5], p[-1, V - 1], p[-1, 3] = 1.0, 0.5, 0.25
    tokens[-1] = 5
    u = torch.full((n,), 0.9, device=DEV)
    out, count, _ = awsrc.awsrc_verify_drafts(p, tokens, u, _ints([n - 2, n]))
    assert out[-2:].tolist() == [5, V - 1] and count.tolist() == [2]


def test_verify_nothing():
    p = torch.empty(0, 10, device=DEV)
    none = _ints([])
    out, n, keep = awsrc.awsrc_verify_drafts(p, none, torch.empty(0, device=DEV), _ints([0, 0, 0]), kv_len=_ints([4, 0]))
    assert n.tolist() == [0, 0] and keep.tolist() == [4, 0] and out.numel() == 0
    out, n, keep = awsrc.awsrc_verify_drafts(p, none, torch.empty(0, device=DEV), _ints([0]))
    assert n.numel() == 0
