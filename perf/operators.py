"""The measured work of the 8-bit serving operators: what one pass of each case does, on which inputs, and what it has to give.

A case is a dict of plain values.  Its kind names the operator:

  linear      activations quantized to int8 per row, times an int8 weight matrix with one scale per output channel
  append      new keys and values rotated by position and quantized into a paged int8 cache (queries rotated on
              the way), and the touched blocks read back as the values that they stand for
  attention   ragged batches of queries over that cache, one scale for each page and head, grouped heads

A batch holds `seqs` sequences.  The longest has `kv` cached tokens after the call, of which the last `new` are this
call's; the others are spread evenly between a quarter of that and all of it.  The arithmetic of the 8-bit
recipe is fp32, each operation rounded once:
  scale = amax / 127, inverse = 1 / scale, code = rint(x * inverse) in [-127, 127].
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
HEADS = {"3b": (16, 2, 128), "32b": (40, 8, 128), "mha64": (12, 12, 64), "gqa256": (8, 4, 256)}  # query heads, cached heads, head width
ROPE_BASE = 1e6
TINY = 2.0 ** -100  # a block or row whose largest magnitude is below this is stored as zeros


def listed():
    return [
        # one token through the fused q, k, v projection of a 3B layer: launches and latency
        {"name": "linear_qkv3b_m1", "kind": "linear", "M": 1, "N": 2560, "K": 2048, "x": "bf16", "out": "bf16", "bias": True},
        # a decode step of 13 sequences through the 3B down projection: few rows, a long sum
        {"name": "linear_down3b_m13", "kind": "linear", "M": 13, "N": 2048, "K": 11008, "x": "f16", "out": "f16", "bias": False},
        # a decode step of 64 sequences through the 32B gate projection: the weights' bytes
        {"name": "linear_gate32b_m64", "kind": "linear", "M": 64, "N": 27648, "K": 5120, "x": "bf16", "out": "bf16", "bias": False},
        # sizes that divide by nothing, from fp32 into fp32
        {"name": "linear_odd", "kind": "linear", "M": 517, "N": 1003, "K": 1337, "x": "f32", "out": "f32", "bias": True},
        # a prompt of 8192 tokens through the 32B gate projection: the matrix cores
        {"name": "linear_gate32b_m8192", "kind": "linear", "M": 8192, "N": 27648, "K": 5120, "x": "bf16", "out": "bf16", "bias": False},
        # one decode step of 48 sequences of a 3B layer
        {"name": "append_step3b", "kind": "append", "heads": "3b", "page": 64, "seqs": 48, "new": 1, "kv": 4099, "x": "bf16", "fresh": False},
        # three prompts of a 32B layer written into an empty cache
        {"name": "append_prompt32b", "kind": "append", "heads": "32b", "page": 64, "seqs": 3, "new": 4001, "kv": 4001, "x": "bf16", "fresh": True},
        # one short conversation, one token: the smallest call
        {"name": "attention_one3b", "kind": "attention", "heads": "3b", "page": 16, "seqs": 1, "new": 1, "kv": 1501, "x": "bf16", "fresh": False},
        # a decode step over a ragged batch of a 32B layer: the cache's bytes
        {"name": "attention_batch32b", "kind": "attention", "heads": "32b", "page": 64, "seqs": 64, "new": 1, "kv": 8192, "x": "bf16", "fresh": False},
        # two long documents, one token each, few heads: the axis has to be split
        {"name": "attention_long3b", "kind": "attention", "heads": "3b", "page": 64, "seqs": 2, "new": 1, "kv": 131071, "x": "bf16", "fresh": False},
        # a prompt of 8192 tokens of a 3B layer: the matrix cores and the exponentials
        {"name": "attention_prompt3b", "kind": "attention", "heads": "3b", "page": 64, "seqs": 1, "new": 8192, "kv": 8192, "x": "bf16", "fresh": True},
        # ragged pieces of prompts against longer histories, ungrouped narrow heads, fp16
        {"name": "attention_chunks64", "kind": "attention", "heads": "mha64", "page": 32, "seqs": 7, "new": 601, "kv": 6007, "x": "f16", "fresh": False},
    ]


def _log(rng, lo, hi):
    n = max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))
    return n + 1 if n == 3072 else n


def draw(rng):
    kind = rng.choice(["linear", "append", "attention", "attention"])
    if kind == "linear":
        case = {"kind": kind, "M": _log(rng, 1, 8192), "N": _log(rng, 64, 27648), "K": _log(rng, 64, 11008),
                "x": rng.choice(["bf16", "f16", "f32"]), "bias": rng.random() < 0.5}
        case["out"] = "f32" if case["x"] == "f32" else case["x"]
        if rng.random() < 0.6:  # most models' widths divide by 64
            case["N"], case["K"] = max(64, case["N"] // 64 * 64), max(64, case["K"] // 64 * 64)
        for n in ("N", "K"):  # no matrix of this repository has this width
            case[n] += 64 if case[n] == 3072 else 0
        return case
    case = {"kind": kind, "heads": rng.choice(sorted(HEADS)), "page": rng.choice([16, 32, 64]), "seqs": _log(rng, 1, 64),
            "new": 1 if rng.random() < 0.5 else _log(rng, 2, 4096), "kv": _log(rng, 1, 32768), "x": rng.choice(["bf16", "f16"])}
    case["fresh"] = case["new"] > 1 and rng.random() < 0.3
    hq, hk, d = HEADS[case["heads"]]
    if case["fresh"]:
        case["kv"] = case["new"]
    case["new"] = min(case["new"], case["kv"])
    while case["seqs"] > 1 and (case["seqs"] * hq * case["new"] * case["kv"] * max(1, d / 128) > 1e9 or case["seqs"] * case["kv"] * hk * d > 5e8):
        case["seqs"] = (case["seqs"] + 1) // 2
    while hq * case["new"] * case["kv"] * max(1, d / 128) > 1e9:
        case["new"] = (case["new"] + 1) // 2
        case["kv"] = case["new"] if case["fresh"] else case["kv"]
    if kind == "append":  # 4096 new tokens in all are a large step of a server
        while case["seqs"] > 1 and case["seqs"] * case["new"] > 12000:
            case["seqs"] = (case["seqs"] + 1) // 2
    return case


def _lengths(case):
    """(cached tokens after the call, new tokens) of each sequence."""
    kv, new = [], []
    for i in range(case["seqs"]):
        f = 1.0 if i == 0 else 0.25 + 0.75 * ((i * 0.6180339887) % 1.0)
        g = 1.0 if i == 0 else 0.25 + 0.75 * ((i * 0.4142135624) % 1.0)
        n = max(1, int(case["kv"] * f))
        kv.append(n)
        new.append(n if case["fresh"] else max(1, min(n, int(case["new"] * g))))
    return kv, new


def _starts(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 17)
    return g


def _channels(g, n, sigma):
    return torch.exp(sigma * torch.randn(n, generator=g, device=DEV))


def _pages(case, kv, g):
    """Page table of the batch: each sequence's pages anywhere in a pool with room to spare."""
    counts = [-(-n // case["page"]) for n in kv]
    pool = sum(counts) + 3
    order = torch.randperm(pool, generator=g, device=DEV)
    at = torch.tensor(_starts(counts)[:-1], device=DEV)
    width = max(counts)
    col = torch.arange(width, device=DEV)
    live = col < torch.tensor(counts, device=DEV)[:, None]
    return torch.where(live, order[(at[:, None] + col).clamp_max(pool - 1)], torch.zeros((), dtype=order.dtype, device=DEV)).int(), pool


def _blocks_of(x):
    """int8 codes and fp32 scales of [pages, heads, a, b] values, one scale for each page and head."""
    s = x.abs().amax((2, 3)) / 127
    return torch.round(x / s[:, :, None, None]).clamp_(-127, 127).to(torch.int8), s


def prepare(case, seed):
    g = _gen(seed)
    x_t = TYPES[case["x"]]
    if case["kind"] == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        # activations with a few loud channels, rows of different loudness
        x = torch.randn(M, K, generator=g, device=DEV) * _channels(g, K, 0.7) * _channels(g, M, 0.5)[:, None]
        ld = -(-K // 16) * 16  # rows of the weight matrix start at multiples of 16 bytes
        w = torch.zeros(N, ld, dtype=torch.int8, device=DEV)
        # codes of a normal weight row: its largest magnitude sits near four deviations
        for n0 in range(0, N, 4096):
            n1 = min(N, n0 + 4096)
            w[n0:n1, :K] = torch.round(torch.randn(n1 - n0, K, generator=g, device=DEV) * 32).clamp_(-127, 127).to(torch.int8)
        scale = 0.02 / 32 * _channels(g, N, 0.3)
        bias = torch.randn(N, generator=g, device=DEV) if case["bias"] else None
        return {"case": case, "x": x.to(x_t), "w": w[:, :K], "scale": scale, "bias": bias}
    hq, hk, d = HEADS[case["heads"]]
    kv, new = _lengths(case)
    table, pool = _pages(case, kv, g)
    T = case["page"]
    loud = _channels(g, hk * d, 0.6).view(1, hk, 1, d)
    k, v = torch.empty(pool, hk, T, d, dtype=torch.int8, device=DEV), torch.empty(pool, hk, d, T, dtype=torch.int8, device=DEV)
    ks, vs = torch.empty(pool, hk, device=DEV), torch.empty(pool, hk, device=DEV)
    step = max(1, (1 << 25) // (hk * T * d))
    for p in range(0, pool, step):
        n = min(step, pool - p)
        k[p:p + n], ks[p:p + n] = _blocks_of(torch.randn(n, hk, T, d, generator=g, device=DEV) * loud)
        v[p:p + n], vs[p:p + n] = _blocks_of(torch.randn(n, hk, d, T, generator=g, device=DEV) * _channels(g, n, 0.3)[:, None, None, None])
    st = {"case": case, "cache": (k, v, ks, vs), "table": table, "kv_len": torch.tensor(kv, dtype=torch.int32, device=DEV),
          "cu": torch.tensor(_starts(new), dtype=torch.int32, device=DEV), "max_new": max(new), "max_kv": max(kv)}
    n = sum(new)
    if case["kind"] == "attention":
        # scores of about two deviations: some tokens matter, none alone
        q = torch.randn(n, hq, d, generator=g, device=DEV)
        st["q"] = (q * 2 / loud.expand(1, hk, 1, d).pow(2).mean().sqrt()).to(x_t)
        return st
    # one row of the fused projection per token: queries, keys, values
    qkv = torch.randn(n, (hq + 2 * hk) * d, generator=g, device=DEV) * _channels(g, (hq + 2 * hk) * d, 0.5)
    st["qkv"] = qkv.to(x_t)
    angle = torch.arange(max(kv), device=DEV).double()[:, None] * ROPE_BASE ** (-torch.arange(0, d, 2, device=DEV).double() / d)
    st["cos"], st["sin"] = torch.cos(angle).float(), torch.sin(angle).float()
    # what is read back: the touched blocks, from each one's first token
    back = [n - (n - m) // T * T for n, m in zip(kv, new)]
    st["cu_back"] = torch.tensor(_starts(back), dtype=torch.int32, device=DEV)
    st["n_back"], st["max_back"] = sum(back), max(back)
    return st


# ------------------------------------------------------------------ the plain forms
def _div(a, b):
    """a / b, both tensors: one correctly rounded division (a Python number would become a product with its inverse)."""
    return torch.div(a, torch.as_tensor(b, dtype=a.dtype, device=a.device).expand_as(a))


def _scale_of(amax):
    return torch.where(amax < TINY, torch.zeros_like(amax), _div(amax, 127.0))


def _inverse(s):
    return torch.where(s > 0, _div(torch.ones_like(s), torch.where(s > 0, s, torch.ones_like(s))), torch.zeros_like(s))


def _plain_linear(st):
    x = st["x"].float()
    s = _scale_of(x.abs().amax(1))
    codes = torch.round(x * _inverse(s)[:, None])
    y = codes @ st["w"].float().T
    y = y * (s[:, None] * st["scale"][None, :])
    if st["bias"] is not None:
        y = y + st["bias"]
    return y.to(TYPES[st["case"]["out"]])


def _tokens(cu, kv_len, n):
    """Sequence and position of each of the last tokens that cu counts."""
    i = torch.arange(n, device=DEV)
    s = torch.searchsorted(cu[1:].long(), i, right=True)
    return s, kv_len.long()[s] - (cu.long()[s + 1] - i)


def _rotate(x, cos, sin):
    h = x.shape[-1] // 2
    a, b = x[..., :h], x[..., h:]
    c, s = cos[:, None, :], sin[:, None, :]
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def _plain_append(st):
    case = st["case"]
    hq, hk, d = HEADS[case["heads"]]
    T = case["page"]
    k, v, ks, vs = st["cache"]
    cu, kv_len, table = st["cu"], st["kv_len"].long(), st["table"].long()
    n = st["qkv"].shape[0]
    seq, pos = _tokens(cu, kv_len, n)
    page, slot = table[seq, pos // T], pos % T
    qkv = st["qkv"].float()
    c, s = st["cos"][pos], st["sin"][pos]
    q = _rotate(qkv[:, :hq * d].view(n, hq, d), c, s).to(st["qkv"].dtype)
    # the touched blocks, each sequence's padded by its last one
    new = (cu[1:] - cu[:-1]).long()
    first, last = (kv_len - new) // T, (kv_len - 1) // T
    width = (st["max_new"] + T - 2) // T + 1
    blocks = table.gather(1, torch.minimum(first[:, None] + torch.arange(width, device=DEV), last[:, None])).reshape(-1)
    fresh = torch.zeros(k.shape[0], dtype=torch.int32, device=DEV).scatter_reduce_(0, page, (slot == 0).int(), "amax")
    for x, codes, scales, turned in ((_rotate(qkv[:, hq * d:(hq + hk) * d].view(n, hk, d), c, s), k, ks, False),
                                     (qkv[:, (hq + hk) * d:].view(n, hk, d), v, vs, True)):
        amax = torch.zeros_like(scales).scatter_reduce_(0, page[:, None].expand(n, hk), x.abs().amax(-1), "amax")
        was = torch.where(fresh[:, None] > 0, torch.zeros_like(scales), scales)[blocks]
        now = torch.maximum(was, _scale_of(amax)[blocks])
        old = codes[blocks].float()
        ratio = (was * _inverse(now))[:, :, None, None]
        codes[blocks] = torch.where((now > was)[:, :, None, None], torch.round(old * ratio), old).to(torch.int8)
        scales[blocks] = now
        fine = torch.round(x * _inverse(scales[page])[:, :, None]).to(torch.int8)
        if turned:
            codes[page, :, :, slot] = fine
        else:
            codes[page, :, slot, :] = fine
    seq, pos = _tokens(st["cu_back"], kv_len, st["n_back"])
    page, slot = table[seq, pos // T], pos % T
    x_t = st["qkv"].dtype
    return {"q": q, "k": (k[page, :, slot].float() * ks[page][:, :, None]).to(x_t), "v": (v[page, :, :, slot].float() * vs[page][:, :, None]).to(x_t)}


def _rows(st, x_type):
    """Queries by sequence, padded, and which cached token each of them sees: [seqs, cached heads, group, new, kv]."""
    case = st["case"]
    hq, hk, d = HEADS[case["heads"]]
    cu, kv_len = st["cu"].long(), st["kv_len"].long()
    n, m, L = case["seqs"], st["max_new"], st["max_kv"]
    at = torch.arange(m, device=DEV)
    new = cu[1:] - cu[:-1]
    live = at < new[:, None]
    row = torch.where(live, cu[:-1, None] + at, torch.zeros_like(at))
    q = st["q"].to(x_type)[row].view(n, m, hk, hq // hk, d).permute(0, 2, 3, 1, 4)
    sees = torch.arange(L, device=DEV) <= (kv_len - new)[:, None, None] + at[:, None]
    return q, sees & live[:, :, None], live


def _plain_attention(st):
    case = st["case"]
    hq, hk, d = HEADS[case["heads"]]
    T, n = case["page"], case["seqs"]
    k, v, ks, vs = st["cache"]
    table, L, m = st["table"].long(), st["max_kv"], st["max_new"]
    kf = (k[table].float() * ks[table][..., None, None]).permute(0, 2, 1, 3, 4).reshape(n, hk, -1, d)[:, :, :L]
    vf = (v[table].float() * vs[table][..., None, None]).permute(0, 2, 1, 4, 3).reshape(n, hk, -1, d)[:, :, :L]
    q, sees, live = _rows(st, torch.float32)
    q = q.reshape(n * hk, hq // hk * m, d)
    s = torch.bmm(q, kf.reshape(n * hk, L, d).transpose(1, 2).contiguous()).view(n, hk, hq // hk, m, L) * (1 / math.sqrt(d))
    s = s.masked_fill_(~sees[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    p = s.sub_(torch.where(torch.isfinite(top), top, torch.zeros_like(top))).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.bmm(p.view(n * hk, -1, L), vf.reshape(n * hk, L, d).contiguous()).view(n, hk, hq // hk, m, d)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    o = o.permute(0, 3, 1, 2, 4).reshape(n * m, hq, d)
    seq, pos = _tokens(st["cu"], st["cu"][1:] - st["cu"][:-1], st["q"].shape[0])
    return o[seq * m + pos].to(st["q"].dtype)


def run(state):
    case = state["case"]
    if not own:
        return {"linear": _plain_linear, "append": _plain_append, "attention": _plain_attention}[case["kind"]](state)
    import paper_2608_23144_amd as awsrc
    if case["kind"] == "linear":
        return awsrc.awsrc_linear_i8(state["x"], state["w"], state["scale"], bias=state["bias"], out_dtype=TYPES[case["out"]])
    cache, kv_len, table = state["cache"], state["kv_len"], state["table"]
    if case["kind"] == "attention":
        return awsrc.awsrc_kv_attention(cache, state["q"], state["cu"], kv_len, table, state["max_new"], state["max_kv"])
    hq, hk, d = HEADS[case["heads"]]
    x = state["qkv"].view(-1, hq + 2 * hk, d)
    q = awsrc.awsrc_kv_append(cache, x[:, hq:hq + hk], x[:, hq + hk:], state["cu"], kv_len, table, state["max_new"],
                              cos=state["cos"], sin=state["sin"], q=x[:, :hq])
    k, v = awsrc.awsrc_kv_read(cache, state["cu_back"], kv_len, table, state["n_back"], state["max_back"], x.dtype)
    return {"q": q, "k": k, "v": v}


# ------------------------------------------------------------------ floors
def work(case):
    if case["kind"] == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": M * K * SIZE[case["x"]] + N * K + 4 * N * (2 if case["bias"] else 1) + M * N * SIZE[case["out"]], "flops": 2 * M * N * K}
    hq, hk, d = HEADS[case["heads"]]
    kv, new = _lengths(case)
    T, b = case["page"], SIZE[case["x"]]
    if case["kind"] == "append":
        back = sum(n - (n - m) // T * T for n, m in zip(kv, new))
        old = back - sum(new)  # tokens that share a block with a new one
        rotated = (hq + hk) * d * sum(new)
        return {"bytes": sum(new) * ((2 * hq + 2 * hk) * d * b + 2 * hk * d + 4 * d) + old * 2 * hk * d + back * 2 * hk * d * b,
                "flops": 3 * rotated + 2 * hk * d * (2 * sum(new) + back)}
    pairs = sum(m * n - m * (m - 1) // 2 for n, m in zip(kv, new))
    blocks = sum(-(-n // T) for n in kv)
    return {"bytes": 2 * sum(kv) * hk * d + 8 * blocks * hk + 2 * sum(new) * hq * d * b, "flops": 4 * pairs * hq * d}


# ------------------------------------------------------------------ the same in 64 bits
def _exact_linear(st):
    out = []
    w = st["w"].double()
    for r in range(0, st["x"].shape[0], 2048):
        x = st["x"][r:r + 2048].double()
        s = x.abs().amax(1, keepdim=True) / torch.full((1, 1), 127.0, dtype=torch.float64, device=DEV)
        y = (torch.round(x / s) @ w.T) * s * st["scale"].double()
        out.append(y if st["bias"] is None else y + st["bias"].double())
    return torch.cat(out)


def _exact_append(st):
    case = st["case"]
    hq, hk, d = HEADS[case["heads"]]
    T = case["page"]
    k, v, ks, vs = st["cache"]
    table, h = st["table"].cpu(), d // 2
    kv, new = _lengths(case)
    qs, got = [], {"k": [], "v": []}
    r = 0
    for b, (n, m) in enumerate(zip(kv, new)):
        x = st["qkv"][r:r + m].double().view(m, hq + 2 * hk, d)
        r += m
        c, s = st["cos"][n - m:n].double()[:, None], st["sin"][n - m:n].double()[:, None]
        y = torch.cat([x[..., :h] * c - x[..., h:] * s, x[..., h:] * c + x[..., :h] * s], -1)
        qs.append(y[:, :hq])
        t0 = (n - m) // T * T  # first token of the first touched block
        pages = table[b, t0 // T:-(-n // T)].long().to(DEV)
        for name, val, codes, scales in (("k", y[:, hq:hq + hk], k, ks), ("v", x[:, hq + hk:], v.transpose(2, 3), vs)):
            was = scales[pages].double()
            if t0 == n - m:
                was[:] = 0
            else:
                was[1:] = 0
            full = torch.zeros(len(pages) * T, hk, d, dtype=torch.float64, device=DEV)
            full[n - m - t0:n - t0] = val
            full = full.view(len(pages), T, hk, d)
            now = torch.maximum(was, full.abs().amax((1, 3)) / 127)
            kept = codes[pages[:1]].double().transpose(1, 2)[:, :n - m - t0]  # old tokens of the first block
            grew = (now[:1] > was[:1])[:, None, :, None]
            step = torch.where(now > 0, now, torch.ones_like(now))[:, None, :, None]
            z = torch.round(full / step)
            z[:1, :n - m - t0] = torch.where(grew, torch.round(kept * was[:1][:, None, :, None] / step[:1]), kept)
            got[name].append((z * now[:, None, :, None]).reshape(-1, hk, d)[:n - t0])
    return {"q": torch.cat(qs), "k": torch.cat(got["k"]), "v": torch.cat(got["v"])}


def _exact_attention(st):
    case = st["case"]
    hq, hk, d = HEADS[case["heads"]]
    T = case["page"]
    k, v, ks, vs = st["cache"]
    kv, new = _lengths(case)
    out = torch.empty(sum(new), hq, d, dtype=torch.float64, device=DEV)
    r = 0
    for b, (n, m) in enumerate(zip(kv, new)):
        pages = st["table"][b, :-(-n // T)].long()
        for h in range(hk):
            kd = (k[pages, h].double() * ks[pages, h].double()[:, None, None]).reshape(-1, d)[:n]
            vd = (v[pages, h].double() * vs[pages, h].double()[:, None, None]).transpose(1, 2).reshape(-1, d)[:n]
            for j in range(h * (hq // hk), (h + 1) * (hq // hk)):
                for i in range(0, m, 2048):
                    e = min(m, i + 2048)
                    sc = st["q"][r + i:r + e, j].double() @ kd.T / math.sqrt(d)
                    sc = sc + torch.triu(torch.full_like(sc, -math.inf), n - m + i + 1)
                    out[r + i:r + e, j] = torch.softmax(sc, -1) @ vd
        r += m
    return out


def exact(case, seed):
    st = prepare(case, seed)
    return {"linear": _exact_linear, "append": _exact_append, "attention": _exact_attention}[case["kind"]](st)
