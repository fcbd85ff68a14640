"""Plain references of the e4m3 codes, the step plan and the draft
verification, written from their definitions: numpy, Python integers, 64 bits."""
import numpy as np

TINY = np.float32(2.0 ** -100)
BLOCK = 128


# ------------------------------------------------------------------ e4m3
def decode(codes):
    """Values of e4m3 codes: sign, 4 exponent bits of bias 7, 3 of mantissa; 0x7F and 0xFF are NaN."""
    c = np.asarray(codes, np.uint8).astype(np.int64)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c & 128, -v, v)


_POSITIVE = decode(np.arange(127))  # increasing, up to 448


def encode(y):
    """Nearest codes of finite values of at most 464 in magnitude, ties to the even code."""
    y = np.asarray(y, np.float64)
    a = np.abs(y)
    hi = np.clip(np.searchsorted(_POSITIVE, a), 0, 126)
    lo = np.clip(hi - 1, 0, 126)
    below, above = a - _POSITIVE[lo], _POSITIVE[hi] - a
    up = (above < below) | ((above == below) & (hi % 2 == 0))
    return (np.where(up, hi, lo) | np.where(np.signbit(y), 128, 0)).astype(np.uint8)


def quantize_blocks(x, block_rows):
    """Codes and scales of fp32 values by the recipe, each operation rounded to fp32."""
    rows, cols = x.shape
    nb, kb = -(-rows // block_rows), -(-cols // BLOCK)
    codes, scale = np.zeros((rows, cols), np.uint8), np.zeros((nb, kb), np.float32)
    for i in range(nb):
        for j in range(kb):
            at = np.s_[i * block_rows:(i + 1) * block_rows, j * BLOCK:(j + 1) * BLOCK]
            b = x[at]
            amax = np.abs(b).max()
            if not np.isfinite(amax):
                scale[i, j] = np.nan
            elif amax >= TINY:
                s = np.float32(amax / np.float32(448))
                scale[i, j] = s
                codes[at] = encode((b * np.float32(np.float32(1) / s)).astype(np.float32))
    return codes, (np.ascontiguousarray(scale.T) if block_rows == 1 else scale)


def values(codes, scale, block_rows):
    """code * scale in 64 bits."""
    rows, cols = codes.shape
    s = scale.T if block_rows == 1 else scale
    s = np.repeat(np.repeat(s.astype(np.float64), block_rows, 0)[:rows], BLOCK, 1)[:, :cols]
    return decode(codes) * s


# ------------------------------------------------------------------ a step's plan
def plan(page, n_pages, free, kv, keep, new, table, rows):
    """The step on Python lists: everything given back is piled on the stack, last slot first, and taken from its top.
    Returns a dict of what awsrc_kv_plan writes; table (numpy) is changed in place."""
    def up(n):
        return -(-n // page)

    most = table.shape[1] * page
    kv = [min(max(0, n), most) for n in kv]
    keep = [min(max(0, k), n) for k, n in zip(keep, kv)]
    new = [max(0, n) for n in new]
    spare = len(free) + sum(max(0, up(n) - up(k + m)) for n, k, m in zip(kv, keep, new))
    served, asked, queued = [], 0, 0
    for n, k, m in zip(kv, keep, new):
        need = max(0, up(k + m) - up(n))
        asked, queued = asked + need, queued + m
        ok = up(k + m) <= table.shape[1] and (need == 0 or asked <= spare) and queued <= rows
        served.append(m if ok else 0)
    given, wanted = [], []
    for s, (n, k, m) in enumerate(zip(kv, keep, served)):
        given += [int(table[s, i]) for i in range(up(k + m), up(n))]
        wanted += [(s, i) for i in range(up(n), up(k + m))]
    pile = list(free) + given[::-1]
    for s, i in wanted:
        table[s, i] = pile.pop()
    cu = np.concatenate([[0], np.cumsum(served)]).astype(np.int32)
    seq, pos = np.full(rows, -1, np.int32), np.full(rows, -1, np.int32)
    slot = np.full(rows, -1, np.int64)
    for s, (k, m) in enumerate(zip(keep, served)):
        for i in range(m):
            r, p = cu[s] + i, int(table[s, (k + i) // page])
            seq[r], pos[r] = s, k + i
            if 0 <= p < n_pages:
                slot[r] = p * page + (k + i) % page
    return {"cu": cu, "seq": seq, "pos": pos, "slot": slot, "kv": np.array([k + m for k, m in zip(keep, served)], np.int32),
            "table": table, "free": pile}


# ------------------------------------------------------------------ drafts
def _counted(w):
    with np.errstate(invalid="ignore"):
        return np.where(np.isfinite(w) & (w > 0), w, 0.0)


def verify(p, q, tokens, u, cu):
    """(tokens that follow, their numbers) from fp32 arrays; products and sums in 64 bits, by definition."""
    p, u = p.astype(np.float64), u.astype(np.float64)
    q = None if q is None else q.astype(np.float64)
    V = p.shape[1]
    out, count = np.full(len(tokens), -1, np.int64), []
    for s in range(len(cu) - 1):
        r, last = int(cu[s]), int(cu[s + 1]) - 1
        if last < r:
            count.append(0)
            continue
        while r < last:
            x = int(tokens[r + 1])
            if not (0 <= x < V and u[r] * (1.0 if q is None else q[r, x]) < p[r, x]):
                break
            out[r] = x
            r += 1
        w = p[r].copy()
        if r < last:
            with np.errstate(invalid="ignore"):
                if q is not None:
                    w = w - q[r]
                elif 0 <= int(tokens[r + 1]) < V:
                    w[int(tokens[r + 1])] -= 1.0
        w = _counted(w)
        if w.sum() == 0:
            w = _counted(p[r])
        if w.sum() > 0:
            c = np.cumsum(w)
            with np.errstate(invalid="ignore"):
                hit = np.flatnonzero((c > u[last] * c[-1]) & (w > 0))
            out[r] = hit[0] if len(hit) else np.flatnonzero(w)[-1]
        count.append(r - int(cu[s]) + 1)
    return out.astype(np.int32), np.array(count, np.int32)
