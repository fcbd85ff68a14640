"""Plain references of the 8-bit serving calls: the fp32 recipe to the bit in
numpy, and the definitions in 64 bits."""
import numpy as np
import torch

TINY = np.float32(2.0 ** -100)


def f32(x):
    return x.detach().float().cpu().numpy()


def scale_of(amax):
    """Recipe scale of largest magnitudes (fp32 array)."""
    amax = np.asarray(amax, np.float32)
    with np.errstate(all="ignore"):
        s = np.where(amax < TINY, np.float32(0), amax / np.float32(127)).astype(np.float32)
    return np.where(np.isfinite(amax), s, np.float32(np.nan)).astype(np.float32)


def inverse(s):
    with np.errstate(all="ignore"):
        return np.where(s == 0, np.float32(0), np.float32(1) / s).astype(np.float32)


def codes(x, inv):
    with np.errstate(all="ignore"):
        r = np.rint((x * inv).astype(np.float32))
    r = np.where(np.isnan(r), 0, r)
    return np.clip(r, -127, 127).astype(np.int8)


def amax(x, axis):
    a = np.abs(x)
    m = np.max(np.where(np.isnan(a), 0, a), axis=axis, initial=0)
    return np.where(np.isnan(a).any(axis=axis), np.float32(np.nan), m).astype(np.float32)


def quantize_rows(x):
    s = scale_of(amax(x, 1))
    return codes(x, inverse(s)[:, None]), s


def rotate(x, pos, cos, sin, interleaved):
    """Rows x [n, heads, D] rotated by their positions, each operation rounded to fp32."""
    if cos is None:
        return x.astype(np.float32)
    half = cos.shape[1]
    y = x.astype(np.float32).copy()
    c = np.full((len(pos), half), np.nan, np.float32)
    s = c.copy()
    ok = (pos >= 0) & (pos < len(cos))
    c[ok], s[ok] = cos[pos[ok]], sin[pos[ok]]
    c, s = c[:, None], s[:, None]
    i0 = np.arange(half) * 2 if interleaved else np.arange(half)
    i1 = i0 + 1 if interleaved else i0 + half
    a, b = y[..., i0].copy(), y[..., i1].copy()
    with np.errstate(all="ignore"):
        y[..., i0] = (a * c).astype(np.float32) - (b * s).astype(np.float32)
        y[..., i1] = (b * c).astype(np.float32) + (a * s).astype(np.float32)
    return y


def append(cache, k, v, q, cu, kv_len, table, cos, sin, interleaved):
    """The cache (numpy arrays k, v, k_scale, v_scale) after the call, in place, and the rotated queries in fp32."""
    ck, cv, ks, vs = cache
    T, pages = ck.shape[2], ck.shape[0]
    pos = np.full(len(k), -1, np.int64)
    for s in range(len(kv_len)):
        n = cu[s + 1] - cu[s]
        pos[cu[s]:cu[s + 1]] = kv_len[s] - n + np.arange(n)
    kr = rotate(k, pos, cos, sin, interleaved)
    for s in range(len(kv_len)):
        rows = [r for r in range(cu[s], cu[s + 1]) if pos[r] >= 0]
        for slot in sorted({int(pos[r]) // T for r in rows}):
            if slot >= table.shape[1] or not 0 <= table[s, slot] < pages:
                continue
            p = table[s, slot]
            mine = [r for r in rows if pos[r] // T == slot]
            at = [int(pos[r]) % T for r in mine]
            for h in range(ck.shape[1]):
                for x, c, sc in ((kr, ck[p, h], ks), (v, cv[p, h].T, vs)):
                    fresh = scale_of(amax(x[mine][:, h].reshape(1, -1), 1))[0]
                    was = np.float32(0) if at[0] == 0 else sc[p, h]
                    now = fresh if fresh > was or np.isnan(fresh) else was
                    inv = inverse(np.float32(now))
                    if now > was and at[0] > 0:
                        c[:at[0]] = codes(c[:at[0]].astype(np.float32), np.float32(was * inv))
                    c[at] = codes(x[mine][:, h].astype(np.float32), inv)
                    sc[p, h] = now
    return rotate(q, pos, cos, sin, interleaved) if q is not None else None


def dense(cache, s, table, n, h):
    """Keys and values of the first n tokens of a sequence in 64 bits, and which of them are there."""
    ck, cv, ks, vs = cache
    T, D = ck.shape[2], ck.shape[3]
    k, v, ok = np.zeros((n, D)), np.zeros((n, D)), np.zeros(n, bool)
    for t in range(n):
        if t // T >= table.shape[1] or not 0 <= table[s, t // T] < ck.shape[0]:
            continue
        p = table[s, t // T]
        k[t] = ck[p, h, t % T].astype(np.float64) * np.float64(ks[p, h])
        v[t] = cv[p, h, :, t % T].astype(np.float64) * np.float64(vs[p, h])
        ok[t] = True
    return k, v, ok


def attention(cache, q, cu, kv_len, table, scale, causal):
    """(outputs, bound on the kernel's error before the output's rounding), both [rows, heads, D] in 64 bits.

    The bound: p is rounded to fp16 (2^-11 of itself, 2^-25 at least), its exponent carries the fp32 sum of D exact products
    (D + 8 roundings of sum |q k| scale, counted against the running maximum too), the fp32 sums over the tokens and the
    joins add 2^-24 for each of n + 16 terms."""
    hk, D = cache[0].shape[1], cache[0].shape[3]
    heads = q.shape[1]
    G = heads // hk
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    for s in range(len(kv_len)):
        n, m = int(kv_len[s]), int(cu[s + 1] - cu[s])
        for h in range(hk):
            k, v, ok = dense(cache, s, table, n, h)
            for g in range(G):
                for i in range(m):
                    r = cu[s] + i
                    lim = min(n, n - m + i + 1) if causal else n
                    if lim <= 0 or not ok[:lim].any():
                        continue
                    see = np.nonzero(ok[:lim])[0]
                    x = q[r, h * G + g].astype(np.float64)
                    sc = k[see] @ x * scale
                    p = np.exp(sc - sc.max())
                    p /= p.sum()
                    out[r, h * G + g] = p @ v[see]
                    mag = (np.abs(k[see]) @ np.abs(x)).max() * abs(scale)
                    rel = 2.0 ** -11 + 2 * (D + 8) * 2.0 ** -24 * mag + (len(see) + 16) * 2.0 ** -23
                    tol[r, h * G + g] = rel * (p @ np.abs(v[see])) + len(see) * 2.0 ** -25 * np.abs(v[see]).max()
    return out, tol
