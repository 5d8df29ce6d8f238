"""Plain forms of the attention calls in 64 bits (numpy), and the inputs of their tests."""

import numpy as np

E4M3 = np.array([(-1.0 if b >> 7 else 1.0) * (np.nan if b & 127 == 127 else (b & 7) * 2.0**-9 if (b >> 3 & 15) == 0
                                              else (8 + (b & 7)) * 2.0**((b >> 3 & 15) - 10)) for b in range(256)])


def round_e4m3(x):
    """Values of at most 448 to the nearest e4m3 value, ties to even; what is not finite to NaN."""
    x = np.asarray(x, np.float64)
    e = np.maximum(np.frexp(x)[1] - 1, -6)
    with np.errstate(invalid="ignore"):
        return np.where(np.isfinite(x), np.round(x / 2.0**(e - 3)) * 2.0**(e - 3), np.nan)


def need_scale(amax):
    """The least 2^e >= 2^-100 with amax <= 448 * 2^e."""
    m, e = np.frexp(np.asarray(amax, np.float64) / 448.0)
    e = np.where(np.asarray(amax) > 0, np.maximum(np.where(m == 0.5, e - 1, e), -100), -100)
    return 2.0**e.astype(np.float64)


def plan(p, c, B, free, table, n_slots):
    """lv_kv_plan, request by request."""
    p, c, table = np.asarray(p, np.int64), np.asarray(c, np.int64), np.array(table, np.int64)
    offsets, slots, E = [0], [], 0
    for i in range(len(p)):
        held, total = -(-c[i] // B), -(-(c[i] + p[i]) // B)
        ok = E + total - held <= len(free)
        for k in range(held, total):
            table[i, k] = free[E + k - held] if ok else -1
        E += total - held
        for pos in range(c[i], c[i] + p[i]):
            b = table[i, pos // B]
            slots.append(b * B + pos % B if b >= 0 else -1)
        offsets.append(len(slots))
    n = len(slots)
    return table, np.array(offsets), np.array(slots + [-1] * (n_slots - n), np.int64), np.array([n, E])


def store(values, scales, x, slots, B):
    """lv_kv_store of one tensor: values [blocks][heads][B][d] (what the codes stand for), scales [blocks][heads]."""
    values, scales, t = values.copy(), scales.copy(), 0
    while t < len(slots):
        if slots[t] < 0:
            t += 1
            continue
        n = 1
        while t + n < len(slots) and slots[t + n] == slots[t] + n and slots[t + n] % B:
            n += 1
        b, off = divmod(int(slots[t]), B)
        new = x[t:t + n].transpose(1, 0, 2)
        s = need_scale(np.where(np.isfinite(new), np.abs(new), 0).max((1, 2)))
        if off:
            s = np.maximum(s, scales[b])
            grew = s > scales[b]
            again = round_e4m3(values[b, :, :off] * (scales[b] / s)[:, None, None])
            values[b, :, :off] = np.where(grew[:, None, None], again, values[b, :, :off])
        values[b, :, off:off + n] = round_e4m3(new / s[:, None, None])
        scales[b] = s
        t += n
    return values, scales


def attend_rows(q, K, V, seen, scale, dtype, d):
    """Rows q [R][d] on keys K, V [n][d], seen [R][n]: o, lse and how far a kernel that sums in fp32 and rounds a weight
    and its output to the 16-bit type may be from them.

    With u the type's half unit in the last place, relative to the least value that has it (2^-8 for bf16, which has 8
    significant bits, 2^-11 for f16, which has 11): the output's own rounding is u |o|; a
    weight's is u each, so at most u sum w|v|; the scores' sums of d products (in fp32, each partial sum cut rather than
    rounded: 2^-22) move a weight by at most twice d 2^-22 max scale sum|q||k|; the sums over keys and the softmax's own
    arithmetic by less than 2^-16 (its exponential is good to 2^-22, its running maximum multiplies that by the number of
    times it grows, a few tens at most).  A weight below 2^-24 of the row's largest may be lost where it is rounded to f16."""
    o, lse, to, tl = np.zeros(q.shape), np.full(len(q), -np.inf), np.zeros(q.shape), np.zeros(len(q))
    u = 2.0**-8 if dtype == "bf16" else 2.0**-11
    for r in range(len(q)):
        k = np.flatnonzero(seen[r])
        if not len(k):
            continue
        s = scale * (K[k] @ q[r])
        m = s.max()
        w = np.exp(s - m)
        lse[r] = m + np.log(w.sum())
        a = (w @ np.abs(V[k])) / w.sum()
        o[r] = (w @ V[k]) / w.sum()
        ds = 2.0 * d * 2.0**-22 * np.max(abs(scale) * (np.abs(K[k]) @ np.abs(q[r])))
        tiny = 2.0**-24 * np.abs(V[k]).sum(0) / w.sum()
        to[r] = u * np.abs(o[r]) + (1.01 * u + ds + 2.0**-16) * a + tiny + 2.0**-24
        tl[r] = ds + 2.0**-18 * (1 + abs(lse[r]))
    return o, lse, to, tl


def close(got, want, tol, what):
    """got within tol of want, infinities equal."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert got.shape == want.shape, what
    fine = np.isfinite(want)
    assert np.array_equal(np.isfinite(got), fine), f"{what}: not finite where it should be, or the reverse"
    assert np.array_equal(got[~fine], want[~fine], equal_nan=True), what
    off = np.abs(got[fine] - want[fine]) - np.broadcast_to(tol, want.shape)[fine]
    assert off.size == 0 or off.max() <= 0, f"{what}: {off.max()} beyond its bound"
