"""The paged 8-bit cache's operators in plain numpy, in 64 bits, written from their
definitions: what its tests compare with."""
import math

import numpy as np

D = 128


def _codes():
    v = np.zeros(256)
    for b in range(128):
        e, m = b >> 3, b & 7
        v[b] = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
    v[127] = np.nan
    v[128:] = -v[:128]
    return v


F8 = _codes()  # the value of every code
_POS = F8[:127]  # ascending


def to_f8(x):
    """Nearest code, ties to the even one, largest 448; NaN for NaN."""
    x = np.asarray(x, np.float64)
    a = np.minimum(np.abs(x), 448.0)
    hi = np.minimum(np.searchsorted(_POS, a), 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - _POS[lo], _POS[hi] - a
    code = np.where((dh < dl) | ((dh == dl) & (hi % 2 == 0)), hi, lo)
    return np.where(np.isnan(x), 127, code + 128 * np.signbit(x)).astype(np.uint8)


def scale_exp(amax):
    """Least e with amax <= 448 * 2^e, within the limits."""
    e = -100
    while e < 119 and amax > 448.0 * 2.0 ** e:
        e += 1
    return e


class Pool:
    """Pages in the layout of moba_cache, as numpy arrays (K and V as codes)."""

    def __init__(self, n, hkv, page, fill=0x7f):
        self.n, self.hkv, self.page = n, hkv, page
        self.k = np.full((n, hkv, page, D), fill, np.uint8)
        self.v = np.full((n, hkv, page // 64, D, 64), fill, np.uint8)
        self.k_scale = np.full((n, hkv), np.nan, np.float32)
        self.v_scale = np.full((n, hkv), np.nan, np.float32)
        self.k_sum = np.full((n, hkv, D), np.nan, np.float32)

    def copy(self):
        p = Pool(1, self.hkv, self.page)
        p.n = self.n
        for x in ("k", "v", "k_scale", "v_scale", "k_sum"):
            setattr(p, x, getattr(self, x).copy())
        return p

    def keys(self, page, g, scaled=True):
        x = F8[self.k[page, g]]
        return x * float(self.k_scale[page, g]) if scaled else x

    def values(self, page, g):
        return F8[self.v[page, g].transpose(0, 2, 1).reshape(self.page, D)] * float(self.v_scale[page, g])


def plan(add, lens, table, free, num_free, page, T):
    """(cu, slots, lens, num_free, refused); table and free change in place."""
    S, W = table.shape
    n = int(num_free)
    held = [-(-int(x) // page) for x in lens]
    new_lens, slots = np.array(lens), np.full(T, -1, np.int64)
    for s in range(S):
        if add[s] < 0:
            free[n:n + held[s]] = table[s, :held[s]]
            n += held[s]
            new_lens[s] = 0
    cu, refused, short = [0], 0, False
    for s in range(S):
        a = max(int(add[s]), 0)
        t0 = cu[-1]
        cu.append(t0 + a)
        if add[s] < 0:
            continue
        total = int(lens[s]) + a
        need = -(-total // page) - held[s]
        fits = held[s] + need <= W and t0 + a <= T
        if fits and need > n:
            short = True  # the list holds too few for it, and for all after it that need one
        if not fits or (short and need > 0):
            refused += 1
            continue
        for j in range(held[s], held[s] + need):
            n -= 1
            table[s, j] = free[n]
        new_lens[s] = total
        for i in range(a):
            pos = int(lens[s]) + i
            slots[t0 + i] = int(table[s, pos // page]) * page + pos % page
    return np.minimum(cu, T), slots, new_lens, n, refused


def write(k, v, slots, pool):
    """k, v [T, Hkv, D] float64; changes the pool in place."""
    P, T = pool.page, len(slots)
    t = 0
    while t < T:
        slot = int(slots[t])
        if not 0 <= slot < pool.n * P:
            t += 1
            continue
        page, o = divmod(slot, P)
        n = 1
        while o + n < P and t + n < T and slots[t + n] == slot + n:
            n += 1
        for g in range(pool.hkv):
            for name, x in (("k", k[t:t + n, g]), ("v", v[t:t + n, g])):
                fine = np.isfinite(x)
                e = scale_exp(np.max(np.abs(x), where=fine, initial=0.0))
                codes = getattr(pool, name)[page, g]
                if name == "v":
                    codes = codes.transpose(0, 2, 1).reshape(P, D)  # a copy
                scale = getattr(pool, name + "_scale")
                if o > 0:
                    was = int(round(math.log2(float(scale[page, g]))))
                    e = max(e, was)
                    if e > was:
                        codes[:o] = to_f8(F8[codes[:o]] * 2.0 ** (was - e))
                codes[o:o + n] = to_f8(np.where(fine, np.where(fine, x, 0.0) * 2.0 ** -e, np.nan))
                scale[page, g] = 2.0 ** e
                if name == "v":
                    pool.v[page, g] = codes.reshape(P // 64, 64, D).transpose(0, 2, 1)
                else:
                    pool.k_sum[page, g] = (F8[codes[:o + n]].sum(0) * 2.0 ** e).astype(np.float32)
        t += n


def decode(q, pool, table, lens, block, topk):
    """out [S, Hq, D], lse [Hq, S], and per row: mass [S, Hq, D] (the weighted sum of |v|),
    size [S, Hq] (the largest sum of |q k| / sqrt(D) log2(e) over the attended keys), keys
    [S, Hq] (their number) and peak [S, Hq] (the largest |v|)."""
    S, Hq = q.shape[:2]
    G, P, W = Hq // pool.hkv, pool.page, table.shape[1]
    out, mass = np.zeros((S, Hq, D)), np.zeros((S, Hq, D))
    lse = np.full((Hq, S), -np.inf)
    size, count, peak = np.zeros((S, Hq)), np.zeros((S, Hq), np.int64), np.zeros((S, Hq))
    for s in range(S):
        L = min(max(int(lens[s]), 0), W * P)
        if L == 0:
            continue
        ids = [int(x) for x in table[s, :-(-L // P)]]
        for g in range(pool.hkv):
            pos, ks, vs = [], [], []
            for j, p in enumerate(ids):
                if 0 <= p < pool.n:
                    m = min(P, L - j * P)
                    pos += range(j * P, j * P + m)
                    ks.append(pool.keys(p, g)[:m])
                    vs.append(pool.values(p, g)[:m])
            if not pos:
                continue
            pos, ks, vs = np.array(pos), np.concatenate(ks), np.concatenate(vs)
            for h in range(g * G, (g + 1) * G):
                use = np.ones(len(pos), bool)
                nblk = -(-W * P // block) if topk else 0
                if topk and topk < nblk:
                    cur, per = (L - 1) // block, block // P
                    sc = []
                    for j in range(cur):
                        rows = [pool.k_sum[p, g].astype(np.float64) for p in ids[j * per:(j + 1) * per]
                                if 0 <= p < pool.n]
                        x = float(q[s, h] @ np.sum(rows, axis=0)) if rows else 0.0
                        sc.append(-np.inf if np.isnan(x) else x)
                    kept = sorted(range(cur), key=lambda j: (-sc[j], j))[:topk - 1] + [cur]
                    use = np.isin(pos // block, kept)
                if not use.any():
                    continue
                z = ks[use] @ q[s, h] / math.sqrt(D)
                m = z.max()
                p = np.exp(z - m)
                l = p.sum()
                out[s, h] = p @ vs[use] / l
                mass[s, h] = p @ np.abs(vs[use]) / l
                lse[h, s] = m + np.log(l)
                size[s, h] = (np.abs(ks[use]) @ np.abs(q[s, h])).max() / math.sqrt(D) * math.log2(math.e)
                count[s, h] = use.sum()
                peak[s, h] = np.abs(vs[use]).max()
    return out, lse, mass, size, count, peak


def check_decode(got, got_lse, ref, what=""):
    """The kernel's rounding, counted.  A logit (log2 domain) of size A = sum |q k| scale is an
    fp32 sum of 128 exact products (each partial sum off by 2^-23 at most, also where the
    matrix core cuts off), scaled and taken from the maximum, all within 132 * 2^-23 A; a
    weight is off by ln 2 times that, 2^-22 of its exponential, and 2^-16 by its two bf16
    terms (half a step of 2^-8 twice).  Sums over n keys: n 2^-23 each of weights and of
    weighted values; joins and the running maximum: a few 2^-23 (64 allowed).  So |out - ref|
    <= w * mass (weights, twice: numerator and sum) and the rounding to bf16, 2^-8 of the
    value; lse within w of its sum and 2^-23 of itself.
    Weights (relative to the largest) below fp32's smallest normal number, 2^-126, may be 0:
    at most n times that, of the largest |v|, is lost, whatever the other weights add up to
    (a row whose largest weight meets a value 0 shows it); bf16's own smallest step is 2^-133."""
    out, lse, mass, size, count, peak = ref
    u = 2.0 ** -23
    w = 132 * u * size + (2 * count + 64) * u
    tol = (2 * w + 2.0 ** -16)[..., None] * mass
    tol += (2.0 ** -126 * count * peak)[..., None] + 2.0 ** -133
    tol += 2.0 ** -8 * (np.abs(out) + tol)
    err = np.abs(got - out)
    assert not np.isnan(got).any(), what
    assert (err <= tol).all(), "%s: %g over its tolerance %g" % (what, err[err > tol].max(), tol[err > tol].min())
    fine = np.isfinite(lse)
    assert (np.isneginf(got_lse) == ~fine).all(), what
    e = np.abs(np.where(fine, got_lse - np.where(fine, lse, 0.0), 0.0))
    t = 2 * w.T + 2.0 ** -22 * np.abs(np.where(fine, lse, 0.0)) + 2.0 ** -22
    assert (e <= t).all(), "%s: lse %g" % (what, e.max())
