"""64-bit oracle of the paged 8-bit cache (numpy, written from the formulas):
page resizing, append with power-of-two group scales, attention; and the error
bounds that the GPU tests hold the kernels to."""
import numpy as np

PAGE, GROUP = 64, 16


def e4m3_values():
    """Value of each of the 256 codes: sign, 4 exponent bits (bias 7), 3 mantissa bits; 0x7F and 0xFF are NaN."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    x = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    x[(c & 127) == 127] = np.nan
    return np.where(c & 128, -x, x)


DECODE = e4m3_values()


def e4m3_encode(x):
    """Codes of the nearest values (ties to the even mantissa), infinities and larger saturated at 448, NaN 0x7F."""
    x = np.asarray(x, np.float64)
    a = np.minimum(np.abs(x), 448.0)
    e = np.maximum(np.floor(np.log2(np.where(a > 0, a, 1.0))), -6)
    q = np.rint(a / 2.0 ** (e - 3)) * 2.0 ** (e - 3)             # rint: ties to even multiples of the step
    mag = np.searchsorted(DECODE[:127], np.where(np.isnan(q), 0.0, q))
    code = np.where(np.signbit(x), 128 + mag, mag)
    return np.where(np.isnan(x), 127, code).astype(np.uint8)


def pow2_scale(amax):
    """Smallest 2^e, -100 <= e <= 120, with amax / 2^e <= 448; 1 for 0."""
    if amax == 0:
        return 1.0
    e = -100
    while amax / 2.0 ** e > 448.0 and e < 120:
        e += 1
    return 2.0 ** e


class Cache:
    """Codes [page][head][token][channel] and scales [page][head][group]."""

    def __init__(self, pages, heads, dh, rng=None):
        shape = (pages, heads, PAGE, dh)
        self.code = {n: (rng.integers(0, 256, shape) if rng else np.zeros(shape)).astype(np.uint8) for n in "kv"}
        self.scale = {n: np.ones((pages, heads, PAGE // GROUP)) for n in "kv"}

    def append(self, k, v, slots):
        r = 0
        while r < len(slots):
            if slots[r] < 0:
                r += 1
                continue
            n = 1
            while r + n < len(slots) and slots[r + n] // GROUP == slots[r] // GROUP and slots[r + n] >= 0:
                n += 1
            run, top = [], -1
            for i in range(r, r + n):
                if slots[i] % GROUP > top:
                    top = slots[i] % GROUP
                    run.append(i)
            page, grp, t0 = slots[r] // PAGE, slots[r] % PAGE // GROUP, slots[r] % GROUP
            for name, rows in (("k", k), ("v", v)):
                for h in range(rows.shape[1]):
                    codes = self.code[name][page, h, grp * GROUP:(grp + 1) * GROUP]
                    vals = {t: DECODE[codes[t]] * self.scale[name][page, h, grp] for t in range(t0)}
                    vals.update({slots[i] % GROUP: rows[i, h].astype(np.float64) for i in run})
                    every = np.abs(np.stack(list(vals.values())))
                    s = pow2_scale(np.where(np.isfinite(every), every, 0.0).max())
                    for t, x in vals.items():
                        codes[t] = e4m3_encode(x / s)
                    self.scale[name][page, h, grp] = s
            r += n

    def values(self, name):
        return DECODE[self.code[name]] * np.repeat(self.scale[name], GROUP, 2)[..., None]


def attention(cache, table, kv_len, row_start, q, causal, scale, num_pages=None):
    """(out, A, S): A = sum p |v| / sum p per channel, S = the row's largest sum of |q||k| scale over seen keys."""
    k, v = cache.values("k"), cache.values("v")
    hkv, G = k.shape[1], q.shape[1] // k.shape[1]
    out, A, S = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape[:2])
    for s in range(len(kv_len)):
        a, b, n = row_start[s], row_start[s + 1], kv_len[s]
        pos = np.arange(n)
        pages = table[s, pos // PAGE] if n else np.zeros(0, int)
        fine = (pages >= 0) & (pages < k.shape[0])
        for r in range(a, b):
            at = n - (b - a) + r - a
            see = fine & ((pos <= at) if causal else np.ones(n, bool))
            p_, t_ = pages[see], pos[see] % PAGE
            if not len(p_):
                continue
            for h in range(hkv):
                kk, vv = k[p_, h, t_], v[p_, h, t_]
                for g in range(G):
                    x = q[r, h * G + g].astype(np.float64)
                    z = kk @ x * scale
                    w = np.exp(z - z.max())
                    w /= w.sum()
                    out[r, h * G + g] = w @ vv
                    A[r, h * G + g] = w @ np.abs(vv)
                    S[r, h * G + g] = (np.abs(kk) @ np.abs(x)).max() * scale
    return out, A, S


def attention_bound(out, A, S, dtype, dh, keys):
    """How far a row may be from the 64-bit one.  Scores: each a sum of dh fp32 products (and their scales and
    the reference's subtraction), off by at most (dh + 8) 2^-24 S, which moves a weight by that relative amount
    in numerator and sum each; exp2 and log2 instructions 2^-21.  Weights rounded to fp16 (2^-11) or two of them
    (2^-22).  Sums of `keys` fp32 terms in numerator and denominator: 2 keys 2^-24.  The output is rounded once
    (half a step: 2^-8 bf16, 2^-24 fp32) after a division (2^-23)."""
    p = 2.0 ** -11 if dtype == "bf16" else 2.0 ** -22
    rel = 2 * (dh + 8) * 2.0 ** -24 * S[..., None] + 2.0 ** -20 + p + 2 * keys * 2.0 ** -24
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    return (half + 2.0 ** -23) * (np.abs(out) + rel * A) + rel * A + 1e-30


class Pages:
    """Plain page rows and free stack; resize as the header describes it."""

    def __init__(self, table, held, free):
        self.table, self.held, self.free = table.copy(), list(held), list(free)

    def resize(self, seq_len, new_len, cap=None):
        """Slots (None where cap is) and whether every sequence fitted."""
        n, width = len(seq_len), self.table.shape[1]
        new = list(new_len) if new_len is not None else [0] * n
        ok = [a >= 0 and b >= 0 and -(-(a + b) // PAGE) <= width for a, b in zip(seq_len, new)]
        target = [-(-(a + b) // PAGE) for a, b in zip(seq_len, new)]
        back = [(s, i) for s in range(n) if ok[s] for i in range(target[s], self.held[s])]
        for s, i in reversed(back):
            self.free.append(int(self.table[s, i]))
            self.table[s, i] = -1
        for s in range(n):
            if ok[s]:
                self.held[s] = min(self.held[s], target[s])
        stuck = False
        for s in range(n):
            want = target[s] - self.held[s] if ok[s] else 0
            if want > 0 and (stuck or want > len(self.free)):
                stuck, ok[s] = True, False
            elif want > 0:
                for i in range(want):
                    self.table[s, self.held[s] + i] = self.free.pop()
                self.held[s] += want
        slots = []
        for s in range(n):
            for j in range(max(new[s], 0)):
                p = seq_len[s] + j
                slots.append(int(self.table[s, p // PAGE]) * PAGE + p % PAGE if ok[s] else -1)
        starts = np.concatenate([[0], np.cumsum([max(x, 0) for x in new])])
        if cap is not None:
            slots, starts = slots[:cap], np.minimum(starts, cap)
        return slots, starts, all(ok)
