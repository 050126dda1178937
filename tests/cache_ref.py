"""Plain 64-bit reference of the session cache's calls on CPU tensors, token by token: the format, append, attention,
the tokens' weights, and eviction.  Shares no code with the library."""
import math

import numpy as np
import torch

PAGE = 64


def e4m3_value(byte):
    s, e, m = byte >> 7, byte >> 3 & 15, byte & 7
    if byte & 127 == 127:
        return math.nan
    v = (8 + m) * 2.0 ** (e - 10) if e else m * 2.0 ** -9
    return -v if s else v


VALUES = np.array([e4m3_value(b) for b in range(256)])
_POSITIVE = VALUES[:127]


def round_e4m3(x):
    """Bytes of the nearest e4m3 values (ties to even mantissas) of |x| <= 448; infinities and NaN as 0x7f."""
    x = np.asarray(x, dtype=np.float64)
    a = np.abs(x)
    fine = np.isfinite(a)
    a = np.where(fine, a, 0.0)
    lo = np.clip(np.searchsorted(_POSITIVE, a, side="right") - 1, 0, 126)
    hi = np.minimum(lo + 1, 126)
    below, above = a - _POSITIVE[lo], _POSITIVE[hi] - a
    up = (above < below) | ((above == below) & (hi % 2 == 0))
    b = np.where(up, hi, lo).astype(np.uint8)
    b = np.where(np.signbit(x), b | 128, b).astype(np.uint8)
    return np.where(fine, b, np.uint8(0x7f))


def exponent(x):
    """127 + the least n >= -100 with |x| <= 448 * 2^n for the finite x."""
    a = np.abs(np.asarray(x, dtype=np.float64))
    a = a[np.isfinite(a)]
    top = a.max() if a.size else 0.0
    n = -100
    while top > 448 * 2.0 ** n:
        n += 1
    return 127 + n


class Pool:
    """A pool on the host: bytes k, v [P, H, 64, d], exponents [P, H], weights [P, H, 64]."""

    def __init__(self, k, v, k_exp, v_exp, weight):
        self.k, self.v, self.k_exp, self.v_exp, self.weight = k, v, k_exp, v_exp, weight

    @classmethod
    def of(cls, cache):
        k, v = (t.view(torch.uint8).cpu().numpy().copy() for t in cache[:2])
        return cls(k, v, *(t.cpu().numpy().copy() for t in cache[2:]))

    def arrays(self):
        return {"k": self.k, "v": self.v, "k_exp": self.k_exp, "v_exp": self.v_exp, "weight": self.weight}

    def tokens(self, name, row, length, h):
        """Head h's `length` tokens of a session in 64 bits [length, d]; pages outside the pool are NaN."""
        x, exp = getattr(self, name), getattr(self, name + "_exp")
        out = np.zeros((length, x.shape[3]))
        for p in range(-(-length // PAGE)):
            n = min(PAGE, length - p * PAGE)
            page = int(row[p])
            if not 0 <= page < x.shape[0] or exp[page, h] == 255:
                out[p * PAGE:p * PAGE + n] = math.nan
            else:
                out[p * PAGE:p * PAGE + n] = VALUES[x[page, h, :n]] * 2.0 ** (int(exp[page, h]) - 127)
        return out


def append(pool, k, v, cu, table, lens, width):
    """In place; returns the new lengths.  k, v: 64-bit [T, H, d]."""
    new = list(lens)
    for s, length in enumerate(lens):
        rows = cu[s + 1] - cu[s]
        if not 0 <= length <= PAGE * width or rows < 0 or length + rows > PAGE * width:
            continue
        new[s] = length + rows
        if rows == 0:
            continue
        for p in range(length // PAGE, -(-(length + rows) // PAGE)):
            page = int(table[s][p])
            if not 0 <= page < pool.k.shape[0]:
                continue
            lo, hi = max(length, p * PAGE), min(length + rows, (p + 1) * PAGE)
            a, b = lo - p * PAGE, hi - p * PAGE
            t = cu[s] + lo - length
            for name, x in (("k", k), ("v", v)):
                data, exp = getattr(pool, name), getattr(pool, name + "_exp")
                for h in range(data.shape[1]):
                    was = int(exp[page, h])
                    e = exponent(x[t:t + b - a, h])
                    if a > 0:
                        e = max(e, was)
                        if e != was:
                            data[page, h, :a] = round_e4m3(VALUES[data[page, h, :a]] * 2.0 ** (was - e))
                    data[page, h, a:b] = round_e4m3(x[t:t + b - a, h] * 2.0 ** (127 - e))
                    exp[page, h] = e
            if pool.weight is not None:
                pool.weight[page, :, a:b] = 0
    return new


def attend(pool, q, cu, table, lens, scale):
    """(o, lse, a): a is the attention over |v|, the size that errors of the weights are relative to.  q: 64-bit
    [T, Hq, d]."""
    T, Hq, d = q.shape
    H = pool.k.shape[1]
    o, lse, size = np.zeros((T, Hq, d)), np.full((T, Hq), -math.inf), np.zeros((T, Hq, d))
    for s, n in enumerate(lens):
        rows = slice(cu[s], cu[s + 1])
        if n == 0 or cu[s + 1] == cu[s]:
            continue
        for h in range(H):
            k, v = pool.tokens("k", table[s], n, h), pool.tokens("v", table[s], n, h)
            for hq in range(h * (Hq // H), (h + 1) * (Hq // H)):
                x = scale * (q[rows, hq] @ k.T)
                top = x.max(1, keepdims=True)
                w = np.exp(x - top)
                total = w.sum(1, keepdims=True)
                o[rows, hq] = w @ v / total
                size[rows, hq] = w @ np.abs(v) / total
                lse[rows, hq] = (top + np.log(total))[:, 0]
    return o, lse, size


def weigh(pool, q, lse, cu, table, lens, scale):
    """The pool's weights in 64 bits with the queries' added."""
    out = pool.weight.astype(np.float64)
    Hq, H = q.shape[1], pool.k.shape[1]
    for s, n in enumerate(lens):
        rows = slice(cu[s], cu[s + 1])
        for h in range(H):
            k = pool.tokens("k", table[s], n, h)
            got = np.zeros(n)
            for hq in range(h * (Hq // H), (h + 1) * (Hq // H)):
                got += np.exp(scale * (q[rows, hq] @ k.T) - lse[rows, hq][:, None]).sum(0)
            for j in range(n):
                if 0 <= table[s][j // PAGE] < out.shape[0]:
                    out[table[s][j // PAGE], h, j % PAGE] += got[j]
    return out


def evict(pool, table, lens, new_table, keep, first, last):
    """In place; returns (new lengths, kept [nseq, H, keep])."""
    H = pool.k.shape[1]
    kept = np.full((len(lens), H, keep), -1, dtype=np.int32)
    before = Pool(*(x.copy() for x in (pool.k, pool.v, pool.k_exp, pool.v_exp, pool.weight)))
    for s, n in enumerate(lens):
        m = min(n, keep)
        for h in range(H):
            def rank(j):
                page = int(table[s][j // PAGE])
                w = float(before.weight[page, h, j % PAGE]) if 0 <= page < before.k.shape[0] else -math.inf
                return -math.inf if math.isnan(w) else w
            if n <= keep:
                ids = list(range(n))
            else:
                middle = sorted(range(first, n - last), key=lambda j: (-rank(j), j))[:keep - first - last]
                ids = list(range(first)) + sorted(middle) + list(range(n - last, n))
            kept[s, h, :m] = ids
            for p in range(-(-m // PAGE)):
                page, here = int(new_table[s][p]), ids[p * PAGE:(p + 1) * PAGE]
                if not 0 <= page < pool.k.shape[0]:
                    continue
                for name in ("k", "v"):
                    x = before.tokens(name, table[s], n, h)[here]
                    e = exponent(x)
                    getattr(pool, name)[page, h, :len(here)] = round_e4m3(x * 2.0 ** (127 - e))
                    getattr(pool, name + "_exp")[page, h] = e
                for i, j in enumerate(here):
                    src = int(table[s][j // PAGE])
                    inside = 0 <= src < before.k.shape[0]
                    pool.weight[page, h, i] = before.weight[src, h, j % PAGE] if inside else -math.inf
    return [min(n, keep) for n in lens], kept


def same_values(a, b):
    """Whether two arrays of e4m3 bytes stand for the same values (every NaN byte is one value; -0 equals 0)."""
    return np.array_equal(VALUES[a], VALUES[b], equal_nan=True)
