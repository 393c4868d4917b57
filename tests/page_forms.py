"""Plain 64-bit forms of the operators around the paged 8-bit store, in numpy and lists."""
import math

import numpy as np

NAN_CODE = 0x7F


def code_values(codes):
    """E4M3 codes (uint8) -> float64."""
    b = np.asarray(codes).astype(np.int64)
    e, m = (b >> 3) & 15, b & 7
    v = np.where(e > 0, (8 + m) * 2.0 ** (e - 10), m * 2.0 ** -9)
    v = np.where((b & 0x7F) == 0x7F, math.nan, v)
    return np.where(b >= 128, -v, v)


_TABLE = code_values(np.arange(127, dtype=np.uint8))  # magnitudes, ascending


def codes_of(y):
    """Nearest codes of float64 numbers, ties to even (of the code), at most 448 in magnitude; NaN for what is not finite."""
    y = np.asarray(y, np.float64)
    a = np.minimum(np.abs(np.nan_to_num(y, nan=0.0, posinf=0.0, neginf=0.0)), 448.0)
    hi = np.clip(np.searchsorted(_TABLE, a), 1, 126)
    lo = hi - 1
    d_lo, d_hi = a - _TABLE[lo], _TABLE[hi] - a  # exact: neighbours are within a factor of two, or below 2^-6
    code = np.where((d_hi < d_lo) | ((d_hi == d_lo) & (hi % 2 == 0)), hi, lo)
    code = np.where(np.signbit(y), code + 128, code)
    return np.where(np.isfinite(y), code, NAN_CODE).astype(np.uint8)


def scale_of(a):
    """The scale of a block whose largest finite magnitude is a."""
    if a == 0:
        return 0.0
    m, e = math.frexp(a / 448)  # the quotient's rounding does not pass a number of four bits: 448 times one is exact
    s = math.ldexp(math.ceil(m * 16) / 16, e)
    assert 448 * s >= a
    return min(max(s, 2.0 ** -117), 2.0 ** 119)


class Pool:
    """A pool in numpy: codes [pages, H, page, d] and scales [pages, H] of K and V."""

    def __init__(self, k_codes, k_scales, v_codes, v_scales):
        self.codes, self.scales = [np.array(k_codes), np.array(v_codes)], [np.array(k_scales, np.float64), np.array(v_scales, np.float64)]
        self.page = self.codes[0].shape[2]

    def append(self, x, which, pages, pos):
        """Rows x [H, n, d] float64 as tokens pos, ... of the sequence whose pages are listed; which: 0 for K, 1 for V."""
        H, n, d = x.shape
        for e in range(pos // self.page, -(-(pos + n) // self.page)):
            p, t0 = pages[e], e * self.page
            lo, hi = max(pos - t0, 0), min(pos + n - t0, self.page)
            for h in range(H):
                rows = x[h, t0 + lo - pos:t0 + hi - pos]
                s = scale_of(np.abs(np.where(np.isfinite(rows), rows, 0.0)).max())
                old = self.scales[which][p, h] if lo else 0.0
                block = self.codes[which][p, h]
                if s > old:
                    if lo:
                        block[:lo] = codes_of(code_values(block[:lo]) * old / s)  # the product has eight bits: exact
                else:
                    s = old
                self.scales[which][p, h] = s
                with np.errstate(invalid="ignore"):
                    block[lo:hi] = codes_of(rows / s if s > 0 else np.where(np.isfinite(rows), rows * 0.0, rows))

    def rows(self, which, pages, tokens):
        """Values [H, len(tokens), d]."""
        H, d = self.codes[which].shape[1], self.codes[which].shape[3]
        out = np.zeros((H, len(tokens), d))
        for i, t in enumerate(tokens):
            p = pages[t // self.page]
            out[:, i] = code_values(self.codes[which][p, :, t % self.page]) * self.scales[which][p][:, None]
        return out


class Pages:
    """Counts and tables as lists, one page after the other."""

    def __init__(self, ref, table):
        self.ref, self.table = [int(x) for x in ref], [[int(x) for x in row] for row in table]
        self.bad = self.none_left = False

    def _lowest(self):
        if 0 in self.ref:
            p = self.ref.index(0)
            self.ref[p] = 1
            return p
        self.none_left = True
        return -1

    def take(self, first, last):
        for c, (a, b) in enumerate(zip(first, last)):
            for e in range(a, b):
                self.table[c][e] = self._lowest()

    def drop(self, first, last):
        for c, (a, b) in enumerate(zip(first, last)):
            for e in range(a, b):
                p, self.table[c][e] = self.table[c][e], -1
                if p == -1:
                    continue
                if not 0 <= p < len(self.ref) or self.ref[p] <= 0:
                    self.bad = True
                else:
                    self.ref[p] -= 1

    def fork(self, src, dst, tokens, page):
        """Returns the copies (from, to)."""
        ok = lambda p: 0 <= p < len(self.ref)  # noqa: E731
        for s, t, n in zip(src, dst, tokens):
            for e in range(n // page):
                p = self.table[s][e]
                self.bad |= not ok(p) and p != -1
                self.table[t][e] = p if ok(p) else -1
                if ok(p):
                    self.ref[p] += 1
        copies = []
        for s, t, n in zip(src, dst, tokens):
            if n % page:
                p = self.table[s][n // page]
                self.bad |= not ok(p) and p != -1
                self.table[t][n // page] = self._lowest() if ok(p) else -1
                if self.table[t][n // page] >= 0:
                    copies.append((p, self.table[t][n // page]))
        return copies

    def compact(self):
        n = sum(r != 0 for r in self.ref)
        moves = list(zip([p for p in range(n, len(self.ref)) if self.ref[p]], [p for p in range(n) if not self.ref[p]]))
        place = dict(moves)
        for row in self.table:
            for e, p in enumerate(row):
                if p != -1 and not 0 <= p < n and p not in place:
                    self.bad = True
                row[e] = place.get(p, p)
        for a, b in moves:
            self.ref[b], self.ref[a] = self.ref[a], 0
        return moves


def seen_tokens(vis, n_sink, begin):
    return [j for j in range(vis) if j < n_sink or j >= begin]


def attention(q, k, v, scale):
    """q [rows, d], k / v [tokens, d] float64: (O, lse, sum p|v|, largest |q||k| scale)."""
    rows, d = q.shape
    if len(k) == 0:
        return np.zeros((rows, d)), np.full(rows, -np.inf), np.zeros((rows, d)), 0.0
    s = q @ k.T * scale
    m = s.max(-1, keepdims=True)
    p = np.exp(s - m)
    z = p.sum(-1, keepdims=True)
    size = float(np.linalg.norm(q, axis=-1).max() * np.linalg.norm(k, axis=-1).max() * scale)
    return p / z @ v, (m + np.log(z))[:, 0], p / z @ np.abs(v), size
