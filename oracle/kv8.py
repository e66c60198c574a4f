"""Plain float64 definition of a KV page held in e4m3.

TEST INFRASTRUCTURE ONLY: never imported by the product path.

A page holds up to 16 tokens of one head's keys (or values) under one scale
2^e: e is the smallest integer in [-100, 119] with |x| <= 448 2^e for every
finite value written, and never falls while the page keeps earlier tokens. A
value is held as the e4m3 number nearest to x 2^-e (ties to even); a non-finite
value is held as NaN. When e grows, the numbers held are rounded again.

e4m3 here is the OCP format: sign, 4 exponent bits of bias 7, 3 fraction bits,
no infinities, largest number 448, 0x7f and 0xff NaN.
"""
import numpy as np

PAGE = 16
MAX = 448.0


def table() -> np.ndarray:
    """The number each byte stands for."""
    b = np.arange(256)
    s, e, f = b >> 7, (b >> 3) & 15, b & 7
    x = np.where(e == 0, f * 2.0 ** -9, (1 + f / 8.0) * 2.0 ** (e.astype(float) - 7))
    x = np.where(s == 1, -x, x)
    x[(b & 127) == 127] = np.nan
    return x


def nearest(x: np.ndarray) -> np.ndarray:
    """The e4m3 number nearest to x (|x| <= 448), ties to the even fraction; NaN where x is not finite."""
    x = np.asarray(x, dtype=np.float64)
    a = np.abs(np.where(np.isfinite(x), x, 0.0))
    # numbers 2^k (1 + f / 8), k >= -6, and multiples of 2^-9 below 2^-6
    step = 2.0 ** (np.floor(np.log2(np.maximum(a, 2.0 ** -6))) - 3)
    y = np.minimum(np.round(a / step) * step, MAX)  # numpy's round is half to even
    return np.where(np.isfinite(x), np.copysign(y, x), np.nan)


def exponent(amax: float) -> int:
    if not amax > 0:
        return -100
    e = int(np.floor(np.log2(amax))) - 10
    while amax > MAX * 2.0 ** e:
        e += 1
    return min(max(e, -100), 119)


class Page:
    """One head's keys or values of one page."""

    def __init__(self, hd: int):
        self.hd, self.e, self.x = hd, None, np.zeros((0, hd))  # x: the e4m3 numbers held

    def append(self, rows: np.ndarray):
        rows = np.asarray(rows, dtype=np.float64)
        finite = np.where(np.isfinite(rows), np.abs(rows), 0.0)
        e = exponent(float(finite.max()))
        if len(self.x):
            e = max(e, self.e)
            if e > self.e:
                self.x = nearest(self.x * 2.0 ** (self.e - e))
        self.e = e
        new = np.where(np.isfinite(rows), np.clip(rows * 2.0 ** -e, -MAX, MAX), np.nan)
        self.x = np.concatenate([self.x, nearest(new)])

    def truncate(self, n: int):
        self.x = self.x[:n]

    def values(self) -> np.ndarray:
        return self.x * 2.0 ** (self.e if self.e is not None else 0)


class Sequence:
    """Keys or values of one sequence: pages of every head."""

    def __init__(self, n_kv: int, hd: int):
        self.n_kv, self.hd, self.len, self.pages = n_kv, hd, 0, []

    def append(self, rows: np.ndarray):
        """rows [n, n_kv, hd], one call's new tokens."""
        i = 0
        while i < len(rows):
            slot = self.len % PAGE
            n = min(PAGE - slot, len(rows) - i)
            if slot == 0:
                self.pages = self.pages[:self.len // PAGE] + [[Page(self.hd) for _ in range(self.n_kv)]]
            for h in range(self.n_kv):
                self.pages[self.len // PAGE][h].append(rows[i:i + n, h])
            self.len += n
            i += n

    def truncate(self, n: int):
        self.len = n
        self.pages = self.pages[:(n + PAGE - 1) // PAGE]
        if n % PAGE:
            for p in self.pages[-1]:
                p.truncate(n % PAGE)

    def values(self) -> np.ndarray:
        """[len, n_kv, hd]"""
        if not self.len:
            return np.zeros((0, self.n_kv, self.hd))
        return np.concatenate([np.stack([p.values() for p in page], axis=1) for page in self.pages])[:self.len]
