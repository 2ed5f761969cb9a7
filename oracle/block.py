"""Oracle of the block-scaled 8-bit cache: one unit (batch entry, kv-head) in
plain numpy, one token after the other, attention in fp64.

Written from the definitions: a block of 32 tokens of one side becomes codes
and one scale (fp32 steps, each rounded once); the tokens of the unfinished
block stay as they are."""
import numpy as np

INT8, E4M3 = 0, 1
BLOCK = 32
TINY = np.float32(2.0 ** -126)


def e4m3_values():
    """Value of each of the 256 codes (NaN for the two without one)."""
    v = np.empty(256)
    for code in range(256):
        e, m = (code >> 3) & 15, code & 7
        x = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        if e == 15 and m == 7:
            x = np.nan
        v[code] = -x if code & 128 else x
    return v


E4M3_VALUES = e4m3_values()


def e4m3_round(y):
    """Codes of the e4m3 numbers nearest to y (ties to the even code; beyond
    the largest number, that one)."""
    grid = E4M3_VALUES[:127]                       # 0 .. 448 ascending
    a = np.minimum(np.abs(y).astype(np.float64), grid[-1])
    hi = np.clip(np.searchsorted(grid, a), 1, 126)
    lo = hi - 1
    up = np.where(a - grid[lo] == grid[hi] - a, hi % 2 == 0,
                  grid[hi] - a < a - grid[lo])
    code = np.where(up, hi, lo).astype(np.uint8)
    return code | np.where(np.signbit(y), np.uint8(128), np.uint8(0))


def quantize(fmt, x):
    """fp32 [32][D] -> (codes uint8 [32][D], scale fp32)."""
    x = np.asarray(x, np.float32)
    inverse = np.float32(1 / np.float64(127 if fmt == INT8 else 448))
    scale = np.float32(np.max(np.abs(x)) * inverse)
    if scale < TINY:
        return np.zeros(x.shape, np.uint8), np.float32(0)
    y = (x * np.float32(np.float32(1) / scale)).astype(np.float32)
    if fmt == INT8:
        return np.clip(np.rint(y), -127, 127).astype(np.int8).view(np.uint8), scale
    return e4m3_round(y), scale


def decode(fmt, codes):
    """Numbers the codes stand for before their scale."""
    codes = np.asarray(codes, np.uint8)
    return (codes.view(np.int8).astype(np.float32) if fmt == INT8
            else E4M3_VALUES[codes].astype(np.float32))


class Unit:
    """Cache of one (batch entry, kv-head).  Rows enter as fp32 (exact copies
    of 16-bit numbers)."""

    def __init__(self, fmt, D, narrow):
        """narrow: fp32 array -> fp32 array rounded to the cache's dtype."""
        self.fmt, self.D, self.narrow = fmt, D, narrow
        self.codes = [np.zeros((0, D), np.uint8) for _ in range(2)]
        self.scales = [np.zeros(0, np.float32) for _ in range(2)]
        self.tail = [np.zeros((0, D), np.float32) for _ in range(2)]
        self.pos = np.zeros(0, np.int64)
        self.weight = np.zeros(0, np.float64)

    @property
    def length(self):
        return len(self.pos)

    def append(self, k, v):
        for t in range(len(k)):
            for side, x in enumerate((k[t], v[t])):
                self.tail[side] = np.concatenate([self.tail[side], x[None]])
                if len(self.tail[side]) == BLOCK:
                    c, s = quantize(self.fmt, self.tail[side])
                    self.codes[side] = np.concatenate([self.codes[side], c])
                    self.scales[side] = np.append(self.scales[side], s)
                    self.tail[side] = self.tail[side][:0]
            self.pos = np.append(self.pos, self.pos[-1] + 1 if len(self.pos) else 0)
            self.weight = np.append(self.weight, 0.0)

    def values(self, side):
        """fp32 [length][D] that the cache stands for."""
        x = decode(self.fmt, self.codes[side]) * np.repeat(self.scales[side], BLOCK)[:, None]
        return np.concatenate([x.astype(np.float32), self.tail[side]])

    def attend(self, q, scale, cap=0.0, window=0, slopes=None, accumulate=False):
        """q: [n][G][D], the last n tokens' queries -> fp64 [n][G][D]."""
        n, G, _ = q.shape
        K, V = (self.values(s).astype(np.float64) for s in (0, 1))
        first = self.length - n
        out = np.zeros(q.shape)
        for i in range(n):
            t = np.arange(first + i + 1)
            away = (self.pos[first + i] - self.pos[t]).astype(np.float64)
            for g in range(G):
                x = scale * (K[t] @ q[i, g].astype(np.float64))
                if cap:
                    x = cap * np.tanh(x / cap)
                if slopes is not None:
                    x = x - float(slopes[g]) * away
                if window:
                    x = np.where(away < window, x, -np.inf)
                p = np.exp(x - x.max())
                p /= p.sum()
                out[i, g] = p @ V[t]
                if accumulate:
                    self.weight[t] += p
        return out

    def evict(self, keep, sink, recent, weight=None):
        """A unit of the kept tokens (weight: the order's, instead of this
        one's own)."""
        L = self.length
        w = np.asarray(self.weight if weight is None else weight, np.float64)
        if L > keep:
            fixed = [t for t in range(L) if t < sink or t >= L - recent]
            rest = sorted((t for t in range(L) if sink <= t < L - recent),
                          key=lambda t: (-w[t], t))
            slots = np.array(sorted(fixed + rest[:keep - len(fixed)]))
        else:
            slots = np.arange(L)
        to = Unit(self.fmt, self.D, self.narrow)
        for side in (0, 1):
            x = self.values(side)[slots]
            full = len(slots) // BLOCK * BLOCK
            for b in range(0, full, BLOCK):
                c, s = quantize(self.fmt, x[b:b + BLOCK])
                to.codes[side] = np.concatenate([to.codes[side], c])
                to.scales[side] = np.append(to.scales[side], s)
            to.tail[side] = self.narrow(x[full:])
        to.pos, to.weight = self.pos[slots], w[slots]
        return to
